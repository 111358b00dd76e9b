"""A step's operators together, as a program uses them: the example that trains and answers with all of them, streams, captured
graphs, and offsets beyond 32 bits."""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst
from oracle import fp4_oracle, step_oracle as o

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8


def np64(t):
    return t.detach().cpu().double().numpy()


def test_the_example_runs_and_its_gradients_are_those_of_its_parts():
    """Every gradient against torch in 64 bits, from what the step before it gave (the 8-bit products have their own tests)."""
    from examples.tied_step import NormedModel
    model = NormedModel(vocab=300, d=96, tokens=64, p=0.25, max_norm=0.05)
    g = torch.Generator(device="cuda").manual_seed(3)
    model.gain.uniform_(0.5, 1.5, generator=g)
    tokens = torch.randint(0, 300, (64,), device="cuda", generator=g)
    targets = torch.randint(0, 300, (64,), device="cuda", generator=g)
    targets[5] = -1
    y, rows8 = model.stream(tokens, 4, model.p)
    logits = model.projection.logits(rows8, torch.empty(64, 300, device="cuda")).clone()
    loss = model.gradients(tokens, targets, 4)
    log_p, _, _, _ = o.log_probabilities(np64(logits))
    t = targets.cpu().numpy()
    want = -log_p[np.arange(64), np.maximum(t, 0)][t >= 0].mean()
    # 63 log probabilities of 300 logits: about (33 + 60 + 6 log 300) 2^-24 of one each, and the mean's roundings
    assert abs(float(loss) - want) <= 200 * U * abs(want)
    weight = np.where(t >= 0, -1 / 63, 0)
    grad = o.logits_gradient(np64(logits), t, 1.0, weight, weight * 0)
    assert np.abs(np64(model.logits[:64]) - grad).max() <= 200 * U / 63
    # from dy on: the stream's own formula in 64 bits
    x = model.x[:64].double().requires_grad_()
    layer, gain = model.layer.double().requires_grad_(), model.gain.double().requires_grad_()
    kept = torch.ones(64, 96, device="cuda")
    dst.dst_dropout(kept, kept, model.p, model.seed, 9)
    h = x + (x @ layer) * kept.double()
    out = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6) * gain
    (out * model.dy[:64].double()).sum().backward()
    near = lambda a, b: float((a.double() - b).abs().max() / b.abs().max())  # noqa: E731
    # fp32 products of 64 and 96 terms, and the sums of the norm: some hundred roundings
    assert near(model.dlayer, layer.grad) < 300 * U and near(model.dgain, gain.grad) < 400 * U
    into = torch.ones(64, 96, device="cuda")
    dst.dst_dropout(into, into, model.p, model.seed, 8, scale=model.scale)
    assert near(model.values[:64], x.grad * into.double()) < 400 * U
    # the table's gradient is the products' and the value rows'; all are brought down to the largest norm
    given = [t.clone() for t in model.grads.tensors]
    dst.dst_grad_norm(model.grads, model.clip, model.max_norm, model.clip_workspace)
    dst.dst_clip(model.grads, model.clip)
    norm, factor, want = o.clip([np64(t) for t in given], model.max_norm)
    assert abs(float(model.clip[0]) - norm) <= 2 * U * norm and factor < 1
    for a, b in zip(model.grads.tensors, want):
        assert np.abs(np64(a) - b).max() <= 6 * U * np.abs(b).max()


def test_the_example_trains_and_answers():
    from examples.tied_step import NormedModel, train
    losses, right = train(steps=3)
    assert all(np.isfinite(losses)) and 0 <= right <= 1
    again, _ = train(steps=3)
    assert losses == again                                    # the same bits from the same seed
    model = NormedModel(vocab=500, d=64, tokens=32)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, 500, (32,), device="cuda", generator=g)
    drawn, logprob, others, others_logprob = model.answer(tokens, torch.rand(32, device="cuda", generator=g), alternatives=4)
    # the answers' logits are those of the 4-bit forms
    y, _ = model.stream(tokens, 0, 0.0)
    a = fp4_oracle.dequantize(*fp4_oracle.quantize(np64(y)))
    w = fp4_oracle.dequantize(*fp4_oracle.quantize(np64(model.weight)))
    logits, mag = a @ w.T, np.abs(a) @ np.abs(w).T
    tol = (256 + 4 + 16) * 2 * U * mag                        # of the product
    got = np64(model.logits[:32])
    assert (np.abs(got - logits) <= tol).all()
    log_p, _, _, _ = o.log_probabilities(got)
    rows = np.arange(32)
    assert np.abs(np64(logprob) - log_p[rows, drawn.cpu().numpy()]).max() <= 200 * U * np.abs(log_p).max()
    assert np.array_equal(others.cpu().numpy(), o.top_tokens(got, 4))
    assert np.abs(np64(others_logprob) - np.take_along_axis(log_p, others.cpu().numpy(), 1)).max() <= 200 * U * np.abs(log_p).max()


class Calls:
    """One call of every operator on buffers of its own."""

    def __init__(self, seed, rows=40, vocab=3000, d=200):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
        self.logits, self.targets = rand(rows, vocab), torch.randint(0, vocab, (rows,), generator=g).cuda()
        self.x, self.r, self.w, self.table = rand(rows, d), rand(rows, d), rand(d), rand(vocab, d)
        new = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
        self.a, self.logprob, self.stats, self.entropy, self.dlogits, self.back = rand(rows), new(rows), new(rows, 2), new(rows), new(rows, vocab), new(rows, vocab)
        self.top, self.top_logprob = torch.zeros(rows, 7, dtype=torch.int64, device="cuda"), new(rows, 7)
        self.sum, self.y, self.inv, self.dx, self.dw = new(rows, d), new(rows, d), new(rows), new(rows, d), new(d)
        self.nws = torch.empty(dst.dst_rmsnorm_backward_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
        self.grads = dst.TensorList([self.dx, self.dw, self.back])
        self.clip, self.cws = new(2), torch.empty(dst.dst_grad_norm_workspace_bytes(self.grads), dtype=torch.uint8, device="cuda")
        self.clipped = dst.TensorList([torch.zeros_like(t) for t in self.grads.tensors])
        self.q, self.projection, self.out4 = dst.Fp8Matrix(rows, d), dst.TiedProjection(vocab, d, rows, training=False, bits=4), new(rows, vocab)

    def __call__(self, stream=None):
        k = {"stream": stream}
        dst.dst_logprob(self.logits, self.targets, self.logprob, entropy=self.entropy, stats=self.stats, top_tokens=self.top, top_logprob=self.top_logprob, **k)
        dst.dst_logprob_loss(self.logits, self.targets, self.a, None, self.dlogits, **k)
        dst.dst_logprob_backward(self.logits, self.targets, self.stats, self.a, self.back, entropy=self.entropy, dentropy=self.a, **k)
        dst.dst_rmsnorm(self.x, self.w, self.y, q=self.q, residual=self.r, sum_out=self.sum, inv_rms=self.inv, **k)
        dst.dst_rmsnorm_backward(self.y, self.sum, self.w, self.inv, self.dx, dweight=self.dw, workspace=self.nws, **k)
        dst.dst_grad_norm(self.grads, self.clip, 0.5, self.cws, **k)
        dst.dst_clip(self.grads, self.clip, self.clipped, **k)
        self.projection.update(self.table, **k)
        self.projection.logits(self.y, self.out4, **k)

    def results(self):
        return [t.clone() for t in (self.logprob, self.entropy, self.stats, self.top, self.top_logprob, self.dlogits, self.back, self.sum, self.y, self.inv, self.dx, self.dw,
                                    self.clip, *self.clipped.tensors, self.out4)]


def test_work_goes_to_the_stream_that_is_named():
    """Inputs written on a side stream just before the calls on that stream."""
    want = Calls(1)
    want()
    torch.cuda.synchronize()
    c = Calls(1)
    kept = [t.clone() for t in (c.logits, c.x, c.table)]
    for t in (c.logits, c.x, c.table):
        t.fill_(float("nan"))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        for t, k in zip((c.logits, c.x, c.table), kept):
            t.copy_(k)
    c(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(c.results(), want.results()))


def test_captured_and_replayed_and_two_at_once():
    """Two graphs with buffers of their own, replayed on two streams at once and again on new inputs."""
    calls = [Calls(2), Calls(3)]
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs = []
    for c, s in zip(calls, side):
        with torch.cuda.stream(s):
            c()
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                c()
        graphs.append(graph)
    for other in (4, 6):
        fresh = [Calls(other), Calls(other + 1)]
        for c, f in zip(calls, fresh):
            for t, k in zip((c.logits, c.targets, c.x, c.r, c.w, c.table, c.a), (f.logits, f.targets, f.x, f.r, f.w, f.table, f.a)):
                t.copy_(k)
        torch.cuda.synchronize()
        for _ in range(5):
            for graph, s in zip(graphs, side):
                with torch.cuda.stream(s):
                    graph.replay()
        torch.cuda.synchronize()
        for c, f in zip(calls, fresh):
            f()
            assert all(torch.equal(a, b) for a, b in zip(c.results(), f.results()))


def test_rows_more_than_two_to_the_31_elements_apart():
    """Row distances whose byte and element offsets pass 32 bits, in one buffer for inputs and outputs."""
    ld, d = (1 << 31) + 8, 520
    buf = torch.empty(2 * ld + 4 * d, dtype=torch.bfloat16, device="cuda")
    rows = lambda at: buf[at:at + 2 * ld + d].as_strided((3, d), (ld, 1))  # noqa: E731
    x, out, r = rows(0), rows(d), rows(2 * d)
    g = torch.Generator().manual_seed(41)
    x.copy_(torch.randn(3, d, generator=g))
    r.copy_(torch.randn(3, d, generator=g))
    out.zero_()
    targets = torch.tensor([0, 519, 77]).cuda()
    one, logprob, top = torch.ones(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, 5, dtype=torch.int64, device="cuda")
    dst.dst_logprob(x, targets, logprob, top_tokens=top)
    log_p, _, _, _ = o.log_probabilities(np64(x))
    assert np.abs(np64(logprob) - log_p[np.arange(3), targets.cpu().numpy()]).max() <= 200 * U * 8 and np.array_equal(top.cpu().numpy(), o.top_tokens(np64(x), 5))
    dst.dst_logprob_loss(x, targets, one, logprob, out)
    want = o.logits_gradient(np64(x), targets.cpu().numpy(), 1.0, np.ones(3), np.zeros(3))
    assert (np.abs(np64(out) - want) <= H * np.abs(want) + 200 * U).all()
    inv = torch.empty(3, device="cuda")
    h = np64((x.float() + r.float()).bfloat16())
    dst.dst_rmsnorm(x, None, out, residual=r, sum_out=r, inv_rms=inv)
    want, inv64 = o.rmsnorm(h, 1.0, 1e-6)
    assert np.array_equal(np64(r), h) and (np.abs(np64(out) - want) <= (H + 36 * U) * np.abs(want)).all()
    dst.dst_rmsnorm_backward(x, r, None, inv, out)
    want, _ = o.rmsnorm_gradient(np64(x), h, 1.0, np64(inv), 0.0)
    assert (np.abs(np64(out) - want) <= H * np.abs(want) + 200 * U * 4).all()
    q = dst.Fp4Matrix(3, d)
    dst.dst_quantize_fp4(x, q)
    assert np.array_equal(np64(q.codes()), fp4_oracle.quantize(np64(x))[0])
    eye = dst.Fp4Matrix(d, d)
    dst.dst_quantize_fp4(torch.eye(d, device="cuda"), eye)
    ws = torch.empty(max(dst.dst_matmul_fp4_workspace_bytes(3, d, d), 256), dtype=torch.uint8, device="cuda")
    dst.dst_matmul_fp4(q, eye, out, ws)
    assert torch.equal(out.float(), q.dequantize())


def test_tensors_of_more_than_two_to_the_31_elements():
    """2.3 billion elements through quantisation and a thin product, log probabilities, the norm and clipping; rows from all over are checked."""
    n, d = 70000, 32768
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(44)
    pattern = torch.randn(1000, d, generator=g).bfloat16().cuda()
    for i in range(0, n, 1000):
        x[i:i + 1000] = pattern
    at = [0, 1, 65535, 65536, n - 1]
    targets = torch.zeros(n, dtype=torch.int64, device="cuda")
    logprob, stats = torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    dst.dst_logprob(x, targets, logprob, stats=stats)
    assert torch.equal(logprob.view(-1, 1000), logprob[:1000].expand(n // 1000, -1))
    log_p, _, _, _ = o.log_probabilities(np64(x[at]))
    assert np.abs(np64(logprob[at]) - log_p[:, 0]).max() <= 250 * U * 12
    q = dst.Fp4Matrix(n, d)
    dst.dst_quantize_fp4(x, q)
    got = torch.stack([q.part(r + 1, d).q[r] for r in at])
    want = torch.stack([q.q[r % 1000] for r in at])
    assert torch.equal(got, want)
    b = dst.Fp4Matrix(20, d)
    dst.dst_quantize_fp4(torch.randn(20, d, generator=g).cuda(), b)
    y = torch.empty(n, 20, device="cuda")
    dst.dst_matmul_fp4(q, b, y, torch.empty(max(dst.dst_matmul_fp4_workspace_bytes(n, 20, d), 256), dtype=torch.uint8, device="cuda"))
    B = np64(b.dequantize())
    A = fp4_oracle.dequantize(*fp4_oracle.quantize(np64(x[at])))
    assert (np.abs(np64(y[at]) - A @ B.T) <= (256 + 4 * d // 256 + 16) * 2 * U * (np.abs(A) @ np.abs(B).T)).all()
    del q
    grads = dst.TensorList([x])
    clip, ws = torch.empty(2, device="cuda"), torch.empty(dst.dst_grad_norm_workspace_bytes(grads), dtype=torch.uint8, device="cuda")
    dst.dst_grad_norm(grads, clip, 0.5, ws)
    norm = (70 * (np64(pattern) ** 2).sum()) ** 0.5
    assert abs(float(clip[0]) - norm) <= 2 * U * norm
    dst.dst_clip(grads, clip)
    for r in at:
        want = np64(pattern[r % 1000]) * float(clip[1])
        assert (np.abs(np64(x[r]) - want) <= (H + U) * np.abs(want)).all()
