"""GPU parity of the operators around the tied weight against their 64-bit definitions (oracle/tied_oracle.py).

Tolerances, with u = 2^-24 (fp32 rounding) and h = 2^-8 (half a bf16 step, relative):
  dropout    out = r + x (k s): three roundings, each at most u of |x k s| or |out|:   4u (|x k s| + |r|) (+ h |out|)
  embed      out = k (w s + p): three roundings:                                       4u k (|w s| + |p|) (+ h |out|)
  product    terms are exact in fp32 (two 4-bit significands, scales of powers of two); sums of 32 are added up in fp32,
             at worst with truncation (2u an addition: four a block of 128, and up to 128 within the steps of one), and one
             rounding for each stretch moved to registers and each part of the inner dimension:
             (128 + 4 blocks + 16) 2u sum|terms| (+ h |out|)
  quantise   codes and scales are exact
  sample     tokens are exact wherever no decision of the definition is nearer than 2^-18 of the sums to falling
             otherwise (the exponential's error, 2 ulp, is below 2^-21); prob 2^-18
"""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst
from oracle import tied_oracle as o

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def np64(t):
    return t.detach().cpu().double().numpy()


def randn(shape, dtype="f32", seed=0, pad=0, skew=0):
    """A [rows, d] CUDA tensor whose rows are d + pad elements apart and start `skew` elements into the buffer."""
    g = torch.Generator().manual_seed(seed)
    rows, d = shape
    buf = torch.randn(rows * (d + pad) + skew, generator=g).to(TYPES[dtype]).cuda()
    return buf[skew:].view(rows, d + pad)[:, :d]


def empty(shape, dtype="f32", pad=0, skew=0):
    """Like randn, filled with NaN; also the whole buffer, to see what else was written."""
    rows, d = shape
    buf = torch.full((rows * (d + pad) + skew,), float("nan"), dtype=TYPES[dtype], device="cuda")
    return buf[skew:].view(rows, d + pad)[:, :d], buf


def close(got, want, tol, out_type):
    got = np64(got)
    if out_type == "bf16":
        tol = tol + H * np.abs(want)
    bad = ~(np.abs(got - want) <= tol + 1e-37)
    assert not bad.any(), "%d out of tolerance, first at %s: %r against %r" % (bad.sum(), np.argwhere(bad)[0], got[bad][0], want[bad][0])


# ---- dropout ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 8), (3, 7), (5, 64), (4, 255), (2, 256), (7, 257), (33, 1024), (2, 5000)])
@pytest.mark.parametrize("xt,ot,residual", [("f32", "f32", True), ("bf16", "bf16", True), ("bf16", "f32", False), ("f32", "bf16", True)])
@pytest.mark.parametrize("pad,skew", [(0, 0), (8, 0), (3, 1)])
def test_dropout(rows, d, xt, ot, residual, pad, skew):
    p, seed, offset, scale = 0.3, 0xABCDEF0123456789, (3 << 32) + 11, 0.75
    x = randn((rows, d), xt, 1, pad, skew)
    res = randn((rows, d), ot, 2, pad, skew) if residual else None
    out, buf = empty((rows, d), ot, pad, skew)
    dst.dst_dropout(x, out, p, seed, offset, residual=res, scale=scale, row_offset=5)
    k = o.drop_factor(rows, d, p, seed, offset, row_offset=5)
    t = np64(x) * k * scale
    r = np64(res) if residual else np.zeros_like(t)
    close(out, r + t, 4 * U * (np.abs(t) + np.abs(r)), ot)
    assert torch.isnan(buf).sum() == buf.numel() - rows * d                     # nothing beside the rows is written


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -17, 0.5])
def test_dropout_limits(p):
    x = randn((9, 40))
    out, _ = empty((9, 40))
    dst.dst_dropout(x, out, p, 5)
    k = o.drop_factor(9, 40, p, 5)
    close(out, np64(x) * k, 4 * U * np.abs(np64(x) * k), "f32")


def test_dropped_elements_hide_what_they_held():
    x = torch.full((16, 64), float("nan"), device="cuda")
    x[:, ::2] = float("inf")
    out, _ = empty((16, 64))
    dst.dst_dropout(x, out, 0.5, 9)
    k = o.drop_factor(16, 64, 0.5, 9)
    got = np64(out)
    assert (got[k == 0] == 0).all() and not np.isfinite(got[k > 0]).any()


@pytest.mark.parametrize("d", [64, 61])
def test_dropout_in_place_parts_and_offset_in_memory(d):
    x = randn((50, d), seed=3)
    want, _ = empty((50, d))
    dst.dst_dropout(x, want, 0.2, 7, 100)
    y = x.clone()
    dst.dst_dropout(y, y, 0.2, 7, 100)
    assert torch.equal(y, want)
    z = torch.empty_like(x)
    dst.dst_dropout(x[:20], z[:20], 0.2, 7, 100)
    dst.dst_dropout(x[20:], z[20:], 0.2, 7, 100, row_offset=20)
    assert torch.equal(z, want)
    dst.dst_dropout(x, z, 0.2, 7, 58, offset_tensor=torch.tensor([42], device="cuda"))
    assert torch.equal(z, want)
    r = x.clone()
    dst.dst_dropout(x, r, 0.2, 7, 100, residual=r)
    close(r, np64(x) + np64(want), 4 * U * (np.abs(np64(x)) + np.abs(np64(want))), "f32")


def test_dropout_in_a_graph_draws_anew_on_every_replay():
    x, out = randn((8, 64)), torch.empty(8, 64, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        dst.dst_dropout(x, out, 0.5, 3, offset_tensor=step)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            dst.dst_dropout(x, out, 0.5, 3, offset_tensor=step)
            step += 1
    step.zero_()
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(np64(out) != 0, o.drop_factor(8, 64, 0.5, 3, i) != 0)


def test_dropout_gradient_is_the_adjoint_and_the_difference():
    rows, d, p, seed, scale = 6, 48, 0.4, 21, 2.0
    x, g = randn((rows, d), seed=4).round(), randn((rows, d), seed=5).round()
    out, dx, moved = (torch.empty(rows, d, device="cuda") for _ in range(3))
    dst.dst_dropout(x, out, p, seed, scale=scale)
    dst.dst_dropout(g, dx, p, seed, scale=scale)
    inner = lambda a, b: float((a.double() * b.double()).sum())  # noqa: E731
    assert abs(inner(g, out) - inner(dx, x)) <= 8 * U * float((g.double() * out.double()).abs().sum())
    for r, c in ((0, 0), (3, 17), (5, 47), (2, 8)):
        x2 = x.clone()
        x2[r, c] += 1
        dst.dst_dropout(x2, moved, p, seed, scale=scale)
        assert abs(inner(g, moved) - inner(g, out) - float(dx[r, c])) <= 1e-5 * (1 + abs(float(dx[r, c])))


# ---- embedding --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,d,vocab", [(1, 1, 1), (5, 8, 3), (40, 64, 1000), (17, 61, 50), (64, 1024, 200), (3, 1000, 10)])
@pytest.mark.parametrize("wt,ot,it", [("f32", "f32", torch.int64), ("f32", "bf16", torch.int32), ("bf16", "bf16", torch.int64), ("bf16", "f32", torch.int32)])
@pytest.mark.parametrize("positions", [0, 1, 7])
def test_embed(n, d, vocab, wt, ot, it, positions):
    p, seed, scale = 0.25, 99, d ** 0.5
    idx = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(n)).to(it).cuda()
    w = randn((vocab, d), wt, 6)
    pos = randn((positions, d), seed=7) if positions else None
    out, _ = empty((n, d), ot)
    dst.dst_embed(idx, w, out, scale=scale, position=pos, p=p, seed=seed, offset=2, row_offset=1)
    k = o.drop_factor(n, d, p, seed, 2, row_offset=1)
    a = np64(w)[idx.cpu().numpy()] * float(np.float32(scale))
    b = np64(pos)[np.arange(n) % positions] if positions else np.zeros_like(a)
    close(out, k * (a + b), 4 * U * k * (np.abs(a) + np.abs(b)), ot)


def test_embed_out_of_range_rows_are_zero_and_counted():
    idx = torch.tensor([0, -1, 4, 5, 2 ** 40, -2 ** 62], device="cuda")
    w, pos = randn((5, 24)), randn((2, 24))
    out, _ = empty((6, 24))
    result = torch.full((6,), 7, dtype=torch.int32, device="cuda")
    dst.dst_embed(idx, w, out, position=pos, result=result)
    got = np64(out)
    assert (got[[1, 3, 4, 5]] == 0).all() and np.allclose(got[[0, 2]], np64(w)[[0, 4]] + np64(pos)[[0, 0]])
    assert result.tolist() == [4, 0, 4, 0, 0, 0]
    dst.dst_embed(idx[:1], w, out[:1], result=result)
    assert result.tolist() == [0] * 6


def test_embedding_gradient_through_densify_matches_differences():
    """loss = sum g * embed(W): the value rows go through dst_densify; compare with the formula and with differences."""
    n, d, vocab, p, seed, scale = 37, 16, 9, 0.3, 13, 4.0
    idx = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(8)).cuda()
    w, g = randn((vocab, d), seed=9), randn((n, d), seed=10)
    out, values, dw = torch.empty(n, d, device="cuda"), torch.empty(n, d, device="cuda"), torch.empty(vocab, d, device="cuda")
    loss = lambda: float((g.double() * dst.dst_embed(idx, w, out, scale=scale, p=p, seed=seed).double()).sum())  # noqa: E731
    dst.dst_dropout(g, values, p, seed, scale=scale)
    dst.Densifier(n, 1, d, vocab).densify(idx, values, None, dw)
    want = np.zeros((vocab, d))
    terms = np64(g) * o.drop_factor(n, d, p, seed) * scale
    np.add.at(want, idx.cpu().numpy(), terms)
    assert np.abs(np64(dw) - want).max() <= 1e-5 * np.abs(terms).sum(0).max()
    for v, c in ((0, 0), (4, 7), (8, 15)):
        base = loss()
        w[v, c] += 0.5
        assert abs((loss() - base) / 0.5 - want[v, c]) <= 1e-4 * (1 + np.abs(terms).sum())
        w[v, c] -= 0.5


# ---- 8-bit matrices -----------------------------------------------------------------------------------------------
def codes(m):
    return m.q[:, :m.cols].view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 130), (128, 128), (129, 257), (200, 16), (300, 1000)])
@pytest.mark.parametrize("xt,pad,skew", [("f32", 0, 0), ("bf16", 0, 0), ("bf16", 5, 3), ("f32", 4, 1)])
@pytest.mark.parametrize("block", [dst.DST_FP8_ROW, dst.DST_FP8_SQUARE])
@pytest.mark.parametrize("which", ["q", "qt", "both"])
def test_quantize(rows, cols, xt, pad, skew, block, which):
    x = randn((rows, cols), xt, 11, pad, skew)
    x *= torch.logspace(-6, 6, cols, base=2, device="cuda").to(x.dtype)                        # blocks of different magnitude
    q = dst.Fp8Matrix(rows, cols, block) if which != "qt" else None
    qt = dst.Fp8Matrix(cols, rows, block) if which != "q" else None
    dst.dst_quantize_fp8(x, q, qt)
    size = 128 if block else 1
    for m, v in ((q, np64(x)), (qt, np64(x).T)):
        if m is not None:
            want, scale = o.quantize(v, size)
            assert np.array_equal(codes(m), want)
            assert np.array_equal(np64(m.scales()), np.repeat(scale.T, size, 0)[:m.rows])
            assert np.array_equal(np64(m.dequantize()), o.dequantize(want, scale, size))


def test_quantize_limits():
    x = torch.zeros(4, 384, device="cuda")
    x[1, 0], x[1, 200] = 3.0e38, 1e-45
    x[2, 5], x[2, 140], x[2, 300] = float("inf"), float("nan"), 448.0
    x[3, 0], x[3, 1], x[3, 128] = 1.75, 1.0, 1.7500001
    m = dst.Fp8Matrix(4, 384)
    dst.dst_quantize_fp8(x, m)
    want, scale = o.quantize(np64(x), 1)
    ok = np.isfinite(scale.T).repeat(128, 1)
    assert np.array_equal(codes(m)[ok], want[ok]) and np.array_equal(np64(m.scales()), scale.T, equal_nan=True)
    assert np.isnan(np64(m.dequantize())[~ok]).all()


def product(a, b, block_a, block_b, ot, pad=0, skew=0, workspace=True):
    M, K = a.shape
    N = b.shape[0]
    qa, qb = dst.Fp8Matrix(M, K, block_a), dst.Fp8Matrix(N, K, block_b)
    dst.dst_quantize_fp8(a, qa)
    dst.dst_quantize_fp8(b, qb)
    ws = torch.full((max(dst.dst_matmul_fp8_workspace_bytes(M, N, K), 256),), 0xFF, dtype=torch.uint8, device="cuda")
    out, buf = empty((M, N), ot, pad, skew)
    dst.dst_matmul_fp8(qa, qb, out, ws)
    assert torch.isnan(buf).sum() == buf.numel() - M * N
    A, B = np64(qa.dequantize()), np64(qb.dequantize())
    tol = (128 + 4 * -(-K // 128) + 16) * 2 * U * (np.abs(A) @ np.abs(B).T)
    close(out, A @ B.T, tol, ot)
    return out


SHAPES = [(1, 1, 1), (1, 128, 128), (1, 1000, 512), (2, 33, 65), (5, 300, 129), (16, 257, 1024), (17, 129, 128), (31, 500, 100), (33, 128, 640), (64, 700, 96),
          (65, 256, 384), (100, 130, 1000), (127, 255, 127), (128, 256, 128), (129, 257, 129), (200, 1000, 64), (257, 513, 300), (300, 100, 2000), (513, 33, 5000), (40, 40, 9000)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("blocks", [(0, 1), (0, 0), (1, 0), (1, 1)])
@pytest.mark.parametrize("ot,pad,skew", [("f32", 0, 0), ("bf16", 0, 0), ("bf16", 3, 1), ("f32", 5, 1)])
def test_matmul(M, N, K, blocks, ot, pad, skew):
    a = randn((M, K), "f32", 12) * torch.logspace(-4, 4, K, base=2, device="cuda")
    b = randn((N, K), "f32", 13) * torch.logspace(-3, 3, N, base=2, device="cuda").view(-1, 1)
    product(a, b, blocks[0], blocks[1], ot, pad, skew)


@pytest.mark.parametrize("M,N,K", [(1, 33708, 1024), (48, 33708, 512), (300, 33708, 1021), (640, 512, 33708), (2000, 1024, 600), (33708, 64, 500)])
def test_matmul_at_the_vocabulary(M, N, K):
    product(randn((M, K), "bf16", 14), randn((N, K), "bf16", 15), 0, 1 if N > K else 0, "bf16" if M != 1 else "f32")


def test_matmul_is_exact_on_small_whole_numbers_and_repeats_bit_for_bit():
    for M, N, K in ((3, 200, 300), (150, 300, 20000), (260, 520, 256)):
        g = torch.Generator().manual_seed(16)
        a = torch.randint(-7, 8, (M, K), generator=g).float().cuda()
        b = torch.randint(-7, 8, (N, K), generator=g).float().cuda()
        first = product(a, b, 0, 0, "f32")
        assert np.array_equal(np64(first), np64(a) @ np64(b).T)
        x, y = randn((M, K), seed=17), randn((N, K), seed=18)
        assert torch.equal(product(x, y, 0, 1, "f32"), product(x, y, 0, 1, "f32"))


def test_matmul_rows_do_not_depend_on_the_batch():
    """A row's values are those of the same row in another batch of the same kernel (no neighbour leaks in)."""
    b = randn((700, 900), seed=19)
    a = randn((300, 900), seed=20)
    whole = product(a, b, 0, 1, "f32")
    a[77] = float("nan")
    qa, qb = dst.Fp8Matrix(300, 900), dst.Fp8Matrix(700, 900, 1)
    dst.dst_quantize_fp8(a, qa)
    dst.dst_quantize_fp8(b, qb)
    ws = torch.empty(max(dst.dst_matmul_fp8_workspace_bytes(300, 700, 900), 256), dtype=torch.uint8, device="cuda")
    out = torch.empty(300, 700, device="cuda")
    dst.dst_matmul_fp8(qa, qb, out, ws)
    assert torch.isnan(out[77]).all()
    out[77] = whole[77]
    assert torch.equal(out, whole)


def test_matmul_of_nothing():
    out = torch.full((3, 5), float("nan"), device="cuda")
    dst.dst_matmul_fp8(dst.Fp8Matrix(3, 0), dst.Fp8Matrix(5, 0), out)
    assert (out == 0).all()
    dst.dst_matmul_fp8(dst.Fp8Matrix(0, 64), dst.Fp8Matrix(5, 64), torch.empty(0, 5, device="cuda"))


@pytest.mark.parametrize("M,V,D", [(1, 1000, 64), (7, 500, 130), (150, 1000, 512), (300, 2000, 333), (2, 10000, 2048), (5, 9000, 700), (33, 1500, 500), (64, 2000, 512), (17, 40, 64), (3, 8000, 1021)])
@pytest.mark.parametrize("xt,ot", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_projection_and_its_gradients(M, V, D, xt, ot):
    """logits, dx and dweight against the formulas on the 8-bit operands; a smaller batch through the same object."""
    proj = dst.TiedProjection(V, D, M + 20)
    w = randn((V, D), seed=21)
    proj.update(w)
    W = np64(proj.weight.dequantize())
    assert np.array_equal(W, np64(proj.weight_t.dequantize()).T)
    for m in (M, max(1, M // 2)):
        x, dl = randn((m, D), xt, 22), randn((m, V), ot, 23)
        logits, _ = empty((m, V), ot)
        dx, _ = empty((m, D), xt)
        dw, _ = empty((V, D))
        proj.logits(x, logits)
        proj.backward(dl, x, dx, dw)
        rows = lambda v: o.dequantize(*o.quantize(v, 1), 1)  # noqa: E731
        X, DL, XT, DLT = rows(np64(x)), rows(np64(dl)), rows(np64(x).T), rows(np64(dl).T)
        for got, a, b, t in ((logits, X, W.T, ot), (dx, DL, W, xt), (dw, DLT, XT.T, "f32")):
            close(got, a @ b, (128 + 4 * -(-a.shape[1] // 128) + 16) * 2 * U * (np.abs(a) @ np.abs(b)), t)


def test_projection_gradient_against_differences():
    """The loss sum(dl * x W^T) moves as dx and dweight say, up to what 8 bits round (4 significant bits: 2^-4)."""
    M, V, D = 40, 300, 64
    proj = dst.TiedProjection(V, D, M)
    w, x, dl = randn((V, D), seed=24), randn((M, D), seed=25), randn((M, V), seed=26)
    proj.update(w)
    dx, dw = torch.empty(M, D, device="cuda"), torch.empty(V, D, device="cuda")
    proj.backward(dl, x, dx, dw)
    loss = lambda a, b: float((dl.double() * (a.double() @ b.double().T)).sum())  # noqa: E731
    for t, grad, other in ((x, dx, lambda y: loss(y, w)), (w, dw, lambda y: loss(x, y))):
        step = randn(t.shape, seed=27)
        moved = (other(t + 1e-2 * step) - other(t - 1e-2 * step)) / 2e-2
        said = float((grad.double() * step.double()).sum())
        size = float(torch.linalg.norm(grad.double()) * torch.linalg.norm(step.double()))
        assert abs(moved - said) <= 2.0 ** -4 * size


# ---- sampling -----------------------------------------------------------------------------------------------------
def check_sample(x, u, temperature=None, top_k=None, top_p=None, min_p=None, token_dtype=torch.int64):
    rows = x.shape[0]
    t = lambda v, d=torch.float32: None if v is None else torch.tensor(v, dtype=d, device="cuda")  # noqa: E731
    tokens = torch.full((rows,), -7, dtype=token_dtype, device="cuda")
    prob = torch.full((rows,), -7.0, device="cuda")
    dst.dst_sample(x, t(u), tokens, temperature=t(temperature), top_k=t(top_k, torch.int32), top_p=t(top_p), min_p=t(min_p), prob=prob)
    X, tokens, prob = x.float().cpu().numpy(), tokens.cpu().numpy(), np64(prob)
    f = lambda v, r, d: d if v is None else float(np.float32(v[r]))  # noqa: E731
    unsure = 0
    for r in range(rows):
        token, pr, margin = o.sample(X[r], float(np.float32(u[r])), f(temperature, r, 1.0), 0 if top_k is None else top_k[r], f(top_p, r, 1.0), f(min_p, r, 0.0))
        if margin < 2.0 ** -18 and token != tokens[r]:
            unsure += 1
            continue
        assert token == tokens[r], (r, token, tokens[r], margin)
        assert abs(pr - prob[r]) <= 2.0 ** -18
    assert unsure <= 1 + rows // 50


def settings(rows, seed):
    rng = np.random.default_rng(seed)
    return dict(u=list(rng.integers(0, 1 << 24, rows) / 2.0 ** 24), temperature=list(rng.uniform(0.3, 2.0, rows)), top_k=[int(k) for k in rng.integers(0, 100, rows)],
                top_p=list(rng.uniform(0.2, 1.05, rows)), min_p=list(rng.choice([0.0, 0.01, 0.1], rows)))


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 2), (3, 7), (2, 31), (5, 33), (4, 1000), (1, 2049), (30, 2048), (1, 33708), (20, 33708), (40, 33708), (80, 5000), (160, 1024), (2, 65536), (300, 100), (3, 131072), (1, 327680)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", ["none", "k", "p", "m", "kp", "kpm"])
def test_sample(rows, vocab, dtype, which):
    x = randn((rows, vocab), "f32", 28) * 3
    x = x.to(TYPES[dtype])
    s = settings(rows, 29 + rows)
    check_sample(x, s["u"], s["temperature"], s["top_k"] if "k" in which else None, s["top_p"] if "p" in which else None, s["min_p"] if "m" in which else None,
                 torch.int32 if rows % 2 else torch.int64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_rows_with_a_stride_and_a_skew(dtype):
    for pad, skew in ((1, 1), (5, 3), (8, 0)):
        x = randn((9, 3001), dtype, 30, pad, skew)
        s = settings(9, 31)
        check_sample(x, s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])


@pytest.mark.parametrize("vocab", [5, 3000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_ties_are_taken_by_index(vocab, dtype):
    x = torch.zeros(12, vocab, device="cuda", dtype=TYPES[dtype])
    x[4:8] = torch.randint(0, 3, (4, vocab), generator=torch.Generator().manual_seed(32)).cuda().to(x.dtype)
    x[8:, 1::3] = -0.0                                                            # equal to +0
    ks, ps = [0, 1, 3, vocab - 1] * 3, [1.0, 0.5, 0.999, 0.01] * 3
    for u in (0.0, 0.3, 1 - 2.0 ** -24):
        check_sample(x, [u] * 12, None, ks, None)
        check_sample(x, [u] * 12, None, None, ps)
        check_sample(x, [u] * 12, None, ks, ps)


def test_sample_masked_and_special_rows():
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    base = randn((14, 4099), seed=33) * 2
    base[0] = -inf                                                                # nothing left
    base[1] = nan
    base[2] = -inf
    base[2, 4098] = -3.0                                                          # one entry left
    base[3] = low                                                                 # masked by the lowest value throughout
    base[4] = low
    base[4, 17] = 1.0
    base[5, ::2] = nan
    base[6, 100], base[6, 3000] = inf, inf
    base[7, :4000] = -inf
    base[8] = low
    base[8, 5], base[8, 6] = torch.finfo(torch.float32).max, -5.0
    base[9, :] = 1e-42                                                            # subnormal
    base[9, 7] = 1e-40
    base[10] *= 1e30
    base[11] *= 1e-30
    n = base.shape[0]
    rng = np.random.default_rng(34)
    u = list(rng.integers(0, 1 << 24, n) / 2.0 ** 24)
    for k, p, m in ((None, None, None), ([40] * n, None, None), (None, [0.9] * n, None), ([40] * n, [0.9] * n, [0.05] * n)):
        for t in (None, [0.0] * n, [1e-3] * n, [100.0] * n):
            check_sample(base, u, t, k, p, m)


def test_sample_limits_of_the_settings():
    x = randn((8, 2500), seed=35)
    u = [0.0, 0.5, 1.0, 2.0, -1.0, 1 - 2.0 ** -24, 0.25, 0.75]
    inf = float("inf")
    check_sample(x, u, [inf, 1e-30, 1e30, -1.0, 0.0, 1e-45, 1.0, 2.0], [5] * 8, [0.5] * 8)
    check_sample(x, u, None, [-3, 0, 1, 2500, 9999, 2499, 2, 7], [0.0, -1.0, 1.0, 2.0, 2.0 ** -30, 1 - 2.0 ** -24, 0.5, 0.5], [0.0, 1.0, 2.0, -1.0, 0.5, 0.0, 0.0, 0.0])


def test_a_row_draws_the_same_whatever_the_batch():
    x = randn((400, 6000), "bf16", 36)
    s = settings(400, 37)
    t = lambda v, d=torch.float32: torch.tensor(v, dtype=d, device="cuda")  # noqa: E731
    args = dict(temperature=t(s["temperature"]), top_k=t(s["top_k"], torch.int32), top_p=t(s["top_p"]), min_p=t(s["min_p"]))
    u, whole, parts = t(s["u"]), torch.empty(400, dtype=torch.int64, device="cuda"), torch.empty(400, dtype=torch.int64, device="cuda")
    dst.dst_sample(x, u, whole, **args)
    for size in (1, 30, 70, 299):                                                 # clusters of different sizes
        at = 0 if size == 1 else at + last
        last = size
        cut = slice(at, at + size)
        dst.dst_sample(x[cut], u[cut], parts[cut], **{k: v[cut] for k, v in args.items()})
    assert torch.equal(whole, parts)


def test_sample_frequencies_follow_the_probabilities():
    logits = torch.tensor([0.0, 1.0, 2.0, -1.0, 1.5], device="cuda").repeat(20000, 1)
    u = torch.rand(20000, generator=torch.Generator().manual_seed(38)).cuda()
    tokens = torch.empty(20000, dtype=torch.int32, device="cuda")
    dst.dst_sample(logits, u, tokens)
    want = torch.softmax(logits[0].double(), 0).cpu().numpy()
    got = np.bincount(tokens.cpu().numpy(), minlength=5) / 20000
    assert (np.abs(got - want) <= 5 * np.sqrt(want * (1 - want) / 20000)).all()


# ---- streams ------------------------------------------------------------------------------------------------------
def test_work_goes_to_the_stream_that_is_named():
    """Inputs written on a side stream just before the calls on that stream."""
    side = torch.cuda.Stream()
    proj = dst.TiedProjection(1000, 64, 32)
    w = randn((1000, 64), seed=39)
    x, logits, want = torch.empty(32, 64, device="cuda"), torch.empty(32, 1000, device="cuda"), torch.empty(32, 1000, device="cuda")
    src = randn((32, 64), seed=40)
    tokens, u = torch.empty(32, dtype=torch.int64, device="cuda"), torch.full((32,), 0.5, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        x.copy_(src)
    proj.update(w, stream=side)
    dst.dst_dropout(x, x, 0.25, 1, stream=side)
    proj.logits(x, logits, stream=side)
    dst.dst_sample(logits, u, tokens, stream=side)
    side.synchronize()
    y = torch.empty_like(src)
    dst.dst_dropout(src, y, 0.25, 1)
    proj.logits(y, want)
    t2 = torch.empty_like(tokens)
    dst.dst_sample(want, u, t2)
    assert torch.equal(logits, want) and torch.equal(tokens, t2)


# ---- offsets beyond 32 bits -----------------------------------------------------------------------------------------
def test_rows_more_than_two_to_the_31_elements_apart():
    """Row distances whose byte and element offsets pass 32 bits, in one buffer for inputs and outputs."""
    ld, d = (1 << 31) + 8, 520
    buf = torch.empty(2 * ld + 4 * d, dtype=torch.bfloat16, device="cuda")
    rows = lambda at, n=d: buf[at:at + 2 * ld + n].as_strided((3, n), (ld, 1))  # noqa: E731
    x, out = rows(0), rows(d)
    x.copy_(randn((3, d), "bf16", 41))
    out.zero_()
    dst.dst_dropout(x, out, 0.25, 3, residual=x)
    want = np64(x) * (1 + o.drop_factor(3, d, 0.25, 3))
    close(out, want, 8 * U * np.abs(want), "bf16")
    q, qt = dst.Fp8Matrix(3, d), dst.Fp8Matrix(d, 3)
    dst.dst_quantize_fp8(x, q, qt)
    assert np.array_equal(codes(q), o.quantize(np64(x), 1)[0]) and np.array_equal(codes(qt), o.quantize(np64(x).T, 1)[0])
    w = dst.Fp8Matrix(d, d, dst.DST_FP8_SQUARE)
    dst.dst_quantize_fp8(randn((d, d), seed=42), w)
    ws = torch.empty(max(dst.dst_matmul_fp8_workspace_bytes(3, d, d), 256), dtype=torch.uint8, device="cuda")
    dst.dst_matmul_fp8(q, w, out, ws)
    A, B = np64(q.dequantize()), np64(w.dequantize())
    close(out, A @ B.T, (128 + 4 * 5 + 16) * 2 * U * (np.abs(A) @ np.abs(B).T), "bf16")
    s = settings(3, 43)
    check_sample(x, s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])


@pytest.mark.parametrize("n,d", [(70000, 32768)])
def test_matrices_of_more_than_two_to_the_31_elements(n, d):
    """2.3 billion elements through dropout, both quantisations and a thin product; rows from all over are checked."""
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    pattern = randn((1000, d), "bf16", 44)
    for i in range(0, n, 1000):
        x[i:i + 1000] = pattern
    out = torch.empty_like(x)
    dst.dst_dropout(x, out, 0.5, 11)
    at = [0, 1, 65535, 65536, n - 1]
    for r in at:
        k = o.drop_factor(1, d, 0.5, 11, row_offset=r)
        assert np.array_equal(np64(out[r:r + 1]), np64(x[r:r + 1]) * k)
    del out
    q = dst.Fp8Matrix(n, d)
    dst.dst_quantize_fp8(x, q)
    want = o.dequantize(*o.quantize(np64(x[at]), 1), 1)
    got = torch.stack([q.q[r, :d].float() * q.scales()[r].repeat_interleave(128) for r in at])
    assert np.array_equal(np64(got), want)
    b = randn((20, d), seed=45)
    qb = dst.Fp8Matrix(20, d)
    dst.dst_quantize_fp8(b, qb)
    y = torch.empty(n, 20, device="cuda")
    dst.dst_matmul_fp8(q, qb, y, torch.empty(max(dst.dst_matmul_fp8_workspace_bytes(n, 20, d), 256), dtype=torch.uint8, device="cuda"))
    B = np64(qb.dequantize())
    close(y[at], want @ B.T, (128 + 4 * (d // 128) + 16) * 2 * U * (np.abs(want) @ np.abs(B).T), "f32")
