"""GPU parity of a step's operators against their 64-bit definitions (oracle/step_oracle.py).

Tolerances, with u = 2^-24 (fp32 rounding) and h = 2^-8 (half a bf16 step, relative):
  log probabilities   z = scale (x - max): a difference, a factor and the constant log2 e each off by u, so an exponential is off
             by 3u |z| and by the 2^-22 = 4u that its instruction allows.  A thread adds at most 64 of them to what it had, two chains (33u a tile),
             joins (lanes 5, warps 5, CTAs 5 additions, each join an exponential and its distance) add 3 (5 + 4 + 4)u.
             rho = (33 tiles + 60 + 3 E|z|) u bounds the relative error of r and of t, E|z| <= 2 log vocab.
               log p: rho r / (1 + r) + 4u log1p(r) + 4u |z| (+ 4u |scale max| for lse), and vocab 2^-126: exponentials below
               2^-126 are zero, as fp32 has no normal number there
               entropy: both terms are at most the entropy:  2 rho (H + r / (1 + r)) + 8u H
               gradient: p's own error (rho + 10u + 4u |z|) times what it multiplies, and that factor's error
             (lse is rounded to fp32, which is an infinity beyond its range)
  norm       the squares' sum: 32 + 5 + 16 additions, half of it in inv_rms, rsqrt 2^-22: 32u; y two more roundings: 36u |y|
             mean(g u): its terms 34u, their sum 53u, and the division:  90u of the absolute terms' mean
             dweight: a warp adds rows / (CTAs teams) rows, then 8 and all CTAs' shares: (that + 8 + 296 + 36) u sum |dy u|
  clip       the norm and the factor are rounded once from 64 bits (4u), the product once (6u in all, + h)
"""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst
from oracle import step_oracle as o

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def np64(t):
    return t.detach().cpu().double().numpy()


def near(got, want, tol, dtype="f32", what=""):
    got = np64(got) if isinstance(got, torch.Tensor) else np.asarray(got, np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    tol = np.broadcast_to(tol, want.shape)[fine] + (H * np.abs(want[fine]) if dtype == "bf16" else 0)
    off = np.abs(got[fine] - want[fine])
    bad = ~(off <= tol + 1e-37)
    assert not bad.any(), "%s: %d out of tolerance, worst %r of %r" % (what, bad.sum(), off[bad].max(), tol[bad].max())


def strided(rows, cols, dtype, pad=0, skew=0, fill=None):
    """A [rows, cols] view whose rows are cols + pad elements apart and start `skew` elements into the buffer; and the buffer."""
    buf = torch.full((rows * (cols + pad) + skew,), float("nan"), dtype=TYPES[dtype], device="cuda")
    t = buf[skew:].view(rows, cols + pad)[:, :cols]
    if fill is not None:
        t.copy_(fill)
    return t, buf


def untouched(buf, view):
    """Whether everything of the buffer outside the view is still NaN."""
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside.as_strided(view.size(), view.stride(), view.storage_offset()).fill_(True)
    return bool(torch.isnan(buf[~inside]).all())


# ---- log probabilities -------------------------------------------------------------------------------------------
def make_logits(rows, vocab, dtype, seed, pad=0, skew=0, masked=False, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * spread + 5
    if masked:
        x[torch.rand(rows, vocab, generator=g) < 0.5] = -float("inf")
        x[:, vocab // 2] = 1.0
    t, _ = strided(rows, vocab, dtype, pad, skew, x)
    return t, torch.randint(0, vocab, (rows,), generator=g).cuda(), g


class Want:
    def __init__(self, x, scale, dtype):
        self.x, self.scale, self.dtype = np64(x), scale, dtype
        self.log_p, self.lse, self.entropy, self.r = o.log_probabilities(self.x, scale)
        vocab = x.shape[1]
        tiles = 1 if vocab <= 131072 else 8
        self.rho = (33 * tiles + 60 + 6 * np.log(max(vocab, 2))) * U
        with np.errstate(invalid="ignore", divide="ignore"):
            self.share = np.where(self.r >= 0, self.r / (1 + self.r), 0)
            self.log_total = np.where(self.r >= 0, np.log1p(np.maximum(self.r, 0)), 0)
            self.z = np.nan_to_num(scale * (self.x - self.x.max(-1, keepdims=True)), nan=0.0, neginf=0.0, posinf=0.0)

    def of(self, t):
        return np.nan_to_num(t, nan=0.0)

    def tol_log_p(self):
        return (self.of(self.rho * self.share + 4 * U * self.log_total))[:, None] + 4 * U * np.abs(self.z) + self.x.shape[1] * 2.0 ** -126

    def tol_entropy(self):
        # (a term of the entropy is at most 90 times its exponential where that is below 2^-126 and the gap is what fp32 can hold of it)
        return self.of(2 * self.rho * (self.entropy + self.share) + 8 * U * self.entropy) + self.x.shape[1] * 200 * 2.0 ** -126

    def tol_grad(self, targets, a, b):
        p = np.exp(np.nan_to_num(self.log_p, nan=0.0))
        lp, h = np.where(p > 0, np.nan_to_num(self.log_p, neginf=0.0, nan=0.0), 0), self.of(self.entropy)[:, None]
        a, b = np.abs(np.where(targets >= 0, a, 0))[:, None], np.abs(b)[:, None]
        rel = self.rho + 10 * U + 4 * U * np.abs(self.z)
        t = p * (rel * (a + b * (np.abs(lp) + h)) + b * (self.tol_log_p() + self.tol_entropy()[:, None]))
        t = t + 2.0 ** -126 * (a + b * (200 + h))              # exponentials below 2^-126 are zero; their logarithm is above -200 where that matters
        rows = np.flatnonzero(targets >= 0)
        at = targets[rows]
        # the target's own: (1 - p) to 4u of itself and to p's error through log p
        t[rows, at] += a[rows, 0] * (4 * U * (1 - p[rows, at]) + p[rows, at] * self.tol_log_p()[rows, at])
        return t * self.scale


def check_logprob(x, targets, scale=1.0, top=0, index=torch.int64):
    rows = x.shape[0]
    dtype = "f32" if x.dtype == torch.float32 else "bf16"
    w = Want(x, scale, dtype)
    new = lambda *s: torch.full(s, 7.5, device="cuda")  # noqa: E731
    logprob, lse, entropy, stats = new(rows), new(rows), new(rows), new(rows, 2)
    more = {}
    if top:
        more = {"top_tokens": torch.full((rows, top), -7, dtype=index, device="cuda"), "top_logprob": new(rows, top)}
    dst.dst_logprob(x, targets.to(index), logprob, scale=scale, lse=lse, entropy=entropy, stats=stats, **more)
    near_sums(w, targets, logprob, lse, entropy)
    if top:
        want = o.top_tokens(w.x, top)
        assert np.array_equal(more["top_tokens"].cpu().numpy(), want)
        listed = np.where(want >= 0, np.take_along_axis(w.log_p, np.maximum(want, 0), 1), -np.inf)
        near(more["top_logprob"], listed, np.take_along_axis(w.tol_log_p(), np.maximum(want, 0), 1), what="top_logprob")
    return logprob, lse, entropy, stats, w


def near_sums(w, targets, logprob, lse, entropy):
    t = targets.cpu().numpy()
    at = np.clip(t, 0, w.x.shape[1] - 1)
    given = (t >= 0) & (t < w.x.shape[1])
    ar = np.arange(len(t))
    near(logprob, np.where(given, w.log_p[ar, at], 0.0), np.where(given, w.tol_log_p()[ar, at], 0.0), what="logprob")
    with np.errstate(over="ignore"):
        want_lse = np.where(np.abs(w.lse) < np.finfo(np.float32).max, w.lse, w.lse.astype(np.float32))   # fp32 holds no more: an infinity
    near(lse, want_lse, w.of(w.rho * w.share + 4 * U * (w.log_total + np.abs(np.nan_to_num(w.lse, neginf=0.0, nan=0.0)) + w.log_total)), what="lse")
    near(entropy, w.entropy, w.tol_entropy(), what="entropy")


def check_gradient(x, targets, a, b, scale=1.0, out="f32", pad=0, skew=0, in_place=False, index=torch.int32):
    """The gradient in one pass and from what the forward call gave."""
    rows, vocab = x.shape
    _, _, entropy, stats, w = check_logprob(x, targets, scale)
    t = targets.cpu().numpy()
    t = np.where(t >= vocab, -1, t)
    want = o.logits_gradient(w.x, t, scale, np64(a), np64(b))
    da, db = a.cuda(), b.cuda()
    for one_pass in (True, False):
        kept = x.clone() if in_place else None
        d, buf = (x, None) if in_place else strided(rows, vocab, out, pad, skew)
        if one_pass:
            got = [torch.empty(rows, device="cuda") for _ in range(3)]
            dst.dst_logprob_loss(x, targets.to(index), da, got[0], d, scale=scale, dentropy=db, lse=got[1], entropy=got[2])
            near_sums(w, targets, *got)
        else:
            dst.dst_logprob_backward(x, targets.to(index), stats, da, d, scale=scale, entropy=entropy, dentropy=db)
        near(d, want, w.tol_grad(t, np64(a), np64(b)), out, "dlogits %s" % one_pass)
        if in_place:
            x.copy_(kept)
        else:
            assert untouched(buf, d)


SIZES = [(1, 1), (3, 2), (2, 7), (5, 33), (4, 1000), (1, 2049), (20, 5000), (1, 33708), (7, 33708), (400, 33708), (3, 65536), (300, 1024), (1, 262147), (2, 300000)]


@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
def test_logprob(rows, vocab, dtype, masked):
    x, targets, _ = make_logits(rows, vocab, dtype, rows + vocab, masked=masked)
    check_logprob(x, targets, 1.0, min(20, 32))
    check_logprob(x, targets, 0.6, 1, torch.int32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,skew", [(3, 1), (8, 0), (1, 5)])
def test_logprob_rows_with_a_stride_and_a_skew(dtype, pad, skew):
    for rows, vocab in ((5, 1001), (2, 33708), (3, 6)):
        x, targets, _ = make_logits(rows, vocab, dtype, 3, pad, skew)
        check_logprob(x, targets, 1.3, 5)


@pytest.mark.parametrize("rows,vocab", [(1, 1), (2, 7), (5, 33), (4, 1000), (20, 5000), (3, 33708), (310, 33708), (2, 65536), (2, 300000)])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("pad,skew", [(0, 0), (3, 1)])
def test_logits_gradient(rows, vocab, dtype, out, pad, skew):
    x, targets, g = make_logits(rows, vocab, dtype, vocab - rows, pad, skew, masked=vocab > 100)
    targets[rows // 2] = -1 if rows > 1 else targets[0]
    a, b = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    check_gradient(x, targets, a, b, 1.4, out, pad, skew)
    check_gradient(x, targets, a, b * 0, 1.0, out, 4, 0)
    if dtype == out:
        check_gradient(x, targets, a, b, 0.8, out, in_place=True)


def test_confident_rows_are_accurate_relative_to_what_the_others_hold():
    x = torch.full((6, 5000), -3.0)
    for i, gap in enumerate((5.0, 10.0, 17.0, 25.0, 60.0, 200.0)):
        x[i, 17 * i] = -3.0 + gap
    x = x.cuda()
    targets = torch.arange(0, 6 * 17, 17).cuda()
    logprob, _, _, _, w = check_logprob(x, targets)
    got, want = np64(logprob), w.log_p[np.arange(6), targets.cpu().numpy()]
    assert np.all(np.abs(got - want)[:5] <= 1e-5 * np.abs(want)[:5]) and got[5] == 0 or abs(got[5]) < 1e-80
    check_gradient(x, targets, torch.ones(6), torch.zeros(6))
    check_gradient(x.bfloat16(), targets, torch.ones(6), torch.ones(6))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 3000, 40000, 300000])
def test_equal_logits_are_listed_by_index(dtype, vocab):
    x = torch.zeros(3, vocab)
    x[1, vocab // 2:] = 1.0
    x[2, :5] = torch.tensor([-0.0, 0.0, 2.0, -0.0, 2.0])
    check_logprob(x.to(TYPES[dtype]).cuda(), torch.zeros(3, dtype=torch.int64).cuda(), 1.0, 32 if vocab > 32 else 9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [12, 9000, 40000])
def test_masked_and_special_rows(dtype, vocab):
    inf, nan = float("inf"), float("nan")
    lowest = torch.finfo(TYPES[dtype]).min
    x = torch.randn(10, vocab, generator=torch.Generator().manual_seed(1))
    x[0] = -inf                                   # nothing left
    x[1] = -inf
    x[1, vocab - 1] = -4.0                        # one token left
    x[2, 3] = nan
    x[3, vocab // 2] = inf
    x[4] = nan
    x[5] = lowest                                 # masks of the lowest value: equal logits
    x[6, ::2] = lowest
    x[7] = -inf
    x[7, 5:9] = 2.5                               # fewer than are asked for
    x[8] = -inf
    x[8, 0] = nan
    x[9] *= 1e4 if dtype == "f32" else 1e3        # far apart
    x = x.to(TYPES[dtype]).cuda()
    targets = torch.tensor([0, vocab - 1, 0, 0, 0, 1, 1, 6, 1, 2]).cuda()
    check_logprob(x, targets, 1.0, 8)
    check_gradient(x, targets, torch.ones(10), torch.zeros(10), out=dtype)
    check_gradient(x, targets, torch.ones(10), torch.ones(10), 2.0, out=dtype)
    zeros = torch.zeros(10)
    d = torch.full_like(x, 3.0)
    dst.dst_logprob_loss(x, targets, zeros.cuda(), torch.empty(10, device="cuda"), d, dentropy=zeros.cuda())
    assert bool((d == 0).all())                   # no derivative, no gradient, whatever the logits
    targets[:] = -100
    dst.dst_logprob_loss(x, targets, torch.ones(10).cuda(), None, d.fill_(3.0))
    assert bool((d == 0).all())


def test_rows_without_a_target_and_out_of_range_ones():
    x, targets, _ = make_logits(6, 500, "f32", 1)
    targets[:] = torch.tensor([0, -1, 500, 499, -(1 << 40), 1 << 40])
    out = torch.full((6,), 9.0, device="cuda")
    result = torch.full((6,), 5, dtype=torch.int32, device="cuda")
    dst.dst_logprob(x, targets, out, result=result)
    assert out[1] == 0 and out[2] == 0 and out[4] == 0 and out[5] == 0 and out[0] < 0
    assert result[0] == 4 and result[2] == 2      # status, n_out_of_range
    d = torch.empty_like(x)
    dst.dst_logprob_loss(x, targets, torch.ones(6, device="cuda"), out, d, result=result)
    assert result[2] == 2 and bool((d[[1, 2, 4, 5]] == 0).all())
    stats = torch.empty(6, 2, device="cuda")
    dst.dst_logprob(x, None, stats=stats)
    back = torch.empty_like(x)
    dst.dst_logprob_backward(x, targets, stats, torch.ones(6, device="cuda"), back)
    assert bool((back[[1, 2, 4, 5]] == 0).all()) and torch.allclose(back, d, atol=1e-6)
    dst.dst_logprob(x, targets.clamp(0, 499), out, result=result)
    assert result[0] == 0 and result[2] == 0


def test_logits_gradient_against_differences():
    g = torch.Generator().manual_seed(4)
    x = torch.randn(3, 50, generator=g)
    targets, a, b = torch.tensor([4, 49, -1]), torch.randn(3, generator=g), torch.randn(3, generator=g)
    d = torch.empty(3, 50, device="cuda")
    dst.dst_logprob_loss(x.cuda(), targets.cuda(), a.cuda(), None, d, scale=1.3, dentropy=b.cuda())

    def loss(x):
        log_p, _, entropy, _ = o.log_probabilities(x, 1.3)
        return sum(float(a[i]) * log_p[i, t] for i, t in enumerate(targets.tolist()) if t >= 0) + float((b.double().numpy() * entropy).sum())
    x64, got, e = x.double().numpy(), np64(d), 1e-5
    for i, j in ((0, 4), (0, 0), (1, 49), (1, 20), (2, 3)):
        up, down = x64.copy(), x64.copy()
        up[i, j] += e
        down[i, j] -= e
        assert abs((loss(up) - loss(down)) / (2 * e) - got[i, j]) < 1e-6   # e^2 of the third derivative, and fp32


def test_a_row_gives_the_same_whatever_the_batch_and_twice():
    x, targets, g = make_logits(600, 5000, "bf16", 5)
    out = [torch.empty(600, device="cuda") for _ in range(2)]
    d = [torch.empty(600, 5000, device="cuda") for _ in range(2)]
    a = torch.randn(600, generator=g).cuda()
    for i in range(2):
        dst.dst_logprob_loss(x, targets, a, out[i], d[i])
    assert torch.equal(*out) and torch.equal(*d)


# ---- norm --------------------------------------------------------------------------------------------------------
def check_norm(rows, d, xt, st, ot, residual, pad=0, skew=0, weight=True, eps=1e-6, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, _ = strided(rows, d, xt, pad, skew, torch.randn(rows, d, generator=g))
    r = strided(rows, d, st, pad, skew, torch.randn(rows, d, generator=g) * 3)[0] if residual else None
    w = torch.randn(d, generator=g).cuda() if weight else None
    s, s_buf = strided(rows, d, st, pad, skew)
    y, y_buf = strided(rows, d, ot, pad, skew)
    q = dst.Fp8Matrix(rows, d)
    inv = torch.empty(rows, device="cuda")
    dst.dst_rmsnorm(x, w, y, q=q, residual=r, sum_out=s, eps=eps, inv_rms=inv)
    h = (x.float() + (r.float() if residual else 0)).to(TYPES[st])
    assert torch.equal(s, h) and untouched(s_buf, s) and untouched(y_buf, y)
    w64 = np64(w) if weight else 1.0
    want, inv64 = o.rmsnorm(np64(h), w64, eps)
    near(inv, inv64, 32 * U * inv64)
    near(y, want, 36 * U * np.abs(want), ot)
    # the 8-bit form is that of the fp32 result of the same call
    y32, q32 = torch.empty(rows, d, device="cuda"), dst.Fp8Matrix(rows, d)
    dst.dst_rmsnorm(x, w, y32, q=q, residual=r, sum_out=s, eps=eps)
    dst.dst_quantize_fp8(y32, q32)
    assert torch.equal(q.q[:, :d].view(torch.uint8), q32.q[:, :d].view(torch.uint8)) and torch.equal(q.scales(), q32.scales())
    near(y32, want, 36 * U * np.abs(want))
    return h, w, inv, w64, g


def check_norm_gradient(rows, d, dt, ht, xt, pad=0, skew=0, weight=True, dsum=True, seed=0):
    h, w, inv, w64, g = check_norm(rows, d, ht, ht, "f32", False, pad, skew, weight, 1e-3, seed)
    h = strided(rows, d, ht, pad, skew, h)[0]
    dy, _ = strided(rows, d, dt, pad, skew, torch.randn(rows, d, generator=g))
    ds = strided(rows, d, xt, pad, skew, torch.randn(rows, d, generator=g))[0] if dsum else None
    dx, buf = strided(rows, d, xt, pad, skew)
    dw = torch.full((d,), float("nan"), device="cuda")
    ws = torch.full((dst.dst_rmsnorm_backward_workspace_bytes(rows, d),), 255, dtype=torch.uint8, device="cuda")
    dst.dst_rmsnorm_backward(dy, h, w, inv, dx, dsum=ds, dweight=dw, workspace=ws)
    i64 = np64(inv)
    want, want_w = o.rmsnorm_gradient(np64(dy), np64(h), w64, i64, np64(ds) if dsum else np.zeros((rows, d)))
    u, gw = np.abs(np64(h)) * i64[:, None], np.abs(np64(dy) * w64)
    tol = i64[:, None] * (4 * U * gw + u * 95 * U * (gw * u).mean(-1, keepdims=True)) + 4 * U * np.abs(want) + 2 * U * (np.abs(np64(ds)) if dsum else 0)
    near(dx, want, tol, xt)
    near(dw, want_w, (rows / 296 + 8 + 296 + 36) * U * (np.abs(np64(dy)) * u).sum(0))
    assert untouched(buf, dx)
    again = torch.empty_like(dw)
    dst.dst_rmsnorm_backward(dy, h, w, inv, dx, dsum=ds, dweight=again, workspace=ws.fill_(1))
    assert torch.equal(dw, again)
    alone, _ = strided(rows, d, xt, pad, skew)
    dst.dst_rmsnorm_backward(dy, h, w, inv, alone, dsum=ds)
    assert torch.equal(alone, dx)
    for t in (ds, dy if dt == xt else None, h if ht == xt else None):   # in place
        if t is not None:
            kept = t.clone()
            dst.dst_rmsnorm_backward(dy, h, w, inv, t, dsum=ds)
            assert torch.equal(t, dx)
            t.copy_(kept)


NORM_SIZES = [(1, 1), (1, 1024), (3, 5), (7, 64), (9, 127), (8, 128), (5, 130), (33, 512), (2, 1021), (3, 1025), (4, 2048), (2, 5000), (1, 16384), (3, 16383)]


@pytest.mark.parametrize("rows,d", NORM_SIZES)
@pytest.mark.parametrize("xt,st,ot", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "bf16"), ("f32", "bf16", "f32")])
@pytest.mark.parametrize("pad,skew", [(0, 0), (3, 1)])
def test_rmsnorm(rows, d, xt, st, ot, pad, skew):
    check_norm(rows, d, xt, st, ot, True, pad, skew, seed=d)
    check_norm(rows, d, xt, st, ot, False, pad, skew, weight=False, seed=d)


@pytest.mark.parametrize("rows,d", NORM_SIZES + [(700, 256), (5000, 33)])
@pytest.mark.parametrize("dt,ht,xt", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f32", "bf16", "bf16")])
@pytest.mark.parametrize("pad,skew", [(0, 0), (3, 1)])
def test_rmsnorm_gradient(rows, d, dt, ht, xt, pad, skew):
    check_norm_gradient(rows, d, dt, ht, xt, pad, skew, seed=rows)
    check_norm_gradient(rows, d, dt, ht, xt, pad, skew, weight=False, dsum=False, seed=rows)


def test_rmsnorm_gradient_against_differences():
    g = torch.Generator().manual_seed(4)
    h, w, dy = torch.randn(2, 20, generator=g), torch.randn(20, generator=g), torch.randn(2, 20, generator=g)
    inv, dx, dw = torch.empty(2, device="cuda"), torch.empty(2, 20, device="cuda"), torch.empty(20, device="cuda")
    ws = torch.empty(dst.dst_rmsnorm_backward_workspace_bytes(2, 20), dtype=torch.uint8, device="cuda")
    dst.dst_rmsnorm(h.cuda(), w.cuda(), torch.empty_like(dx), eps=0.01, inv_rms=inv)
    dst.dst_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), inv, dx, dweight=dw, workspace=ws)
    loss = lambda h, w: float((dy.double().numpy() * o.rmsnorm(h, w, 0.01)[0]).sum())  # noqa: E731
    h64, w64, e = h.double().numpy(), w.double().numpy(), 1e-5
    for i, j in ((0, 0), (1, 19), (1, 7)):
        up, down, wu, wd = h64.copy(), h64.copy(), w64.copy(), w64.copy()
        up[i, j] += e; down[i, j] -= e; wu[j] += e; wd[j] -= e
        assert abs((loss(up, w64) - loss(down, w64)) / (2 * e) - float(dx[i, j])) < 2e-6
        assert abs((loss(h64, wu) - loss(h64, wd)) / (2 * e) - float(dw[j])) < 2e-6


def test_rmsnorm_in_place_and_rows_of_special_values():
    g = torch.Generator().manual_seed(6)
    x, r, w = (torch.randn(9, 300, generator=g).cuda() for _ in range(2)), None, None
    x, r = x
    y = torch.empty_like(x)
    s = torch.empty_like(x)
    dst.dst_rmsnorm(x, w, y, residual=r, sum_out=s)
    x1, r1 = x.clone(), r.clone()
    dst.dst_rmsnorm(x1, w, x1, residual=r1, sum_out=r1)
    assert torch.equal(x1, y) and torch.equal(r1, s)
    x[0] = 0.0
    x[1, 5], x[2, 7] = float("nan"), float("inf")
    q = dst.Fp8Matrix(9, 300)
    dst.dst_rmsnorm(x, w, y, q=q)
    assert bool((y[0] == 0).all()) and bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[2, 7])) and bool((y[2, :7] == 0).all())
    assert torch.isnan(q.scales()[1]).all() and torch.isnan(q.scales()[2, 0]) and not torch.isnan(q.scales()[3:]).any()


# ---- norm and clipping of gradients ------------------------------------------------------------------------------
def check_clip(tensors, max_norm, in_place=False, out_types=None):
    lists = dst.TensorList(tensors)
    outs = tensors if in_place else [torch.full_like(t, 7.0, dtype=ot) for t, ot in zip(tensors, out_types or [t.dtype for t in tensors])]
    given = [np64(t) for t in tensors]
    norm, factor, want = o.clip(given, max_norm)
    clip = torch.full((2,), 7.0, device="cuda")
    ws = torch.full((dst.dst_grad_norm_workspace_bytes(lists),), 255, dtype=torch.uint8, device="cuda")
    dst.dst_grad_norm(lists, clip, max_norm, ws)
    dst.dst_clip(lists, clip, None if in_place else dst.TensorList(outs))
    got = clip.cpu().double().numpy()
    if np.isfinite(norm):
        assert abs(got[0] - norm) <= 2 * U * norm + 1e-45 and abs(got[1] - factor) <= 4 * U * factor
    else:
        assert not np.isfinite(got[0]) and got[1] == 0
    for t, w in zip(outs, want):
        near(t, w, 6 * U * np.abs(w), "f32" if t.dtype == torch.float32 else "bf16")
    return got


def make_tensors(sizes, dtypes, seed=0, scale=1.0, skew=0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n + skew, generator=g) * scale).to(TYPES[dtypes[i % len(dtypes)]]).cuda()[skew:] for i, n in enumerate(sizes)]


@pytest.mark.parametrize("sizes", [[], [0], [1], [7, 0, 3], [16384], [16383, 16385, 1], [100000, 5, 8, 33333], [8] * 97, [3] * 200, [20000] * 100])
@pytest.mark.parametrize("dtypes", [["f32"], ["bf16"], ["f32", "bf16"]])
@pytest.mark.parametrize("skew", [0, 1])
def test_grad_norm_and_clip(sizes, dtypes, skew):
    for max_norm in (0.5, 1e9, 0.0):
        check_clip(make_tensors(sizes, dtypes, 1, skew=skew), max_norm)
        check_clip(make_tensors(sizes, dtypes, 1, skew=skew), max_norm, in_place=True)
    tensors = make_tensors(sizes, dtypes, 2, skew=skew)
    check_clip(tensors, 1.0, out_types=[torch.bfloat16 if t.dtype == torch.float32 else torch.float32 for t in tensors])


def test_norms_beyond_the_range_of_32_bit_squares():
    assert check_clip(make_tensors([5000, 300], ["f32"], scale=1e25), 1.0)[0] > 1e26
    small = check_clip(make_tensors([5000, 300], ["f32", "bf16"], scale=1e-30), 1.0)
    assert 0 < small[0] < 1e-27 and small[1] == 1


def test_norms_that_are_not_finite_give_zeros():
    for bad in (float("nan"), float("inf"), -float("inf")):
        for dtypes in (["f32"], ["bf16"]):
            tensors = make_tensors([40000, 10], dtypes)
            tensors[0][33333] = bad
            check_clip(tensors, 1.0)
            check_clip(tensors, 1.0, in_place=True)


def test_norm_is_the_same_twice_and_a_factor_of_one_in_place_keeps_every_bit():
    tensors = make_tensors([1 << 22, 12345], ["f32", "bf16"])
    lists, ws = dst.TensorList(tensors), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    clips = [torch.empty(2, device="cuda") for _ in range(2)]
    for c in clips:
        dst.dst_grad_norm(lists, c, 1e9, ws)
    assert torch.equal(*clips)
    kept = [t.clone() for t in tensors]
    dst.dst_clip(lists, clips[0])
    assert all(torch.equal(a, b) for a, b in zip(tensors, kept))


# ---- many rows at once, which share a ring in shared memory ------------------------------------------------------
@pytest.mark.parametrize("vocab,dtype", [(33708, "bf16"), (33708, "f32"), (9000, "bf16"), (70001, "bf16"), (30011, "f32")])
def test_many_rows_give_the_same_bits_every_time(vocab, dtype):
    rows = 700
    x, targets, g = make_logits(rows, vocab, dtype, 8, pad=3)
    a = torch.randn(rows, generator=g).cuda()
    out = [torch.empty(rows, device="cuda") for _ in range(2)]
    d = [torch.empty(rows, vocab, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    dst.dst_logprob_loss(x, targets, a, out[0], d[0])
    for _ in range(20):
        d[1].zero_()
        dst.dst_logprob_loss(x, targets, a, out[1], d[1])
        assert torch.equal(*out) and torch.equal(*d)
    some = torch.randint(0, rows, (12,), generator=g)
    w = Want(x[some.cuda()], 1.0, dtype)
    t, b = targets[some.cuda()].cpu().numpy(), np.zeros(12)
    near(d[0][some.cuda()], o.logits_gradient(w.x, t, 1.0, np64(a[some.cuda()]), b), w.tol_grad(t, np64(a[some.cuda()]), b), dtype)
    near_sums(w, targets[some.cuda()], out[0][some.cuda()], torch.from_numpy(w.lse).float(), torch.from_numpy(w.entropy).float())


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("vocab", [9000, 40000])
@pytest.mark.parametrize("pad", [0, 5])
def test_special_and_confident_rows_among_many(dtype, out, vocab, pad):
    inf, nan, n = float("inf"), float("nan"), 12
    x = torch.randn(n, vocab, generator=torch.Generator().manual_seed(1))
    x[0] = -inf
    x[1] = -inf
    x[1, vocab - 1] = -4.0
    x[2, 3] = nan
    x[3, vocab // 2] = inf
    x[4] = nan
    x[5] = torch.finfo(TYPES[dtype]).min
    x[6, ::2] = torch.finfo(TYPES[dtype]).min
    x[7, 77] = 30.0                               # nearly all on one token
    x[8, vocab - 1] = 60.0
    x[9, 0] = 20.0
    x[10] *= 100
    x, targets = x.to(TYPES[dtype]), torch.tensor([0, vocab - 1, 0, 0, 0, 1, 1, 77, vocab - 1, 5, 2, -1])
    w = Want(x.cuda(), 1.5, dtype)
    many, _ = strided(n * 40, vocab, dtype, pad, 0, x.repeat(40, 1))
    for b in (0.0, 0.5):
        a, e = torch.linspace(-1, 1, n), torch.full((n,), b)
        a[10] = 0.0
        logprob, lse, entropy = (torch.empty(n * 40, device="cuda") for _ in range(3))
        d, buf = strided(n * 40, vocab, out, pad, 0)
        dst.dst_logprob_loss(many, targets.repeat(40).cuda(), a.repeat(40).cuda(), logprob, d, scale=1.5, dentropy=e.repeat(40).cuda(), lse=lse, entropy=entropy)
        for part in (0, 17, 39):
            at = slice(part * n, part * n + n)
            near_sums(w, targets, logprob[at], lse[at], entropy[at])
            near(d[at], o.logits_gradient(w.x, targets.numpy(), 1.5, np64(a), np64(e)), w.tol_grad(targets.numpy(), np64(a), np64(e)), out)
        assert pad == 0 or untouched(buf, d)


def test_lists_keep_their_memory_and_refuse_shared_outputs():
    x = torch.arange(20.0, device="cuda")
    clip = torch.tensor([1.0, 0.5], device="cuda")
    for shared in ([x, x], [x[:11], x[10:]], [x, x[3:4]]):
        with pytest.raises(ValueError):
            dst.dst_clip(dst.TensorList(shared), clip)
    dst.dst_clip(dst.TensorList([x[:10], x[10:], x[:0]]), clip)   # side by side
    assert torch.equal(x.cpu(), torch.arange(20.0) * 0.5)
    t = torch.ones(1000, device="cuda")
    lists, seen = dst.TensorList([t]), t.detach()
    t.data = torch.zeros(5, device="cuda")                        # other memory: the list has what it was made of
    dst.dst_clip(lists, clip)
    assert bool((seen == 0.5).all()) and bool((t == 0).all()) and lists.tensors[0].data_ptr() == seen.data_ptr()


# ---- row counts and lengths on both sides of the rules by which a variant is chosen ------------------------------
@pytest.mark.parametrize("rows", [74, 75, 148, 149, 297])
@pytest.mark.parametrize("dtype,out,vocab", [("f32", "f32", 5003), ("bf16", "bf16", 9000), ("bf16", "f32", 33708), ("f32", "bf16", 27000)])
def test_logits_gradient_by_rows(rows, dtype, out, vocab):
    x, targets, g = make_logits(rows, vocab, dtype, rows, 5, 1, masked=True)
    targets[3], targets[rows - 1] = -1, vocab + 7
    a, b = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    a[5] = b[5] = 0.0
    check_gradient(x, targets, a, b, 1.1, out, 5, 1)
    if dtype == out:
        check_gradient(x, targets, a, b * 0, 1.0, out, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("per_lane", [0, 1])
def test_logits_gradient_where_the_ring_ends(dtype, per_lane):
    """Rows as long as four vectors a thread, and as the ring holds with two CTAs an SM and with one, and one vector more."""
    n = 4 if dtype == "f32" else 8
    for vectors in (1024, (9 - 2) * 768, (14 - 2) * 960):
        vocab = (vectors + per_lane) * n - n + 1                  # (whose vectors are counted for the worst place within 16 bytes)
        x, targets, g = make_logits(80, vocab, dtype, vocab, 3, 1)
        check_gradient(x, targets, torch.randn(80, generator=g), torch.randn(80, generator=g), 1.0, dtype, 3, 1)


@pytest.mark.parametrize("rows,d", [(3, 4097), (5, 6002), (400, 8192), (2, 8191), (300, 8193), (310, 4096)])
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("pad,skew", [(0, 0), (4, 4), (3, 1)])
def test_rmsnorm_of_wide_rows(rows, d, t, pad, skew):
    check_norm(rows, d, t, t, t, True, pad, skew, seed=d)
    check_norm_gradient(rows, d, t, t, t, pad, skew, seed=rows)


@pytest.mark.parametrize("d", [40, 128, 300, 1000])
def test_a_norm_in_8_bits_goes_into_the_product_whatever_its_buffers_held(d):
    g = torch.Generator().manual_seed(d)
    x, w = torch.randn(21, d, generator=g).cuda(), dst.Fp8Matrix(50, d, dst.DST_FP8_SQUARE)
    dst.dst_quantize_fp8(torch.randn(50, d, generator=g).cuda(), w)
    ws = torch.empty(max(256, dst.dst_matmul_fp8_workspace_bytes(21, 50, d)), dtype=torch.uint8, device="cuda")
    outs = []
    for held in (0, 255):
        q = dst.Fp8Matrix(21, d)
        q.q.view(torch.uint8).fill_(held)
        q.scale.fill_(held)
        dst.dst_rmsnorm(x, None, q=q)
        outs.append(torch.empty(21, 50, device="cuda"))
        dst.dst_matmul_fp8(q, w, outs[-1], ws)
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(1, 33), (2, 300), (1, 5000), (40, 1000), (600, 3001), (1, 33708), (90, 33708), (1, 300000)])
def test_alternatives_of_logits_that_fall_with_the_index(rows, vocab, dtype):
    g = torch.Generator().manual_seed(vocab)
    x = -1.2 * torch.log(torch.arange(1, vocab + 1, dtype=torch.float32)) + 0.3 * torch.randn(rows, vocab, generator=g)
    x[0, vocab // 3:] = -float("inf")
    x, targets = x.to(TYPES[dtype]).cuda(), torch.zeros(rows, dtype=torch.int64).cuda()
    for n in (1, 8, 9, 32):
        check_logprob(x, targets, 1.0, n)
        check_logprob(x.flip(1).contiguous(), targets + vocab - 1, 1.0, n, torch.int32)
    check_logprob(torch.zeros_like(x), targets, 1.0, 9)           # as many equal ones as there are
