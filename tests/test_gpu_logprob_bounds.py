"""Log probabilities against bounds that follow the kernels' own sums: what one very likely token leaves, every number that the call for
many rows gives, and the same rows in batches of any size.

With u = 2^-24.  A thread takes tiles of four vectors (16 fp32 or 32 bf16 logits) and adds up each tile in two chains that begin with what it
has: 8 or 16 additions, the chains' joining, and the largest logit's 1 taken off and put back: 2 kN + 3 roundings of a sum of positive
terms.  Where a tile raises its largest logit the sum is multiplied by an exponential (4u, a product, and 3u for each unit of the
distance, distances that add up to what E|z| counts).  Long rows are streamed by 256 threads at least, short ones leave a thread two
tiles: at most 2 + vocab / (1024 kN) of them.  Then 13 joins (lanes 5, warps 5, CTAs 3) of an addition, a product and an exponential's 4u; each
exponential itself 4u + 3u |z|:
    rho = (tiles (2 kN + 8) + 13 * 6 + 4 + 3 E|z|) u
bounds the relative error of r, the sum without the largest logit's 1, and of t; E|z|, the mean distance of what r holds, is at most
log vocab where all tokens count, and the gap where one token is far above equal others.
    log p:   rho r / (1 + r) + 4u log1p(r) + 4u |z|            entropy:  2 rho (H + r / (1 + r)) + 8u H
"""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst
import test_gpu_step as base
from oracle import step_oracle as o

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
np64, TYPES = base.np64, base.TYPES


def rho(vocab, dtype, mean_z):
    n = 4 if dtype == "f32" else 8
    return ((2 + -(-vocab // (1024 * n))) * (2 * n + 8) + 13 * 6 + 4 + 3 * mean_z) * U


class Want(base.Want):
    def __init__(self, x, scale, dtype):
        super().__init__(x, scale, dtype)
        self.rho = rho(x.shape[1], dtype, np.log(x.shape[1]))


# as many rows as are cut among CTAs, as are streamed or kept, and as the ring takes
@pytest.mark.parametrize("copies", [1, 12, 40, 120])
@pytest.mark.parametrize("vocab,dtype", [(5000, "f32"), (9000, "bf16"), (33708, "f32"), (33708, "bf16")])
def test_what_the_likeliest_token_leaves_is_accurate_relative_to_itself(vocab, dtype, copies):
    gaps = np.array([5.0, 10.0, 17.0, 25.0, 60.0])
    x = torch.full((6, vocab), -3.0)
    at = torch.tensor([0, 17, vocab // 2, vocab - 1, 4097, 99])
    for i, gap in enumerate(gaps):
        x[i, at[i]] = -3.0 + gap
    x[5, at[5]] = 197.0                                      # what is left is below 2^-126 and counts as zero
    x, targets, n = x.to(TYPES[dtype]).repeat(copies, 1).cuda(), at.repeat(copies).cuda(), 6 * copies
    new = lambda *s: torch.full(s, 7.5, device="cuda")  # noqa: E731
    logprob, entropy, stats, fused, fused_entropy = new(n), new(n), new(n, 2), new(n), new(n)
    one, d, back = torch.ones(n, device="cuda"), torch.empty(n, vocab, device="cuda"), torch.empty(n, vocab, device="cuda")
    dst.dst_logprob(x, targets, logprob, entropy=entropy, stats=stats)
    dst.dst_logprob_loss(x, targets, one, fused, d, entropy=fused_entropy)
    dst.dst_logprob_backward(x, targets, stats, one, back)
    r = (vocab - 1) * np.exp(-gaps)
    p, left = np.exp(-gaps) / (1 + r), r / (1 + r)           # of another token, and of all of them
    want, want_h = -np.log1p(r), np.log1p(r) + gaps * left
    rel = rho(vocab, dtype, gaps)
    for got, h in ((logprob, entropy), (fused, fused_entropy)):
        got, h = np64(got).reshape(copies, 6), np64(h).reshape(copies, 6)
        assert (np.abs(got[:, :5] - want) <= (rel + 4 * U) * np.abs(want)).all()
        assert (np.abs(h[:, :5] - want_h) <= (4 * rel + 8 * U) * want_h).all()
        assert (got[:, 5] == 0).all() and (h[:, 5] == 0).all()
    for g in (d, back):
        g = np64(g).reshape(copies, 6, vocab)
        mine = g[:, np.arange(5), at[:5].numpy()]
        # -expm1(log p): a rounding or two and log p's own error, for 1 - p as for log p
        assert (np.abs(mine - left) <= (rel + 12 * U) * left).all()
        other = g[:, np.arange(5), 1]
        assert (np.abs(other + p) <= (rel + 10 * U + 3 * U * gaps) * p).all()
        assert (g[:, 5] == 0).all()


@pytest.mark.parametrize("vocab,dtype", [(33708, "bf16"), (33708, "f32"), (9000, "bf16"), (70001, "bf16"), (30011, "f32")])
@pytest.mark.parametrize("slope", [0.0, 0.3])
def test_every_number_of_the_call_for_many_rows(vocab, dtype, slope):
    rows = 300
    x, targets, g = base.make_logits(rows, vocab, dtype, vocab, pad=3, masked=True)
    targets[7], targets[8] = -1, vocab + 5
    a, b = torch.randn(rows, generator=g), slope * torch.randn(rows, generator=g)
    logprob, lse, entropy = (torch.full((rows,), 7.5, device="cuda") for _ in range(3))
    d, buf = base.strided(rows, vocab, dtype, 3)
    dst.dst_logprob_loss(x, targets, a.cuda(), logprob, d, scale=0.9, dentropy=b.cuda(), lse=lse, entropy=entropy)
    w = Want(x, 0.9, dtype)
    base.near_sums(w, targets, logprob, lse, entropy)
    t = targets.cpu().numpy()
    t = np.where(t >= vocab, -1, t)
    base.near(d, o.logits_gradient(w.x, t, 0.9, np64(a), np64(b)), w.tol_grad(t, np64(a), np64(b)), dtype)
    assert base.untouched(buf, d)


@pytest.mark.parametrize("vocab,dtype", [(5000, "bf16"), (9001, "f32"), (33708, "bf16"), (33708, "f32")])
def test_rows_agree_to_rounding_in_batches_of_any_size_and_bit_for_bit_in_the_same(vocab, dtype):
    x, targets, g = base.make_logits(600, vocab, dtype, 5)
    a = torch.randn(600, generator=g).cuda()
    rows = slice(0, 3)
    w = Want(x[rows], 1.0, dtype)
    t = targets[rows].cpu().numpy()
    grad, tol = o.logits_gradient(w.x, t, 1.0, np64(a[rows]), np.zeros(3)), w.tol_grad(t, np64(a[rows]), np.zeros(3))
    for n in (3, 20, 60, 75, 150, 298, 600):
        seen = []
        for _ in range(2):
            out = [torch.full((n,), 7.5, device="cuda") for _ in range(5)]
            stats, d, back = torch.empty(n, 2, device="cuda"), torch.empty(n, vocab, device="cuda"), torch.empty(n, vocab, device="cuda")
            dst.dst_logprob(x[:n], targets[:n], out[0], lse=out[1], entropy=out[2], stats=stats)
            dst.dst_logprob_loss(x[:n], targets[:n], a[:n], out[3], d, entropy=out[4])
            dst.dst_logprob_backward(x[:n], targets[:n], stats, a[:n], back)
            seen.append(out + [stats, d, back])
        assert all(torch.equal(p, q) for p, q in zip(*seen))
        base.near_sums(w, targets[rows], out[0][rows], out[1][rows], out[2][rows])
        base.near_sums(w, targets[rows], out[3][rows], out[1][rows], out[4][rows])
        base.near(d[rows], grad, tol, what="in one pass, %d rows" % n)
        base.near(back[rows], grad, tol, what="apart, %d rows" % n)
