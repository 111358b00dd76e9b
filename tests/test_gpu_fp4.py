"""GPU parity of matrices in 4 bits against their 64-bit definition (oracle/fp4_oracle.py).

Tolerances, with u = 2^-24 and h = 2^-8 (half a bf16 step, relative): codes and scales are exact; a product's terms are exact in
fp32 (two 2-bit significands, scales of powers of two), sums of 64 are added up in fp32, at worst with truncation (2u an addition: four a step of
256, and up to 256 within the steps of one), and one rounding for each stretch moved to registers and each part of the inner dimension:
(256 + 4 steps + 16) 2u sum|terms| (+ h |out|)
"""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst
from oracle import fp4_oracle as o

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def np64(t):
    return t.detach().cpu().double().numpy()


def randn(rows, cols, dtype="f32", seed=0, pad=0, skew=0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn(rows * (cols + pad) + skew, generator=g).to(TYPES[dtype]).cuda()
    return buf[skew:].view(rows, cols + pad)[:, :cols]


def quantized(x):
    m = dst.Fp4Matrix(*x.shape)
    m.q.fill_(255)
    m.scale.fill_(255)
    dst.dst_quantize_fp4(x, m)
    return m


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (7, 64), (128, 128), (129, 257), (200, 16), (40, 1000), (5, 255)])
@pytest.mark.parametrize("xt,pad,skew", [("f32", 0, 0), ("bf16", 0, 0), ("bf16", 5, 3), ("f32", 8, 0), ("f32", 4, 1)])
def test_quantize(rows, cols, xt, pad, skew):
    x = randn(rows, cols, xt, rows + cols, pad, skew)
    x[rows // 2, cols // 2] *= 50
    m = quantized(x)
    codes, scales = o.quantize(np64(x))
    assert np.array_equal(np64(m.scales()), scales) and np.array_equal(np64(m.codes()), codes)
    words = -(-cols // 8) * 4
    spare = torch.stack([m.q[:, :words] & 15, m.q[:, :words] >> 4], -1).reshape(rows, -1)[:, cols:]
    assert bool((spare == 0).all()) and bool((m.q[:, words:] == 255).all())   # the rest of a word, and what was left alone
    assert torch.equal(m.dequantize(), m.codes() * m.scales().repeat_interleave(32, 1)[:, :cols])


def test_quantize_limits():
    f32 = torch.finfo(torch.float32)
    x = torch.zeros(8, 64)
    x[0, 1] = float("nan")
    x[1, 33] = float("-inf")
    x[2, :] = 2.0 ** -120
    x[3, :] = f32.max
    x[4, :5] = torch.tensor([6.0, 2.5, 3.5, 5.0, -0.25])
    x[5, :2] = torch.tensor([6.0000005, 1.0])
    x[6, 0] = f32.tiny / 4
    m = quantized(x.cuda())
    s, c = m.scales().cpu(), m.codes().cpu()
    assert torch.isnan(s[0, 0]) and s[0, 1] == 2.0 ** -102 and torch.isnan(s[1, 1]) and not torch.isnan(s[1, 0])
    assert bool((c[2] == 0).all()) and bool((c[3] * s[3, 0] >= f32.max * 0.75).all())
    assert c[4, :5].tolist() == [6, 2, 4, 4, 0] and s[4, 0] == 1 and s[5, 0] == 2 and bool((c[7] == 0).all())


def product(a, b, ot, pad=0, skew=0):
    M, N, K = a.rows, b.rows, a.cols
    buf = torch.full((M * (N + pad) + skew,), float("nan"), dtype=TYPES[ot], device="cuda")
    out = buf[skew:].view(M, N + pad)[:, :N]
    ws = torch.full((max(256, dst.dst_matmul_fp4_workspace_bytes(M, N, K)),), 255, dtype=torch.uint8, device="cuda")
    dst.dst_matmul_fp4(a, b, out, ws)
    x, y = np64(a.dequantize()), np64(b.dequantize())
    want, mag = x @ y.T, np.abs(x) @ np.abs(y).T
    tol = (256 + 4 * -(-K // 256) + 16) * 2 * U * mag + (H * np.abs(want) if ot == "bf16" else 0)
    off = np.abs(np64(out) - want)
    assert (off <= tol + 1e-37).all(), "worst %r of %r" % (off.max(), tol.flat[off.argmax()])
    spare = torch.ones_like(buf, dtype=torch.bool)
    spare.as_strided(out.size(), out.stride(), out.storage_offset()).fill_(False)
    assert bool(torch.isnan(buf[spare]).all())
    return out


SHAPES = [(1, 1, 1), (1, 300, 64), (5, 40, 33), (16, 16, 256), (17, 500, 255), (33, 129, 300), (64, 1000, 512), (65, 700, 257), (100, 129, 1000), (128, 128, 128),
          (129, 300, 513), (300, 65, 700), (1000, 10, 500), (257, 513, 1021), (1000, 1000, 64), (3, 5, 5000), (200, 300, 9000)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("ot,pad,skew", [("f32", 0, 0), ("bf16", 0, 0), ("bf16", 3, 1), ("f32", 5, 1)])
def test_matmul(M, N, K, ot, pad, skew):
    product(quantized(randn(M, K, seed=M)), quantized(randn(N, K, seed=N + 1) * 0.1), ot, pad, skew)


@pytest.mark.parametrize("M,N,K", [(1, 33708, 1024), (48, 33708, 512), (300, 33708, 1021), (2000, 1024, 600), (33708, 64, 500)])
def test_matmul_at_the_vocabulary(M, N, K):
    product(quantized(randn(M, K, seed=1)), quantized(randn(N, K, seed=2)), "f32")


def test_matmul_is_exact_on_small_whole_numbers_and_repeats_bit_for_bit():
    g = torch.Generator().manual_seed(3)
    for M, N, K in ((300, 400, 1000), (7, 4000, 600), (90, 500, 300)):
        values = torch.tensor([0.0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6])
        a, b = (values[torch.randint(0, 11, (n, K), generator=g)] for n in (M, N))
        a[:, ::32] = 6.0
        b[:, ::32] = -6.0                                     # every block's scale is 1
        qa, qb = quantized(a.cuda()), quantized(b.cuda())
        out = product(qa, qb, "f32")
        assert torch.equal(out.cpu().double(), a.double() @ b.double().T)
        assert torch.equal(out, product(qa, qb, "f32"))


def test_matmul_of_nothing_and_of_blocks_that_are_nan():
    out = torch.full((3, 4), 7.0, device="cuda")
    dst.dst_matmul_fp4(dst.Fp4Matrix(3, 0), dst.Fp4Matrix(4, 0), out)
    assert bool((out == 0).all())
    dst.dst_matmul_fp4(dst.Fp4Matrix(0, 5), dst.Fp4Matrix(4, 5), out[:0])
    x = torch.ones(3, 100)
    x[1, 40] = float("nan")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    dst.dst_matmul_fp4(quantized(x.cuda()), quantized(torch.ones(4, 100).cuda()), out, ws)
    assert bool(torch.isnan(out[1]).all()) and bool((out[[0, 2]] == 100).all())


def test_parts_of_larger_buffers():
    big_a, big_b = dst.Fp4Matrix(400, 900), dst.Fp4Matrix(500, 900)
    a, b = big_a.part(130, 333), big_b.part(270, 333)
    for m in (big_a, big_b):
        m.q.fill_(255)
        m.scale.fill_(255)
    dst.dst_quantize_fp4(randn(130, 333, seed=1), a)
    dst.dst_quantize_fp4(randn(270, 333, seed=2), b)
    product(a, b, "f32")


@pytest.mark.parametrize("M,V,D", [(1, 1000, 64), (7, 500, 130), (150, 1000, 512), (2, 10000, 2048), (5, 9000, 700), (33, 1500, 500), (64, 2000, 512), (17, 40, 64), (3, 8000, 1021), (20, 3000, 256)])
@pytest.mark.parametrize("xt,ot", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_projection(M, V, D, xt, ot):
    """The call that quantises on the way gives what quantising first gives."""
    x, w = randn(M, D, xt, 1, 3, 1), randn(V, D, "f32", 2)
    p = dst.TiedProjection(V, D, M, training=False, bits=4)
    p.update(w)
    assert np.array_equal(np64(p.weight.codes()), np64(quantized(w).codes()))
    out, apart = (torch.full((M, V), float("nan"), dtype=TYPES[ot], device="cuda") for _ in range(2))
    p.logits(x, out)
    q = quantized(x)
    p.logits(q, apart)
    a, b = np64(q.dequantize()), np64(p.weight.dequantize())
    want, tol = a @ b.T, (256 + 4 * -(-D // 256) + 16) * 2 * U * (np.abs(a) @ np.abs(b).T)
    for t in (out, apart):
        off = np.abs(np64(t) - want)
        assert (off <= tol + (H * np.abs(want) if ot == "bf16" else 0) + 1e-37).all(), off.max()
