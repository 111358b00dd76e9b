"""Refusals of the operators around the tied weight: bad arguments are rejected before any CUDA call."""
import ctypes

import pytest
import torch

import paper_1905_04035_b200 as dst
from paper_1905_04035_b200 import binding
from paper_1905_04035_b200.build import build_library

FAKE = 0x10000            # never dereferenced
F32, BF16, I32, I64 = 0, 1, 0, 1


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    return dst.load_library()


def drop(p=0.1, seed=1, offset=0, device=None, row_offset=0):
    return ctypes.byref(binding._Dropout(p, seed, offset, device, row_offset))


def fp8(rows, cols, ld=None, ld_scale=None, block=0, q=FAKE, scale=FAKE):
    ld = -(-cols // 16) * 16 if ld is None else ld
    return ctypes.byref(binding._Fp8(q, scale, rows, cols, ld, -(-cols // 512) if ld_scale is None else ld_scale, block, 0))


def dropout(lib, x=FAKE, ldx=8, xt=F32, res=None, ldr=0, out=FAKE * 2, ldo=8, ot=F32, rows=4, d=8, dr=None):
    return lib.dst_dropout(x, ldx, xt, res, ldr, out, ldo, ot, rows, d, 1.0, drop() if dr is None else dr, None)


def test_dropout_refusals(lib):
    assert dropout(lib, xt=2) == 2 and dropout(lib, ot=-1) == 2
    assert dropout(lib, x=None) == 1 and dropout(lib, out=None) == 1
    assert dropout(lib, ldx=7) == 1 and dropout(lib, ldo=7) == 1 and dropout(lib, res=FAKE, ldr=7) == 1
    assert dropout(lib, rows=-1) == 1 and dropout(lib, d=-1) == 1
    assert dropout(lib, x=FAKE + 2) == 1 and dropout(lib, out=FAKE + 1, ot=BF16) == 1 and dropout(lib, res=FAKE + 2, ldr=8) == 1
    for p in (-0.1, 1.1, float("nan")):
        assert dropout(lib, dr=drop(p)) == 1
    assert dropout(lib, dr=drop(device=FAKE + 4)) == 1
    assert dropout(lib, dr=drop(row_offset=-1)) == 1 and dropout(lib, dr=drop(row_offset=(1 << 32) - 3)) == 1
    assert dropout(lib, out=FAKE, ldo=16, rows=4) == 1                          # in place with another row distance
    assert dropout(lib, out=FAKE, ot=BF16) == 1                                 # in place with another type
    assert dropout(lib, res=FAKE * 2, ldr=16) == 1
    assert lib.dst_dropout(FAKE, 8, F32, None, 0, FAKE * 2, 8, F32, 4, 8, 1.0, None, None) == 1
    assert dropout(lib, rows=(1 << 32) + 1) == 2 and dropout(lib, d=(1 << 30) + 1, ldx=1 << 31, ldo=1 << 31) == 2
    assert dropout(lib, x=None, out=None, rows=0) == 0 and dropout(lib, x=None, out=None, d=0, ldx=0, ldo=0) == 0


def embed(lib, idx=FAKE, n=4, it=I64, w=FAKE, vocab=10, d=8, wt=F32, pos=None, n_pos=0, out=FAKE, ot=F32, dr=None, res=None):
    return lib.dst_embed(idx, n, it, w, vocab, d, wt, pos, n_pos, out, ot, 1.0, dr, res, None)


def test_embed_refusals(lib):
    assert embed(lib, it=2) == 2 and embed(lib, wt=3) == 2 and embed(lib, ot=3) == 2
    for bad in (dict(idx=None), dict(w=None), dict(out=None), dict(n=-1), dict(vocab=-1), dict(d=-1), dict(idx=FAKE + 4), dict(it=I32, idx=FAKE + 2),
                dict(w=FAKE + 2), dict(out=FAKE + 2), dict(pos=FAKE, n_pos=0), dict(pos=FAKE + 2, n_pos=3), dict(n_pos=-1), dict(res=FAKE + 4), dict(dr=drop(2.0))):
        assert embed(lib, **bad) == 1, bad
    assert embed(lib, vocab=(1 << 30) + 1) == 2 and embed(lib, n=(1 << 32) + 1) == 2
    assert embed(lib, idx=None, out=None, n=0) == 0 and embed(lib, idx=FAKE, w=None, out=None, d=0) == 0


def test_quantize_refusals(lib):
    def call(x=FAKE, ldx=200, xt=F32, rows=10, cols=200, q="", qt=None):
        return lib.dst_quantize_fp8(x, ldx, xt, rows, cols, fp8(10, 200) if q == "" else q, qt, None)
    assert call(xt=5) == 2
    assert call(q=None) == 1 and call(x=None) == 1 and call(ldx=199) == 1 and call(x=FAKE + 1) == 1
    assert call(q=fp8(11, 200)) == 1 and call(q=fp8(10, 199)) == 1 and call(qt=fp8(10, 200)) == 1
    assert call(q=fp8(10, 200, ld=200)) == 1 and call(q=fp8(10, 200, ld=192)) == 1                    # not a multiple of 16, too short
    assert call(q=fp8(10, 200, q=FAKE + 8)) == 1 and call(q=fp8(10, 200, q=None)) == 1 and call(q=fp8(10, 200, scale=None)) == 1
    assert call(q=fp8(10, 200, ld_scale=0)) == 1 and call(q=fp8(10, 200, scale=FAKE + 8)) == 1 and call(q=fp8(10, 200, block=2)) == 1
    assert call(q=fp8(10, 200, block=1), qt=fp8(200, 10, block=0)) == 1                              # kinds that disagree
    assert call(rows=-1) == 1
    assert lib.dst_quantize_fp8(None, 0, F32, 0, 0, fp8(0, 0), None, None) == 0


def test_matmul_refusals(lib):
    need = dst.dst_matmul_fp8_workspace_bytes
    def call(a="", b="", out=FAKE, ldo=40, ot=F32, ws=FAKE, ws_bytes=None):
        return lib.dst_matmul_fp8(fp8(30, 200) if a == "" else a, fp8(40, 200) if b == "" else b, out, ldo, ot, ws,
                                  need(30, 40, 200) if ws_bytes is None else ws_bytes, None)
    assert call(ot=7) == 2
    assert call(a=None) == 1 and call(b=None) == 1 and call(out=None) == 1 and call(ldo=39) == 1 and call(out=FAKE + 2) == 1
    assert call(b=fp8(40, 208)) == 1                                                                  # inner sizes differ
    assert call(a=fp8(30, 200, ld=199)) == 1 and call(b=fp8(40, 200, block=1, ld_scale=0)) == 1
    assert lib.dst_matmul_fp8(fp8(0, 200), fp8(40, 200), None, 40, F32, None, 0, None) == 0
    assert lib.dst_matmul_fp8(fp8(30, 200), fp8(0, 200), None, 0, F32, None, 0, None) == 0
    big = need(512, 512, 1 << 17)
    if big:
        many = dict(a=fp8(512, 1 << 17), b=fp8(512, 1 << 17), ldo=512)
        assert call(**many, ws_bytes=4) == 3 and call(**many, ws=None, ws_bytes=big) == 1 and call(**many, ws=FAKE + 8, ws_bytes=big) == 1
    for M, N, K in ((30, 40, 200), (512, 512, 1 << 17), (8000, 512, 33708), (8000, 33708, 512)):
        assert all(need(m, n, k) <= need(M, N, K) for m in (1, M // 3, M - 1) for n in (1, N // 2, N) for k in (1, K // 2, K))
    assert need(0, 5, 5) == 0 and need(-1, 5, 5) == 0 and need(1 << 31, 5, 5) == 0


def test_linear_refusals(lib):
    need = dst.dst_linear_fp8_workspace_bytes(30, 40, 200)
    assert need > 0 and dst.dst_linear_fp8_workspace_bytes(30, -1, 200) == 0
    def call(x=FAKE, ldx=200, xt=F32, m=30, w="", out=FAKE, ldo=40, ot=F32, ws=FAKE, ws_bytes=need):
        return lib.dst_linear_fp8(x, ldx, xt, m, fp8(40, 200, block=1) if w == "" else w, out, ldo, ot, ws, ws_bytes, None)
    assert call(xt=3) == 2 and call(ot=3) == 2
    assert call(x=None) == 1 and call(ldx=199) == 1 and call(m=-1) == 1 and call(w=None) == 1 and call(out=None) == 1 and call(ldo=39) == 1
    assert call(ws=None) == 1 and call(ws=FAKE + 8) == 1 and call(ws_bytes=100) == 3
    assert call(m=0, x=None, out=None) == 0


def test_sample_refusals(lib):
    def call(x=FAKE, ld=100, t=F32, rows=3, vocab=100, u=FAKE, temp=None, k=None, p=None, mp=None, tok=FAKE, tt=I64, prob=None):
        return lib.dst_sample(x, ld, t, rows, vocab, u, temp, k, p, mp, tok, tt, prob, None)
    assert call(t=2) == 2 and call(tt=2) == 2 and call(vocab=327681, ld=327681) == 2 and call(rows=(1 << 27) + 1) == 2
    for bad in (dict(x=None), dict(ld=99), dict(u=None), dict(tok=None), dict(rows=-1), dict(vocab=-1), dict(vocab=0), dict(x=FAKE + 2), dict(tok=FAKE + 4),
                dict(tt=I32, tok=FAKE + 2), dict(u=FAKE + 1), dict(temp=FAKE + 1), dict(k=FAKE + 1), dict(p=FAKE + 1), dict(mp=FAKE + 1), dict(prob=FAKE + 1)):
        assert call(**bad) == 1, bad
    assert call(rows=0, x=None, u=None, tok=None) == 0


def test_binding_refuses_tensors_off_the_gpu_and_of_other_types():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        dst.dst_dropout(x, torch.zeros(4, 8), 0.1, 1)
    with pytest.raises(ValueError):
        dst.dst_sample(x, torch.zeros(4), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(TypeError):
        dst.dst_embed(torch.zeros(3), x, x)
    with pytest.raises(TypeError):
        dst.dst_sample(x, torch.zeros(4), torch.zeros(4))
    with pytest.raises(ValueError):
        dst.dst_quantize_fp8(x, None, None)
    with pytest.raises(ValueError):
        dst.Fp8Matrix(4, 8, 3, device="cpu")
    m = dst.Fp8Matrix(300, 200, device="cpu")
    with pytest.raises(ValueError):
        m.part(301, 200)
    assert m.part(10, 130).q.shape[0] == 10 and m.q.shape == (300, 208) and m.scale.shape == (3, 1, 512)
