"""Refusals of a step's operators and of the matrices in 4 bits: bad arguments are rejected before any CUDA call."""
import ctypes

import pytest
import torch

import paper_1905_04035_b200 as dst
from paper_1905_04035_b200 import binding, step
from paper_1905_04035_b200.build import build_library

FAKE = 0x10000            # never dereferenced
F32, BF16, I32, I64 = 0, 1, 0, 1
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    return dst.load_library()


def test_logprob_refusals(lib):
    def call(x=FAKE, ld=100, t=F32, rows=3, vocab=100, targets=FAKE, it=I64, scale=1.0, lp=FAKE, lse=None, ent=None, stats=None, n=0, tok=None, tlp=None, res=None):
        return lib.dst_logprob(x, ld, t, rows, vocab, targets, it, scale, lp, lse, ent, stats, n, tok, tlp, res, None)
    assert call(t=2) == 2 and call(it=2) == 2 and call(n=33, tok=FAKE) == 2
    assert call(vocab=(1 << 30) + 1, ld=1 << 31) == 2 and call(rows=(1 << 27) + 1) == 2
    for bad in (dict(x=None), dict(ld=99), dict(rows=-1), dict(vocab=-1), dict(vocab=0), dict(x=FAKE + 2), dict(x=FAKE + 1, t=BF16), dict(targets=FAKE + 4), dict(targets=FAKE + 2, it=I32),
                dict(targets=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(scale=3e38), dict(lp=FAKE + 2), dict(lse=FAKE + 1), dict(ent=FAKE + 2),
                dict(stats=FAKE + 2), dict(n=-1), dict(n=2, tok=FAKE + 4), dict(n=2, tlp=FAKE + 2), dict(res=FAKE + 4)):
        assert call(**bad) == 1, bad
    assert call(rows=0, x=None, targets=None) == 0 and call(rows=0, vocab=0, ld=0, x=None) == 0


def test_logprob_gradient_refusals(lib):
    def loss(x=FAKE, ld=100, t=F32, rows=3, vocab=100, targets=FAKE, it=I64, scale=1.0, a=FAKE, b=None, lp=FAKE, lse=None, ent=None, d=2 * FAKE, ldd=100, dt=F32, res=None):
        return lib.dst_logprob_loss(x, ld, t, rows, vocab, targets, it, scale, a, b, lp, lse, ent, d, ldd, dt, res, None)

    def back(x=FAKE, ld=100, t=F32, rows=3, vocab=100, targets=FAKE, it=I64, scale=1.0, stats=FAKE, ent=None, a=FAKE, b=None, d=2 * FAKE, ldd=100, dt=F32):
        return lib.dst_logprob_backward(x, ld, t, rows, vocab, targets, it, scale, stats, ent, a, b, d, ldd, dt, None)
    for call in (loss, back):
        assert call(t=2) == 2 and call(it=-1) == 2 and call(dt=2) == 2 and call(vocab=(1 << 30) + 1, ld=1 << 31, ldd=1 << 31) == 2
        for bad in (dict(x=None), dict(d=None), dict(ldd=99), dict(d=FAKE + 2), dict(a=FAKE + 2), dict(b=FAKE + 1), dict(targets=None), dict(scale=-1.0), dict(vocab=0),
                    dict(d=FAKE, ldd=104), dict(d=FAKE, dt=BF16)):
            assert call(**bad) == 1, (call.__name__, bad)
        assert call(rows=0, x=None, d=None) == 0
    assert loss(lp=FAKE + 1) == 1 and loss(lse=FAKE + 2) == 1 and loss(ent=FAKE + 1) == 1 and loss(res=FAKE + 4) == 1 and loss(targets=None, a=None) == 1
    assert back(stats=None) == 1 and back(stats=FAKE + 2) == 1 and back(b=FAKE, ent=None) == 1 and back(ent=FAKE + 2) == 1


def fp8(rows, cols, block=0, q=FAKE, scale=FAKE, ld=None, ld_scale=None):
    return ctypes.byref(binding._Fp8(q, scale, rows, cols, -(-cols // 16) * 16 if ld is None else ld, -(-cols // 512) if ld_scale is None else ld_scale, block, 0))


def test_rmsnorm_refusals(lib):
    A, B, C, D = (FAKE * i for i in (1, 2, 3, 4))
    def call(x=A, ldx=8, xt=F32, r=B, ldr=8, s=C, lds=8, st=F32, w=FAKE, eps=1e-6, out=D, ldo=8, ot=F32, q=None, inv=None, rows=4, d=8):
        return lib.dst_rmsnorm(x, ldx, xt, r, ldr, s, lds, st, w, eps, out, ldo, ot, q, inv, rows, d, None)
    assert call(xt=2) == 2 and call(st=2) == 2 and call(ot=2) == 2 and call(d=16385, ldx=16385, ldr=16385, lds=16385, ldo=16385) == 2 and call(rows=(1 << 31) + 1) == 2
    for bad in (dict(x=None), dict(ldx=7), dict(ldr=7), dict(lds=7), dict(ldo=7), dict(x=A + 2), dict(r=B + 1), dict(s=C + 2), dict(out=D + 2), dict(w=FAKE + 2), dict(inv=FAKE + 2),
                dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(out=None), dict(rows=-1), dict(d=-1), dict(q=fp8(4, 9)), dict(q=fp8(5, 8)), dict(q=fp8(4, 8, block=1)),
                dict(q=fp8(4, 8, q=FAKE + 8)), dict(out=A, ldo=16), dict(out=A, ot=BF16), dict(out=B, ldo=16), dict(out=C), dict(s=A, lds=16), dict(s=B, lds=16), dict(s=A, st=BF16, xt=F32)):
        assert call(**bad) == 1, bad
    assert call(rows=0, x=None, r=None, s=None, out=None) == 0 and call(d=0, ldx=0, ldr=0, lds=0, ldo=0, x=None) == 0


def test_rmsnorm_backward_refusals(lib):
    need = dst.dst_rmsnorm_backward_workspace_bytes(4, 8)
    assert need > 0 and dst.dst_rmsnorm_backward_workspace_bytes(-1, 8) == 0 and dst.dst_rmsnorm_backward_workspace_bytes(4, 16385) == 0
    A, B, C, D = (FAKE * i for i in (1, 2, 3, 4))
    def call(dy=A, ldy=8, yt=F32, h=B, ldh=8, ht=F32, w=FAKE, inv=FAKE, ds=C, ldds=8, dx=D, ldx=8, xt=F32, dw=FAKE, rows=4, d=8, ws=FAKE, nb=need):
        return lib.dst_rmsnorm_backward(dy, ldy, yt, h, ldh, ht, w, inv, ds, ldds, dx, ldx, xt, dw, rows, d, ws, nb, None)
    assert call(yt=2) == 2 and call(ht=2) == 2 and call(xt=2) == 2 and call(rows=(1 << 31) + 1) == 2
    for bad in (dict(dy=None), dict(h=None), dict(dx=None), dict(inv=None), dict(ldy=7), dict(ldh=7), dict(ldds=7), dict(ldx=7), dict(dy=A + 2), dict(h=B + 2), dict(ds=C + 1), dict(dx=D + 2),
                dict(w=FAKE + 1), dict(inv=FAKE + 2), dict(dw=FAKE + 2), dict(ws=None), dict(ws=FAKE + 8), dict(dx=A, ldx=16), dict(dx=A, xt=BF16, ds=None), dict(dx=B, ldx=16), dict(dx=C, ldx=16)):
        assert call(**bad) == 1, bad
    assert call(nb=need - 1) == 3 and call(d=0, ldy=0, ldh=0, ldds=0, ldx=0) == 0 and call(rows=0, dw=None, inv=None, ws=None) == 0


def tensors(*items):
    a = (binding._Tensor * max(1, len(items)))()
    for c, (data, n, t) in zip(a, items):
        c.data, c.n, c.type = data, n, t
    return a


def test_grad_norm_and_clip_refusals(lib):
    good = tensors((FAKE, 10, F32), (None, 0, BF16))
    need = lib.dst_grad_norm_workspace_bytes(good, 2)
    assert need > 0 and lib.dst_grad_norm_workspace_bytes(tensors(), 0) == 0 and lib.dst_grad_norm_workspace_bytes(tensors((None, 5, F32)), 1) == 0
    def norm(t=good, n=2, most=1.0, clip=FAKE, ws=FAKE, nb=need):
        return lib.dst_grad_norm(t, n, most, clip, ws, nb, None)
    for bad in (dict(n=-1), dict(t=None), dict(clip=None), dict(clip=FAKE + 2), dict(most=-1.0), dict(most=NAN), dict(ws=None), dict(ws=FAKE + 8), dict(t=tensors((FAKE + 2, 3, F32)), n=1),
                dict(t=tensors((FAKE, -1, F32)), n=1), dict(t=tensors((FAKE, 3, 2)), n=1), dict(t=tensors((None, 3, F32)), n=1)):
        assert norm(**bad) == 1, bad
    assert norm(nb=need - 1) == 3 and norm(t=tensors((FAKE, (1 << 44) + 1, F32)), n=1) == 2
    def clip(t=good, o=good, n=2, c=FAKE):
        return lib.dst_clip(t, o, n, c, None)
    for bad in (dict(n=-1), dict(t=None), dict(o=None), dict(c=None), dict(c=FAKE + 1), dict(o=tensors((FAKE, 11, F32), (None, 0, F32))), dict(o=tensors((FAKE, 10, BF16), (None, 0, F32)))):
        assert clip(**bad) == 1, bad
    assert clip(n=0, t=None, o=None) == 0
    many = tensors(*[(FAKE, 1 << 20, F32)] * 500)
    assert lib.dst_grad_norm_workspace_bytes(many, 500) >= lib.dst_grad_norm_workspace_bytes(many, 100) > 0


def fp4(rows, cols, ld=None, ld_scale=None, q=FAKE, scale=FAKE):
    return ctypes.byref(binding._Fp4(q, scale, rows, cols, -(-cols // 32) * 16 if ld is None else ld, -(-cols // 128) if ld_scale is None else ld_scale))


def test_fp4_refusals(lib):
    def quant(x=FAKE, ldx=200, xt=F32, rows=10, cols=200, q=""):
        return lib.dst_quantize_fp4(x, ldx, xt, rows, cols, fp4(10, 200) if q == "" else q, None)
    assert quant(xt=5) == 2
    for bad in (dict(q=None), dict(x=None), dict(ldx=199), dict(x=FAKE + 1), dict(q=fp4(11, 200)), dict(q=fp4(10, 199)), dict(q=fp4(10, 200, ld=104)), dict(q=fp4(10, 200, ld=96)), dict(q=fp4(10, 200, q=FAKE + 8)),
                dict(q=fp4(10, 200, q=None)), dict(q=fp4(10, 200, scale=None)), dict(q=fp4(10, 200, scale=FAKE + 8)), dict(q=fp4(10, 200, ld_scale=1)), dict(rows=-1)):
        assert quant(**bad) == 1, bad
    assert lib.dst_quantize_fp4(None, 0, F32, 0, 0, fp4(0, 0), None) == 0
    need = dst.dst_matmul_fp4_workspace_bytes
    def mul(a="", b="", out=FAKE, ldo=40, ot=F32, ws=FAKE, nb=None):
        return lib.dst_matmul_fp4(fp4(30, 200) if a == "" else a, fp4(40, 200) if b == "" else b, out, ldo, ot, ws, need(30, 40, 200) if nb is None else nb, None)
    assert mul(ot=7) == 2
    for bad in (dict(a=None), dict(b=None), dict(out=None), dict(ldo=39), dict(out=FAKE + 2), dict(b=fp4(40, 208)), dict(a=fp4(30, 200, ld=100))):
        assert mul(**bad) == 1, bad
    assert lib.dst_matmul_fp4(fp4(0, 200), fp4(40, 200), None, 40, F32, None, 0, None) == 0
    big = dict(a=fp4(512, 1 << 18), b=fp4(512, 1 << 18), ldo=512)
    nb = need(512, 512, 1 << 18)
    assert nb > 0 and mul(**big, nb=4) == 3 and mul(**big, ws=None, nb=nb) == 1 and mul(**big, ws=FAKE + 8, nb=nb) == 1
    for M, N, K in ((30, 40, 200), (512, 512, 1 << 17), (8000, 33708, 1024), (8000, 512, 33708)):
        assert all(need(m, n, k) <= need(M, N, K) for m in (1, M // 3, M - 1) for n in (1, N // 2, N) for k in (1, K // 2, K))
    assert need(0, 5, 5) == 0 and need(1 << 31, 5, 5) == 0
    lin = dst.dst_linear_fp4_workspace_bytes(30, 40, 200)
    def linear(x=FAKE, ldx=200, xt=F32, m=30, w="", out=FAKE, ldo=40, ot=F32, ws=FAKE, nb=lin):
        return lib.dst_linear_fp4(x, ldx, xt, m, fp4(40, 200) if w == "" else w, out, ldo, ot, ws, nb, None)
    assert linear(xt=3) == 2 and linear(ot=3) == 2 and linear(nb=100) == 3 and linear(m=0, x=None, out=None) == 0
    for bad in (dict(x=None), dict(ldx=199), dict(m=-1), dict(w=None), dict(out=None), dict(ldo=39), dict(ws=None), dict(ws=FAKE + 8)):
        assert linear(**bad) == 1, bad


def test_binding_refuses_tensors_off_the_gpu_and_of_other_types_and_shapes():
    x, v = torch.zeros(4, 8), torch.zeros(4)
    with pytest.raises(ValueError):
        dst.dst_logprob(x, torch.zeros(4, dtype=torch.int64), v)
    with pytest.raises(ValueError):
        dst.dst_rmsnorm(x, None, x)
    with pytest.raises(ValueError):
        dst.TensorList([x])
    with pytest.raises(ValueError):
        dst.dst_quantize_fp4(x, dst.Fp4Matrix(4, 8, device="cpu"))
    empty = dst.TensorList([])
    assert len(empty) == 0 and empty.distinct
    with pytest.raises(ValueError):
        dst.dst_grad_norm(empty, torch.zeros(2), 1.0)
    # what the binding looks at before it calls, with the CPU's tensors taken for a device's
    CPU = -1
    with pytest.raises(TypeError):
        step._stats(torch.zeros(4, 2, dtype=torch.float64), 4, CPU)
    for bad in (torch.zeros(4), torch.zeros(4, 3), torch.zeros(2, 4).t()):
        with pytest.raises(ValueError):
            step._stats(bad, 4, CPU)
    assert step._stats(None, 4, CPU) is None and step._stats(torch.zeros(4, 2), 4, CPU)


def test_lists_know_whether_their_tensors_share_memory():
    assert step._apart([]) and step._apart([(4, 8)]) and step._apart([(8, 12), (0, 4), (4, 8)])
    assert step._apart([(4, 4), (0, 8), (2, 2)])                  # (what is empty shares nothing)
    for bad in ([(0, 4), (0, 4)], [(8, 12), (0, 9)], [(0, 100), (8, 12), (200, 300)], [(0, 8), (7, 8)]):
        assert not step._apart(bad), bad
