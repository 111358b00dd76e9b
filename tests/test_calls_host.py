"""The library's entries as a Python module: arguments reach the library as through ctypes, and what is no argument is refused."""
import pytest
import torch

import paper_1905_04035_b200 as dst
from paper_1905_04035_b200 import binding, tied
from paper_1905_04035_b200.build import build_library

FAKE = 0x10000            # never dereferenced
CPU = -1


@pytest.fixture(scope="module", autouse=True)
def calls():
    build_library()
    return binding.load_calls()


def entries(calls):
    return [n for n in dir(calls) if n.startswith("dst_")]


def test_every_entry_has_the_library_s_arguments(calls):
    names = entries(calls)
    assert len(names) >= 16 and set(names) <= set(binding.SYMBOLS)
    for name in names:
        n = len(binding.SYMBOLS[name][1])
        for bad in (n - 1, n + 1):
            with pytest.raises(TypeError):
                getattr(calls, name)(*[None] * bad)
        with pytest.raises(TypeError):                        # a number is missing
            getattr(calls, name)(*[None] * n)


def test_numbers_and_pointers_arrive_where_they_belong(calls):
    lib = dst.load_library()
    good = [FAKE, 100, 0, 0, 100, None, 1, 1.0, None, None, None, None, 0, None, None, None, None]
    for name in ("dst_logprob",):
        assert getattr(calls, name)(*good) == getattr(lib, name)(*good) == 0
        for place, value in ((0, FAKE + 1), (1, 99), (2, 7), (3, -1), (4, 1 << 31), (5, FAKE + 4), (6, 9), (7, 0.0), (7, float("nan")), (8, FAKE + 2), (11, FAKE + 3), (12, 33), (12, -1), (13, FAKE + 4), (15, FAKE + 4)):
            args = list(good)
            args[place] = value
            assert getattr(calls, name)(*args) == getattr(lib, name)(*args) != 0, (place, value)
    for place, value in ((2, 1 << 31), (6, -(1 << 31) - 1), (1, 1 << 63), (0, 1 << 64)):
        args = list(good)
        args[place] = value
        with pytest.raises(OverflowError):
            calls.dst_logprob(*args)
    for place in (0, 1, 7):
        args = list(good)
        args[place] = "x"
        with pytest.raises(TypeError):
            calls.dst_logprob(*args)


def test_descriptions_are_told_apart(calls):
    q8, q4 = dst.Fp8Matrix(4, 256, device="cpu"), dst.Fp4Matrix(4, 256, device="cpu")
    args = [FAKE, 256, 0, 4, 256, q4._c, None]
    assert calls.dst_quantize_fp4(FAKE, 255, 0, 4, 256, q4._c, None) == 1
    assert calls.dst_quantize_fp4(*args[:5], None, None) == 1
    for wrong in (q8._c, 5, q4):
        with pytest.raises(TypeError):
            calls.dst_quantize_fp4(*args[:5], wrong, None)
    with pytest.raises(TypeError):
        calls.dst_matmul_fp8(q8._c, q4._c, FAKE, 4, 0, None, 0, None)
    lists = (binding._Tensor * 3)()
    assert calls.dst_grad_norm(lists, 3, 1.0, FAKE + 1, None, 0, None) == 1


def test_tensors_are_looked_at(calls):
    x = torch.zeros(3, 8)
    assert calls.matrix(x, 3, 8, CPU, "x") == (x.data_ptr(), 8, 0) and calls.matrix(x.bfloat16()[:, :5], 3, 5, CPU, "x")[1:] == (8, 1)
    for bad, error, said in ((x.double(), TypeError, "x must be float32 or bfloat16, got torch.float64"), (x[0], ValueError, r"x must be \[3, 8\]"), (x.t(), ValueError, r"x must be \[3, 8\]"),
                             (x.expand(3, 8).t().contiguous().t(), ValueError, "contiguous rows"), (x[:1].expand(3, 8), ValueError, "contiguous rows"), ([1], TypeError, "x must be a tensor"), (None, TypeError, "x must be a tensor")):
        with pytest.raises(error, match=said):
            calls.matrix(bad, 3, 8, CPU, "x")
    with pytest.raises(ValueError, match="same device"):
        calls.matrix(x, 3, 8, 0, "x")
    v = torch.zeros(6, dtype=torch.int32)
    assert calls.vector(v, 6, torch.int32, CPU, "v") == v.data_ptr() and calls.vector(None, 6, torch.int32, CPU, "v") is None
    assert tied._vector(None, 6, torch.int32, CPU, "v") is None
    for bad, error, said in ((v.long(), TypeError, "v must be torch.int32, got torch.int64"), (v[:5], ValueError, r"v must be contiguous \[6\]"), (torch.zeros(12, dtype=torch.int32)[::2], ValueError, "contiguous"),
                             (v.view(2, 3), ValueError, "contiguous"), (3, TypeError, "v must be a tensor")):
        with pytest.raises(error, match=said):
            calls.vector(bad, 6, torch.int32, CPU, "v")
    with pytest.raises(ValueError, match="same device"):
        calls.vector(v, 6, torch.int32, 2, "v")
    assert calls.table(x, 3, torch.float32, CPU, "x") == (x.data_ptr(), 8) and calls.table(x[:, :0].contiguous(), 3, torch.float32, CPU, "x")[1] == 0
    for bad, error, said in ((x.int(), TypeError, "x must be torch.float32, got torch.int32"), (x[:2], ValueError, r"x must be contiguous \[3, n\]"), (x[:, :4], ValueError, "contiguous"), (v, TypeError, "float32"), (None, TypeError, "x must be a tensor")):
        with pytest.raises(error, match=said):
            calls.table(bad, 3, torch.float32, CPU, "x")
    with pytest.raises(ValueError, match="same device"):
        calls.table(x, 3, torch.float32, 0, "x")
    for wrong in (lambda: calls.matrix(x, 3, 8, CPU), lambda: calls.matrix(x, 3, 8, CPU, 5), lambda: calls.matrix(x, "3", 8, CPU, "x"), lambda: calls.vector(v, 6)):
        with pytest.raises(TypeError):
            wrong()
