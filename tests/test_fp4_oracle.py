"""The definitions in oracle/fp4_oracle.py by hand, and what the owner of a matrix in 4 bits says without a GPU."""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst
from oracle import fp4_oracle as o


def test_rounding_to_nearest_even():
    v = [0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 2.6, 3.5, 5.0, 5.01, 6.0, -0.75, -5.0]
    assert o.to_e2m1(np.array(v)).tolist() == [0, 0, 0.5, 1.0, 1.0, 2.0, 2.0, 3.0, 4.0, 4.0, 6.0, 6.0, -1.0, -4.0]


def test_scales():
    assert o.scale_of(6.0) == 1.0 and o.scale_of(6.1) == 2.0 and o.scale_of(3.0) == 0.5 and o.scale_of(1.0) == 0.25
    assert o.scale_of(0.0) == o.scale_of(2.0 ** -100) == 2.0 ** -102 and np.isnan(o.scale_of(np.inf)) and np.isnan(o.scale_of(np.nan))
    codes, scales = o.quantize(np.array([[6.0] + [0.3] * 31 + [12.0, -7.0]]))
    assert scales.tolist() == [[1.0, 2.0]] and codes[0, :2].tolist() == [6.0, 0.5] and codes[0, 32:].tolist() == [6.0, -4.0]
    assert o.dequantize(codes, scales)[0, 33] == -8.0


def test_owner_of_a_matrix_in_4_bits():
    m = dst.Fp4Matrix(130, 70, device="cpu")
    assert m.q.shape == (130, 48) and m.scale.shape == (2, 1, 512)
    m.q.zero_()
    m.q[129, 34] = 0x9F                                      # columns 68 and 69: -6 and -0.5
    m.scale.fill_(127)
    m.scale[1, 0, 16 * 1 + 4 * 0 + 2] = 130                  # row 129, block 2
    assert m.codes()[129, 66:].tolist() == [0, 0, -6.0, -0.5] and m.scales()[129].tolist() == [1, 1, 8]
    assert m.dequantize()[129, 68:].tolist() == [-48.0, -4.0]
    assert m.part(3, 33).scales().shape == (3, 2)
    for bad in (lambda: m.part(131, 70), lambda: dst.Fp4Matrix(-1, 3, device="cpu")):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):
        dst.TiedProjection(100, 64, 8, bits=4, device="cpu")  # no gradient through 4 bits
    with pytest.raises(ValueError):
        dst.TiedProjection(100, 64, 8, bits=5, training=False, device="cpu")
    p = dst.TiedProjection(100, 64, 8, bits=4, training=False, device="cpu")
    with pytest.raises(TypeError):
        p.logits(dst.Fp8Matrix(4, 64, device="cpu"), torch.empty(4, 100))
    with pytest.raises(TypeError):
        dst.TiedProjection(100, 64, 8, training=False, device="cpu").logits(dst.Fp4Matrix(4, 64, device="cpu"), torch.empty(4, 100))
