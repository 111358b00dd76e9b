"""Parts of matrices in 4 bits that hold more: what lies beyond the part's columns and rows has no say in a product."""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def np64(t):
    return t.detach().cpu().double().numpy()


def product(a, b):
    out = torch.full((a.rows, b.rows), float("nan"), device="cuda")
    ws = torch.empty(max(256, dst.dst_matmul_fp4_workspace_bytes(a.rows, b.rows, a.cols)), dtype=torch.uint8, device="cuda")
    dst.dst_matmul_fp4(a, b, out, ws)
    x, y = np64(a.dequantize()), np64(b.dequantize())
    # sums of exact terms: 256 additions a step of 256 at most, four a step and the parts', with truncation (2u)
    tol = (256 + 4 * -(-a.cols // 256) + 16) * 2 * U * (np.abs(x) @ np.abs(y).T)
    assert (np.abs(np64(out) - x @ y.T) <= tol).all()
    return out


@pytest.mark.parametrize("cols", [128, 256, 384, 512, 640])
@pytest.mark.parametrize("m,n", [(5, 40), (130, 270), (300, 65)])
def test_first_columns_of_a_matrix_with_nan_beyond(m, n, cols):
    g = torch.Generator().manual_seed(cols)
    x, y = torch.randn(300, 900, generator=g), torch.randn(400, 900, generator=g)
    whole = [dst.Fp4Matrix(*t.shape) for t in (x, y)]
    own = [dst.Fp4Matrix(k, cols) for k in (m, n)]
    for t, k, matrix, alone in zip((x, y), (m, n), whole, own):
        dst.dst_quantize_fp4(t[:k, :cols].contiguous().cuda(), alone)
        t[:, cols:] = float("nan")
        t[k:] = float("nan")
        dst.dst_quantize_fp4(t.cuda(), matrix)
    got = product(whole[0].part(m, cols), whole[1].part(n, cols))
    assert torch.equal(got, product(*own))


@pytest.mark.parametrize("cols", [1, 31, 33, 100, 129, 333])
def test_parts_quantised_into_whatever_their_buffers_held(cols):
    g = torch.Generator().manual_seed(cols)
    a, b = dst.Fp4Matrix(200, 900), dst.Fp4Matrix(200, 900)
    nan = torch.full((200, 900), float("nan"), device="cuda")
    for matrix in (a, b):
        dst.dst_quantize_fp4(nan, matrix)
    parts = a.part(20, cols), b.part(150, cols)
    for part in parts:
        dst.dst_quantize_fp4(torch.randn(part.rows, cols, generator=g).cuda(), part)
    product(*parts)
