"""Where the norm's outputs may lie: in x's and in residual's place, with the stream kept elsewhere or not at all; never in the stream's own."""
import pytest
import torch

import paper_1905_04035_b200 as dst

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,d", [(3, 300), (400, 512), (5, 1021), (2, 9000)])
def test_the_result_in_an_input_s_place(rows, d, dtype):
    g = torch.Generator().manual_seed(d)
    x, r = (torch.randn(rows, d, generator=g).to(dtype).cuda() for _ in range(2))
    w = torch.randn(d, generator=g).cuda()
    want, stream = torch.empty_like(x), torch.empty_like(x)
    dst.dst_rmsnorm(x, w, want, residual=r, sum_out=stream)
    for place in ("x", "residual"):
        for keeps in (True, False):
            a, b, s = x.clone(), r.clone(), torch.empty_like(x)
            dst.dst_rmsnorm(a, w, a if place == "x" else b, residual=b, sum_out=s if keeps else None)
            assert torch.equal(a if place == "x" else b, want) and torch.equal(b if place == "x" else a, r if place == "x" else x)
            assert not keeps or torch.equal(s, stream)
    a, b = x.clone(), r.clone()
    dst.dst_rmsnorm(a, w, a, residual=b, sum_out=b)           # both inputs replaced
    assert torch.equal(a, want) and torch.equal(b, stream)
    for s in (a, b, torch.empty_like(x)):
        with pytest.raises(dst.DstError):
            dst.dst_rmsnorm(a, w, s, residual=b, sum_out=s)
