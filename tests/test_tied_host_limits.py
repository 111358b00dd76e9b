"""What the binding of the operators around the tied weight takes and refuses, without a GPU."""
import pytest
import torch

from paper_1905_04035_b200 import tied

CPU = -1                                                    # torch's index of the device of a CPU tensor


def test_a_single_column_or_row_has_no_stride_of_its_own():
    x = torch.zeros(1, 5).t()                               # [5, 1] whose column reports a stride of 5
    assert x.stride() == (1, 5) and tied._matrix(x, 5, 1, CPU, "x")[1] == 1
    wide = torch.zeros(5, 8)
    assert tied._matrix(wide[:, 3:4], 5, 1, CPU, "x")[1] == 8
    assert tied._matrix(wide.t()[:, 2:3], 8, 1, CPU, "x")[1] == 1
    assert tied._matrix(wide[2:3], 1, 8, CPU, "x")[1] == 8
    assert tied._matrix(torch.zeros(8).expand(1, 8), 1, 8, CPU, "x")[1] == 8
    assert tied._matrix(torch.zeros(1).expand(1, 1), 1, 1, CPU, "x")[1] == 1
    assert tied._matrix(torch.zeros(3, 0), 3, 0, CPU, "x")[1] >= 0
    for bad in (torch.zeros(8).expand(5, 8), torch.zeros(1).expand(5, 1), torch.zeros(8, 5).t(), torch.zeros(5, 16)[:, ::2], torch.zeros(8, 1).t()[:, ::2]):
        with pytest.raises(ValueError):
            tied._matrix(bad, *bad.shape, CPU, "x")


def test_a_workspace_has_all_the_bytes_that_it_reports():
    for bad in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(64, 64)[:, ::2]):
        with pytest.raises(ValueError):
            tied._workspace(bad, CPU)
    whole = torch.empty(64, 64)
    assert tied._workspace(whole, CPU) == (whole.data_ptr(), 64 * 64 * 4) and tied._workspace(None, CPU) == (None, 0)
