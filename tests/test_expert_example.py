"""The expert-layer example's parts without a GPU."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


@pytest.mark.parametrize("n", [64, 128, 192, 256, 1000, 1024])
def test_scales_of_8_bit_rows(n):
    """Column c has the scale of its group of 128, whatever the row's length."""
    import expert_alltoall

    scale = 2.0 ** torch.arange(2 * -(-n // 128)).view(2, -1)
    q = torch.ones(2, n).to(torch.float8_e4m3fn)
    got = expert_alltoall.rows_in_floats(q, scale)
    assert torch.equal(got.float(), scale[:, torch.arange(n) // 128])
