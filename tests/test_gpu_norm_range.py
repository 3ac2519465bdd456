"""Norm kernels where a rounding or a range could be lost: the 8-bit copy value
by value, scales of rows with small weights, gradients of large and small rows.
"""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X
from test_gpu_norm import gen, rows, run_norm

pytestmark = pytest.mark.gpu
U = F.U


def by_column(scale, d, group):
    return scale[:, torch.arange(d) // (group or d)]


@pytest.mark.parametrize("group", [32, 64, 128, 256, 0])
@pytest.mark.parametrize("n,d", [(4000, 64), (3001, 1999), (500, 3), (2000, 4096), (300, 16384),
                                 (601, 9001)])
def test_eight_bits_are_the_quotient(n, d, group):
    """32-bit rows, so that `out` is y unrounded: q is the quotient y / scale
    in 32 bits, to nearest even, in every value."""
    x = rows(gen(n + d), n, d, torch.float32)
    w = 1 + 0.1 * torch.randn(d, generator=gen(d), device="cuda")
    out, _, q, scale = run_norm(x, w, None, 1e-6, group)
    want = (out.cpu() / by_column(scale.cpu(), d, group)).to(torch.float8_e4m3fn)
    assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))
