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


def row_maxima(y, group):
    """max(max |y|, 2^-100) of every group of columns."""
    group = group or y.shape[1]
    return torch.stack([y[:, i:i + group].abs().amax(1).clamp_min(F.AMAX_MIN)
                        for i in range(0, y.shape[1], group)], 1)


@pytest.mark.parametrize("group", [32, 64, 128, 256, 0])
@pytest.mark.parametrize("n,d", [(4000, 64), (3001, 1999), (500, 3), (2000, 4096), (300, 16384),
                                 (601, 9001)])
def test_scales_are_the_maxima(n, d, group):
    """Of the values themselves: maxima and the quotient by 448 round alike."""
    x = rows(gen(n + d), n, d, torch.float32)
    w = 1 + 0.1 * torch.randn(d, generator=gen(d), device="cuda")
    out, _, _, scale = run_norm(x, w, None, 1e-6, group)
    assert torch.equal(scale.cpu(), row_maxima(out.cpu(), group) / 448)


@pytest.mark.parametrize("group", [64, 0])
@pytest.mark.parametrize("d", [50, 520, 4096, 16384])
def test_scales_of_small_weights(d, group):
    """h w leaves the range of normal numbers, y does not."""
    x = 1e-18 * (1 + torch.rand(9, d, generator=gen(d), device="cuda"))
    w = 1e-28 * (1 + torch.rand(d, generator=gen(1), device="cuda"))
    out, _, q, scale = run_norm(x, w, None, 0.0, group)
    assert torch.equal(scale.cpu(), row_maxima(out.cpu(), group) / 448)
    want = (out.cpu() / by_column(scale.cpu(), d, group)).to(torch.float8_e4m3fn)
    assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))
