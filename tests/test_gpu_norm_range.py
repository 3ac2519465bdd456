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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-17, 1e-15, 1e-13, 1e12, 1e13, 1e15, 1e17])
@pytest.mark.parametrize("n,d", [(5, 7), (40, 100), (600, 200), (30, 1999), (9, 4096), (3, 16384)])
def test_backward_of_large_and_small_rows(n, d, size, dtype):
    """1 / sqrt(mean) cubed leaves the range, the gradient does not. Bounds as
    for rows of ordinary size."""
    g = gen(n + d)
    h = (size * (0.5 + torch.rand(n, d, generator=g, device="cuda"))).to(dtype)
    dy = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    w = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    dx, dw = torch.empty_like(h), torch.empty(d, device="cuda")
    work = torch.empty(X.norm_workspace(d), dtype=torch.uint8, device="cuda")
    X.norm_backward_tensors(dy, h, w, dx, dw, work, eps=0.0)
    want, want_dw, terms, terms_dw = F.norm_backward(dy, h, w, 0.0, None)
    F.close(dx, want, dtype, 64 * U * terms)
    F.close(dw, want_dw, torch.float32, (100 + n / 256) * U * terms_dw)
