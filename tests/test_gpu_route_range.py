"""Router kernels on large finite logits: the largest of a row may be any
number, also a usual fill of padding rows like -1e30.

Bounds as in test_gpu_route.py. The rows' differences are 0, at most 40 or so
large that a power is 0, since powers below 2^-126 may be 0.
"""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X
from test_gpu_route import backward, check, run

pytestmark = pytest.mark.gpu

SIZES = [1e6, 1.5e9, 5e9, 1e10, 3e10, 1e20, 1e30, 2e38]
# 16 lanes per token ranked and one at a time, 32 lanes, 64 lanes
EXPERTS = [(40, 5), (40, 9), (300, 5), (700, 6)]


def large_rows(e, dtype, size, n):
    """n rows: ordinary ones between rows whose largest logit is about `size`
    in size, above or below zero."""
    g = torch.Generator(device="cuda").manual_seed(e)
    x = torch.randn(n, e, generator=g, device="cuda")
    x[1::9] = size
    x[2::9] = -size
    x[3::9] = 0
    x[3::9, 7] = size
    x[4::9, 11:] = -size
    x[5::9] = -size
    x[5::9, ::5] = -size * (1 - 2.0 ** -6)
    x[6::9] = size * (1 - 2.0 ** -6)
    x[6::9, 3::4] = size
    if size == 1e6:  # steps of 1/16 in 32 bits
        x[7::9] = -size + 20 * torch.rand(len(x[7::9]), e, generator=g, device="cuda")
    return x.to(dtype)


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("e,k", EXPERTS)
def test_forward(e, k, size, dtype, renorm):
    check(large_rows(e, dtype, size, 40), k, renorm=renorm, capacity=20)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("e,k", EXPERTS)
def test_forward_in_several_blocks(e, k, size):
    """Every row with a number counts, so the loss's shares stay in their range."""
    got = check(large_rows(e, torch.float32, size, 300), k)
    assert int(got["rows"]) == 300


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("e,k", EXPERTS)
def test_backward(e, k, size, dtype, renorm):
    backward(large_rows(e, dtype, size, 40), k, renorm)


@pytest.mark.parametrize("e", [40, 300, 700])
def test_bits_do_not_depend_on_the_neighbours(e):
    x = large_rows(e, torch.float32, 1e20, 40)
    plain = torch.randn(40, e, generator=torch.Generator(device="cuda").manual_seed(1),
                        device="cuda")
    a, mixed = run(plain, 4), plain.clone()
    mixed[1::3] = x[1::3]
    b = run(mixed, 4)
    keep = [t for t in range(40) if t % 3 != 1]
    assert torch.equal(a["weights"][keep], b["weights"][keep])


def test_a_batch_with_one_padding_row():
    """Eight equal logits of -1e30: 1/8 each, and nothing of it elsewhere."""
    x = torch.randn(64, 8, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    x[17] = -1e30
    got = run(x, 2)
    assert got["experts"][17].tolist() == [0, 1] and int(got["rows"]) == 64
    assert got["loss"].isfinite().all()
    F.close(got["weights"][17], torch.tensor([0.5, 0.5]), torch.float32, 20 * F.U)
    F.close(got["prob_sums"].sum().view(1), torch.tensor([64.0]), torch.float32, 64 * 200 * F.U)
    weights = X.route(x, 2, renorm=False)[1]
    F.close(weights[17], torch.tensor([0.125, 0.125]), torch.float32, 20 * F.U)
