"""Dropout against the generator word by word."""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)


def rows(seed, n, d, dtype, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, d + pad, generator=gen, device="cuda").to(dtype)[:, :d]


def rng(seed, offset):
    return torch.tensor([seed, offset], device="cuda")


@TYPES
@pytest.mark.parametrize("n,d", [(1, 1), (3, 2), (5, 7), (2, 8), (9, 33), (70, 64), (4, 2050),
                                 (3, 5001)])
def test_dropout(dtype, n, d):
    for p, residual, pad in ((0.1, True, 0), (0.5, False, 3), (0.37, True, 5)):
        x, r = rows(1, n, d, dtype, pad), rows(2, n, d, dtype, pad) if residual else None
        state = rng(1234567890123, 1 << 33)
        out = torch.full((n, d + 3), 7.0, dtype=dtype, device="cuda")
        X.dropout_tensors(x, state, out[:, :d], p=p, residual=r)
        want, slack = F.dropout(x, state.cpu(), p, r)
        F.close(out[:, :d], want, dtype, slack)
        assert (out[:, d:] == 7).all()


def test_shares_and_ends():
    x = torch.ones(1000, 1001, device="cuda")
    for p in (0.0, 2.0 ** -33, 0.25, 0.9, 1 - 2.0 ** -33, 1.0):
        out = torch.empty_like(x)
        X.dropout_tensors(x, rng(-7, -1), out, p=p)
        share = (out == 0).double().mean().item()
        # six standard deviations of a share of 1001000 values
        assert abs(share - p) <= 6 * (p * (1 - p) / x.numel()) ** 0.5 + 1e-9
        if 0 < p < 0.95:
            assert torch.equal(out[out != 0], torch.full_like(out[out != 0], 1 / (1 - p)))
    assert (out == 0).all()


def test_rows_past_one_launch():
    """2^21 rows of 8200 16-bit columns, 34 GB in place, take two launches."""
    n, d = 1 << 21, 8200
    x = torch.ones(n, d, dtype=torch.float16, device="cuda")
    state = rng(9, 10)
    X.dropout_tensors(x, state, x, p=0.5)
    for first in (0, 1677720, n - 2):
        later = rng(9, 10 + first * (d // 2)).cpu()
        want = 2.0 * F.kept(later, 2, d, 0.5).half()
        assert torch.equal(x[first:first + 2].cpu(), want)


def test_what_is_dropped_is_not_looked_at():
    x = torch.full((64, 256), float("nan"), device="cuda")
    r = rows(3, 64, 256, torch.float32)
    state = rng(5, 6)
    out = torch.empty_like(x)
    X.dropout_tensors(x, state, out, p=0.5, residual=r)
    keep = F.kept(state.cpu(), 64, 256, 0.5).cuda()
    assert out[keep].isnan().all() and torch.equal(out[~keep], r[~keep])
    X.dropout_tensors(x, state, out, p=1.0, residual=r)
    assert torch.equal(out, r)
