"""Router kernels against the 64-bit form.

Choices, slots and counts have one right value. An exponential of x <= 0 is
within (4 |x| + 4) U, a softmax's sum adds at most 24 roundings, so with the
logits' range R a probability is within (8 R + 40) U of itself; sums over
tokens add a term per addition in a chain (at most 100 + tokens / 256).
"""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X

pytestmark = pytest.mark.gpu
U = F.U


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def run(logits, k, mask=None, capacity=0, coef=0.01, renorm=True):
    n, e = logits.shape
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.full(s, -7.0, device="cuda")  # noqa: E731
    o = {"experts": i32(n, k), "weights": f32(n, k), "slots": i32(n, k), "counts": i32(e),
         "prob_sums": f32(e), "loss": f32(1), "rows": i32(1)}
    work = torch.empty(X.route_workspace(e), dtype=torch.uint8, device="cuda")
    X.route_tensors(logits, *o.values(), work, mask=mask, capacity=capacity, coef=coef,
                    renorm=renorm)
    return o


def check(logits, k, **kw):
    got, want = run(logits, k, **kw), F.route(logits, k, **kw)
    for name in ("experts", "slots", "counts"):
        assert torch.equal(got[name].cpu(), want[name]), name
    assert int(got["rows"]) == want["rows"]
    near = (8 * F.logit_range(logits, kw.get("mask")) + 40) * U
    w = want["weights"]
    F.close(got["weights"], w, torch.float32, near * w.abs())
    chain = near + (100 + len(logits) / 256) * U
    F.close(got["prob_sums"], want["prob_sums"], torch.float32, chain * want["prob_sums"])
    F.close(got["loss"], torch.tensor([want["loss"]]), torch.float32,
            (2 * chain) * abs(want["loss"]))
    return got


def logits_of(n, e, dtype, seed, pad=0):
    g = gen(seed)
    x = 2 * torch.randn(n, e + pad, generator=g, device="cuda")
    x += torch.randn(e + pad, generator=g, device="cuda")
    return x.to(dtype)[:, :e]


@pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)
@pytest.mark.parametrize("n,e,k", [(1, 1, 1), (1, 8, 2), (5, 16, 16), (64, 17, 4), (65, 60, 4),
                                   (130, 64, 6), (200, 128, 8), (333, 160, 7), (257, 256, 8),
                                   (70, 257, 8), (40, 512, 16), (33, 1000, 5), (17, 1024, 1)])
def test_choices_slots_counts_loss(dtype, n, e, k):
    for i, (mask, cap, renorm, pad) in enumerate(
            [(None, 0, True, 0), (3, max(1, n * k // e), False, 3), (2, 1, True, 8)]):
        x = logits_of(n, e, dtype, n * e + i, pad)
        m = None
        if mask:
            m = (torch.arange(n, device="cuda") % mask != 0).to(torch.uint8)
        check(x, k, mask=m, capacity=cap, renorm=renorm)


@pytest.mark.parametrize("n,e", [(6000, 24), (2100, 128), (1500, 300), (20000, 5)])
def test_many_tokens(n, e):
    """Several blocks and tiles per block."""
    check(logits_of(n, e, torch.bfloat16, n), min(e, 3), capacity=n // 4)


def test_largest_grid():
    """Tiles in turn within a block (more tokens than blocks hold at once):
    places are the ranks among the tokens before."""
    n, e, k = 70001, 12, 2
    x = logits_of(n, e, torch.float32, 5)
    got = run(x, k, capacity=9000)
    order = torch.sort(x.cpu(), dim=1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(got["experts"].cpu().long(), order)
    hot = torch.zeros(n, e, dtype=torch.int64).scatter_(1, order, 1)
    place = (hot.cumsum(0) - hot).gather(1, order)
    assert torch.equal(got["slots"].cpu().long(), torch.where(place < 9000, place, -1))
    assert torch.equal(got["counts"].cpu().long(), hot.sum(0))
    p = torch.softmax(x.cpu().double(), 1).sum(0)
    near = (8 * F.logit_range(x) + 140 + n / 256) * U
    F.close(got["prob_sums"], p, torch.float32, near * p)


@pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)
def test_ties_go_to_the_lowest_index(dtype):
    for e in (7, 64, 200, 600):
        x = torch.zeros(9, e, dtype=dtype, device="cuda")
        x[1::2, e // 2:] = 1
        x[2, 3] = -0.0  # equal to 0
        x[4] = torch.finfo(dtype).min  # the lowest number is a number
        x[5] = torch.finfo(dtype).min
        x[5, e - 1] = torch.finfo(dtype).max
        check(x, 5)
        check((torch.arange(9 * e, device="cuda") * 7919 % 4).view(9, e).to(dtype), 6)


def test_rows_without_a_choice():
    """Minus infinities, masked tokens (whatever they hold), fewer numbers
    than choices."""
    e, k = 20, 4
    x = logits_of(12, e, torch.float32, 1)
    x[0] = -torch.inf
    x[1, 2:] = -torch.inf
    x[2, :e - 1] = -torch.inf
    m = torch.ones(12, dtype=torch.uint8, device="cuda")
    m[4:8] = 0
    x[4], x[5, 3], x[6] = torch.nan, torch.inf, -torch.inf
    got = check(x, k, mask=m, capacity=3)
    assert int(got["rows"]) == 7 and (got["experts"][0] == -1).all()
    assert (got["experts"][1, 2:] == -1).all() and (got["weights"][1, 2:] == 0).all()
    for renorm in (True, False):
        got = check(x, k, mask=torch.zeros_like(m), renorm=renorm)
        assert int(got["rows"]) == 0 and float(got["loss"]) == 0
        assert (got["prob_sums"] == 0).all() and (got["weights"] == 0).all()
    check(torch.full((70, 3), -torch.inf, device="cuda"), 2)


def test_nan_logits():
    """A NaN is never chosen and shows in the sums and the loss."""
    x = logits_of(6, 10, torch.float32, 2)
    x[2, 4] = torch.nan
    got = run(x, 3)
    want = F.route(x, 3)
    assert torch.equal(got["experts"].cpu(), want["experts"])
    assert not (got["experts"][2] == 4).any()
    assert got["prob_sums"].isnan().all() and got["loss"].isnan().all()
    assert int(got["rows"]) == 6


@pytest.mark.parametrize("renorm", [True, False])
def test_rows_of_nan(renorm):
    """A row without a number has no choice and weights of 0, whatever its
    probabilities; one with a single number chooses that."""
    for e in (12, 100, 300):
        x = logits_of(5, e, torch.float32, e)
        x[1] = torch.nan
        x[3] = torch.nan
        x[3, 7] = 0.5
        got = run(x, 3, renorm=renorm)
        assert (got["experts"][1] == -1).all() and (got["weights"][1] == 0).all()
        assert got["experts"][3].tolist() == [7, -1, -1]
        assert (got["weights"][3, 1:] == 0).all()
        assert (got["slots"][1] == -1).all() and got["loss"].isnan().all()


def test_no_tokens():
    got = run(torch.empty(0, 9, device="cuda"), 2)
    assert (got["counts"] == 0).all() and (got["prob_sums"] == 0).all()
    assert float(got["loss"]) == 0 and int(got["rows"]) == 0


def test_same_bits_again():
    x = logits_of(5000, 64, torch.float32, 3)
    a, b = run(x, 4), run(x, 4)
    for name in a:
        assert torch.equal(a[name], b[name])


def backward(x, k, renorm, mask=None, dloss=1.0, dweights=True, coef=0.3, scale_counts=1):
    r = run(x, k, mask=mask, coef=coef, renorm=renorm)
    n, e = x.shape
    dw = torch.randn(n, k, generator=gen(9), device="cuda") if dweights else None
    dl = None if dloss is None else torch.tensor([dloss], device="cuda")
    counts, rows = r["counts"] * scale_counts, r["rows"] * scale_counts
    out = torch.full((n, e), 3.0, dtype=x.dtype, device="cuda")
    X.route_backward_tensors(x, r["experts"], counts, rows, out, dweights=dw, dloss=dl, mask=mask,
                             coef=coef, renorm=renorm)
    want, size = F.route_backward(x, r["experts"].cpu(), counts, int(rows), k, dw, dloss, mask,
                                  coef, renorm)
    F.close(out, want, x.dtype, (8 * F.logit_range(x, mask) + 80) * U * size)
    return out


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)
@pytest.mark.parametrize("n,e,k", [(1, 1, 1), (3, 8, 2), (50, 16, 16), (65, 60, 4), (130, 64, 6),
                                   (99, 100, 3), (257, 256, 8), (70, 300, 8), (33, 1000, 5),
                                   (3000, 24, 2)])
def test_backward(renorm, dtype, n, e, k):
    m = (torch.arange(n, device="cuda") % 4 != 1).to(torch.uint8)
    backward(logits_of(n, e, dtype, n + e), k, renorm)
    backward(logits_of(n, e, dtype, n + e, 3), k, renorm, m, -2.0)
    backward(logits_of(n, e, dtype, n + e), k, renorm, m, None)
    backward(logits_of(n, e, dtype, n + e), k, renorm, None, 1.0, False, scale_counts=4)


@pytest.mark.parametrize("renorm", [True, False])
def test_backward_of_rows_without_a_choice(renorm):
    x = logits_of(9, 12, torch.float32, 1)
    x[0] = -torch.inf
    x[1, 2:] = -torch.inf
    x[2, 3] = -torch.inf
    m = torch.ones(9, dtype=torch.uint8, device="cuda")
    m[4:6] = 0
    x[4], x[5, 3] = torch.nan, torch.inf
    out = backward(x, 3, renorm, m)
    assert (out[0] == 0).all() and (out[4:6] == 0).all() and (out[1, 2:] == 0).all()
    assert out[2, 3] == 0 and out.isfinite().all()


@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(renorm):
    """The choices stay fixed over the step, as in the gradient: the k largest
    logits are raised above the others. Step 1e-4: truncation 1e-8, rounding
    of the kernel below 1e-5 of the vectors' lengths."""
    n, e, k, coef = 11, 20, 3, 5.0
    x = torch.randn(n, e, generator=gen(6), device="cuda")
    x[:, 4:4 + k] += 6 + torch.arange(k, device="cuda")
    c = torch.randn(n, k, generator=gen(7), device="cuda")
    x.requires_grad_()
    experts, weights, _, counts, _, loss, _ = X.route(x, k, coef=coef, renorm=renorm)
    ((weights * c).sum() + loss.sum() * 2).backward()
    at, load = experts.cpu().long(), counts.cpu().double()

    def value(x):
        p = torch.softmax(x, 1)
        w = p.gather(1, at)
        if renorm:
            w = w / w.sum(1, keepdim=True)
        balance = coef * e * (load / (n * k) * p.sum(0) / n).sum()
        return (w * c.cpu().double()).sum() + 2 * balance

    x0, g = x.detach().cpu().double(), x.grad.cpu().double()
    for _ in range(3):
        v = torch.randn(n, e, dtype=torch.float64)
        slope = (value(x0 + 1e-4 * v) - value(x0 - 1e-4 * v)) / 2e-4
        assert abs(slope - (g * v).sum()) <= 1e-5 * g.norm() * v.norm()
