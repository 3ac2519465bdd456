"""Dispatch and combine kernels against plain copies and the 64-bit form.

Dispatch moves bytes, so it is compared exactly. Combine's sum of k terms in
32 bits is within (k + 2) U of the terms' sizes, a dot product over d columns
within (d / 64 + 20) U of its (at most d / 64 + 8 additions per lane, 8 above).
"""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X

pytestmark = pytest.mark.gpu
U = F.U


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def choices(n, e, k, capacity, seed=0, masked=0):
    """experts, slots, counts as the router gives them."""
    x = torch.randn(n, e, generator=gen(seed), device="cuda")
    x[:, 0] += 1.5  # a popular expert runs over its capacity
    m = None
    if masked:
        m = (torch.arange(n, device="cuda") % masked != 0).to(torch.uint8)
    r = X.route(x, k, mask=m, capacity=capacity)
    return r[0], r[2], r[3], r[1]


def raw(t):
    return t.view(torch.uint8).cpu()


CASES = [(1, 1, 1, 1, 1), (1, 8, 2, 3, 16), (7, 4, 2, 3, 5), (50, 8, 3, 20, 64), (33, 24, 8, 9, 1),
         (65, 16, 4, 20, 1111), (20, 64, 16, 6, 200), (100, 3, 3, 101, 24), (40, 10, 5, 22, 4096),
         (9, 200, 2, 1, 2050)]


@pytest.mark.parametrize("n,e,k,cap,d", CASES)
def test_dispatch(n, e, k, cap, d):
    experts, slots, counts, _ = choices(n, e, k, cap, n, 3 if n > 30 else 0)
    for dtype in (torch.uint8, torch.int16, torch.bfloat16, torch.float32):
        for pad in (0, 3):
            x = torch.randint(0, 256, (n, (d + pad) * dtype.itemsize), generator=gen(d),
                              device="cuda").to(torch.uint8).view(dtype)[:, :d]
            out = torch.full((e * cap * d * dtype.itemsize,), 0xAB, dtype=torch.uint8,
                             device="cuda").view(dtype).view(e, cap, d)
            X.dispatch_tensors(x, experts, slots, counts, out)
            want = F.dispatch(x.contiguous().view(torch.uint8), experts, slots, e, cap)
            assert torch.equal(raw(out.view(e * cap, d)), want.view(e * cap, -1))


@pytest.mark.parametrize("d,g", [(1, 1), (64, 1), (300, 3), (512, 4), (1000, 8), (4096, 32)])
def test_dispatch_with_scales(d, g):
    n, e, k, cap = 45, 12, 3, 13
    experts, slots, counts, _ = choices(n, e, k, cap, d)
    x = torch.randn(n, d, generator=gen(1), device="cuda").to(torch.float8_e4m3fn)
    scale = torch.rand(n, g + 1, generator=gen(2), device="cuda")[:, :g]
    out = torch.empty(e, cap, d, dtype=torch.float8_e4m3fn, device="cuda")
    out_scale = torch.full((e, cap, g), -1.0, device="cuda")
    X.dispatch_tensors(x, experts, slots, counts, out, scale=scale, out_scale=out_scale)
    assert torch.equal(raw(out), F.dispatch(x.view(torch.uint8), experts, slots, e, cap))
    assert torch.equal(out_scale.cpu(), F.dispatch(scale, experts, slots, e, cap))


@pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)
@pytest.mark.parametrize("n,e,k,cap,d", CASES)
def test_combine(dtype, n, e, k, cap, d):
    experts, slots, _, w = choices(n, e, k, cap, n, 4 if n > 30 else 0)
    b = torch.randn(e, cap, d, generator=gen(d), device="cuda").to(dtype)
    for weights in (w, None):
        out = torch.full((n, d + 3), 5.0, dtype=dtype, device="cuda")
        X.combine_tensors(b, experts, slots, out[:, :d], weights=weights)
        want, size = F.combine(b, experts, slots, weights)
        F.close(out[:, :d], want, dtype, (k + 2) * U * size)
        assert (out[:, d:] == 5).all()


@pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)
@pytest.mark.parametrize("n,e,k,cap,d", CASES + [(1500, 6, 2, 400, 72)])
def test_combine_backward(dtype, n, e, k, cap, d):
    experts, slots, counts, w = choices(n, e, k, cap, n, 4 if n > 30 else 0)
    b = torch.randn(e, cap, d, generator=gen(d), device="cuda").to(dtype)
    dout = torch.randn(n, d + 1, generator=gen(2), device="cuda").to(dtype)[:, :d]
    db, dw = torch.full_like(b, 9), torch.full((n, k), 9.0, device="cuda")
    X.combine_backward_tensors(dout, b, experts, slots, counts, w, db, dw)
    want_db, want_dw, size = F.combine_backward(dout, b, experts, slots, w)
    F.close(db, want_db, dtype, U * want_db.abs())
    F.close(dw, want_dw, torch.float32, (d / 64 + 20) * U * size)


def test_choices_outside_the_buffer_are_none():
    """Experts and slots below zero or past the buffer have no row."""
    experts = torch.tensor([[0, -1, 5], [2, 1, 0], [2**31 - 1, -2**31, 1]], dtype=torch.int32,
                           device="cuda")
    slots = torch.tensor([[0, 0, 0], [-1, 4, 1], [0, 0, 2**31 - 1]], dtype=torch.int32,
                         device="cuda")
    counts = torch.tensor([2, -5, 2**31 - 1], dtype=torch.int32, device="cuda")
    x = torch.arange(1, 61, device="cuda", dtype=torch.float32).view(3, 20)
    out = torch.full((3, 4, 20), 7.0, device="cuda")
    X.dispatch_tensors(x, experts, slots, counts, out)
    assert torch.equal(out[0, 0], x[0]) and torch.equal(out[0, 1], x[1])
    assert (out[0, 2:] == 0).all() and (out[1] == 0).all() and (out[2] == 7).all()
    got = torch.empty(3, 20, device="cuda")
    X.combine_tensors(out, experts, slots, got)
    assert torch.equal(got[:2], x[:2]) and (got[2] == 0).all()


def test_offsets_past_32_bits():
    """Rows whose element offset passes 2^31 and byte offset 2^32."""
    e, cap, d = 4, (1 << 17) + 3, 4096
    experts = torch.tensor([[0, 3], [3, 2], [1, 3]], dtype=torch.int32, device="cuda")
    slots = torch.tensor([[1, cap - 1], [0, cap - 2], [5, 7]], dtype=torch.int32, device="cuda")
    counts = torch.full((e,), cap, dtype=torch.int32, device="cuda")
    x = torch.randn(3, d, generator=gen(1), device="cuda").bfloat16()
    out = torch.zeros(e, cap, d, dtype=torch.bfloat16, device="cuda")
    X.dispatch_tensors(x, experts, slots, counts, out)
    for t in range(3):
        for j in range(2):
            assert torch.equal(out[experts[t, j].item(), slots[t, j].item()], x[t])
    got = torch.empty_like(x)
    X.combine_tensors(out, experts, slots, got)
    assert torch.equal(got, 2 * x)
    w = torch.tensor([[1.0, 2.0], [0.5, 4.0], [1.0, -1.0]], device="cuda")
    dw = torch.empty(3, 2, device="cuda")
    db = torch.empty_like(out)
    X.combine_backward_tensors(x, out, experts, slots, counts, w, db, dw)
    assert torch.equal(db[3, cap - 1], 2 * x[0]) and torch.equal(db[2, cap - 2], 4 * x[1])
    counts[3] = 8
    db.fill_(1)
    experts[0, 1] = -1
    X.combine_backward_tensors(x, out, experts, slots, counts, w, db, dw)
    assert (db[3, 8:] == 0).all() and (db[3, 6] == 1).all() and torch.equal(db[3, 7], -x[2])


def test_no_tokens():
    counts = torch.zeros(3, dtype=torch.int32, device="cuda")
    none = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    out = torch.ones(3, 2, 10, device="cuda")
    X.dispatch_tensors(torch.empty(0, 10, device="cuda"), none, none, counts, out)
    assert (out == 0).all()
    X.combine_tensors(out, none, none, torch.empty(0, 10, device="cuda"))
    out.fill_(1)
    X.combine_backward_tensors(torch.empty(0, 10, device="cuda"), out, none, none, counts,
                               torch.empty(0, 2, device="cuda"), out.add(0), out[0, :0, :2])


def test_gradients_against_differences():
    """x -> dispatch -> b -> combine is linear in x and in the weights, so
    differences with any step are exact but for rounding (64-bit forms)."""
    n, e, k, cap, d = 13, 5, 2, 4, 30
    experts, slots, counts, w = choices(n, e, k, cap, 3)
    w = w.detach().requires_grad_()
    x = torch.randn(n, d, generator=gen(1), device="cuda").requires_grad_()
    c = torch.randn(n, d, generator=gen(2), device="cuda")
    f = torch.randn(e, 1, d, generator=gen(3), device="cuda")
    out = X.combine(X.dispatch(x, experts, slots, counts, cap) * f, experts, slots, counts, w)
    (out * c).sum().backward()

    def value(x, w):
        b = F.dispatch(x, experts, slots, e, cap) * f.cpu().double()
        return (F.combine(b, experts, slots, w)[0] * c.cpu().double()).sum()

    x0, w0 = x.detach().cpu().double(), w.detach().cpu().double()
    for _ in range(3):
        vx, vw = torch.randn(n, d, dtype=torch.float64), torch.randn(n, k, dtype=torch.float64)
        slope = value(x0 + vx, w0) - value(x0 - vx, w0) + value(x0, w0 + vw) - value(x0, w0 - vw)
        got = (x.grad.cpu().double() * vx).sum() + (w.grad.cpu().double() * vw).sum()
        length = x.grad.norm().item() * vx.norm() + w.grad.norm().item() * vw.norm()
        assert abs(slope / 2 - got) <= 1e-5 * length
