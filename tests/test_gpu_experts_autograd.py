"""What autograd may and may not do with the differentiable operators."""
import pytest
import torch

from paper_2111_04867_amd import experts as X

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed),
                       device="cuda")


def routed():
    return X.route(randn(1, 20, 6), 2, capacity=9)


@pytest.mark.parametrize("op", ["norm", "route", "dispatch", "combine", "combine_weights"])
def test_second_derivatives_are_refused(op):
    """A gradient penalty that also reaches its input another way has a second
    derivative without the operator's part; it raises."""
    experts, weights, slots, counts = (routed()[i] for i in (0, 1, 2, 3))
    x = randn(2, 9 * 6 if op == "combine" else 20, 8)
    if op == "route":
        x = randn(1, 20, 6)
    if op == "combine_weights":
        x = weights
    x = x.detach().requires_grad_()
    if op == "norm":
        out = X.norm(x, torch.ones(8, device="cuda"))[0]
    elif op == "route":
        out = X.route(x, 2)[1]
    elif op == "dispatch":
        out = X.dispatch(x, experts, slots, counts, 9)
    elif op == "combine":
        out = X.combine(x.view(6, 9, 8), experts, slots, counts, weights)
    else:
        out = X.combine(randn(3, 6, 9, 8), experts, slots, counts, x)
    g, = torch.autograd.grad((out ** 3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="twice|once_differentiable"):
        (g * x).sum().backward()


def test_mask_written_between_the_passes():
    """The gradient needs the forward pass's mask: a changed one raises."""
    x = randn(1, 30, 8).requires_grad_()
    mask = torch.ones(30, dtype=torch.uint8, device="cuda")
    mask[::3] = 0
    loss = X.route(x, 2, mask=mask)[5]
    mask.fill_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


@pytest.mark.parametrize("renorm", [True, False])
def test_boolean_mask(renorm):
    """The same as its bytes, in both passes."""
    got = []
    for dtype in (torch.uint8, torch.bool):
        x = randn(1, 300, 12).requires_grad_()
        mask = (torch.arange(300, device="cuda") % 4 != 1).to(dtype)
        out = X.route(x, 3, mask=mask, capacity=50, renorm=renorm)
        ((out[1] * randn(2, 300, 3)).sum() + out[5].sum()).backward()
        got.append([*out, x.grad])
    for a, b in zip(*got):
        assert torch.equal(a, b)
    with pytest.raises(ValueError, match="mask"):
        X.route(x, 3, mask=mask.float())
    with pytest.raises(ValueError, match="mask"):
        X.route(x, 3, mask=torch.ones(600, dtype=torch.bool, device="cuda")[::2])


def test_combine_without_weights():
    """Weights of 1, and their gradient left out."""
    experts, weights, slots, counts = (routed()[i] for i in (0, 1, 2, 3))
    got = []
    for w in (None, torch.ones_like(weights)):
        buffer = randn(3, 6, 9, 8).requires_grad_()
        out = X.combine(buffer, experts, slots, counts, w)
        (out * randn(4, 20, 8)).sum().backward()
        got.append((out, buffer.grad))
    assert torch.equal(got[0][0], got[1][0])
    used = torch.arange(9, device="cuda") < counts[:, None]
    assert int((~used).sum()) > 0 and (got[0][1][~used] == 0).all()
    assert torch.equal(got[0][1], got[1][1])


def test_sizes_past_32_bits():
    """Columns, experts and choices whose low 32 bits alone would pass are
    refused, not cut. No array holds anything but the weight (8.6 GB, not
    touched): there are no rows."""
    d = (1 << 32) + 64
    x = torch.empty(0, d, dtype=torch.float16, device="cuda")
    w = torch.empty(d, dtype=torch.float16, device="cuda")
    with pytest.raises(X.binding.TacclError, match="more than 16384 columns"):
        X.norm_tensors(x, w, x)
    del w
    none = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(X.binding.TacclError, match="more than 1024 experts"):
        X.combine_tensors(torch.empty((1 << 32) + 4, 0, 8, device="cuda"), none, none,
                          torch.empty(0, 8, device="cuda"))
    many = torch.empty(0, (1 << 32) + 2, dtype=torch.int32, device="cuda")
    with pytest.raises((ValueError, X.binding.TacclError), match="choices"):
        X.route_backward_tensors(torch.empty(0, 8, device="cuda"), many, *(
            torch.zeros(s, dtype=torch.int32, device="cuda") for s in (8, 1)),
            torch.empty(0, 8, device="cuda"))
