"""The experts' operators under autograd, on streams and in graphs, and together."""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed),
                       device="cuda")


def layer(dtype, e=4, c=12, d=24, f=16, sources=None):
    shape = (e, c) if sources is None else (sources, e, c)
    counts = torch.arange(len(range(shape[0] * (1 if sources is None else e))), device="cuda") * 3
    return (randn(1, *shape, d).to(dtype), counts.view(shape[:-1]).int(),
            (randn(2, e, 2 * f, d) / d ** 0.5).to(dtype), (randn(3, e, d, f) / f ** 0.5).to(dtype))


def plain(buffer, counts, w_in, w_out):
    """In 64 bits, by autograd itself."""
    f = w_out.shape[2]
    x = buffer if buffer.dim() == 4 else buffer[None]
    h = torch.stack([torch.stack([x[s, e] @ w_in[e].t() for e in range(x.shape[1])])
                     for s in range(x.shape[0])])
    a = h[..., :f] * torch.sigmoid(h[..., :f]) * h[..., f:]
    y = torch.stack([torch.stack([a[s, e] @ w_out[e].t() for e in range(x.shape[1])])
                     for s in range(x.shape[0])])
    there = torch.arange(x.shape[2], device=x.device) < counts.view(x.shape[:2])[..., None]
    return (y * there[..., None]).view(buffer.shape)


@pytest.mark.parametrize("sources", [None, 3])
def test_gradients_are_the_formulas(sources):
    """In 32 bits, against autograd's of the plain form in 64: the sums have at
    most 36 rows and 32 columns of numbers of a size about 1, so 1e-5 is ten
    times their rounding."""
    buffer, counts, w_in, w_out = layer(torch.float32, sources=sources)
    dout = randn(4, *buffer.shape)
    got = [t.clone().requires_grad_() for t in (buffer, w_in, w_out)]
    out = X.ffn(got[0], counts, got[1], got[2])
    out.backward(dout)
    ref = [t.double().requires_grad_() for t in (buffer, w_in, w_out)]
    want = plain(ref[0], counts, ref[1], ref[2])
    want.backward(dout.double())
    assert (out - want).abs().max() < 1e-5
    for a, b in zip(got, ref):
        assert (a.grad - b.grad).abs().max() < 1e-5 * max(1, b.grad.abs().max().item())


def test_gradients_are_differences():
    """Along random directions, of the plain form in 64 bits: a step of 2^-12
    moves g and u by about 5 such steps, so a central difference is off by a few
    times (5 * 2^-12)^2 = 1.5e-6 of the terms' sizes, the gradient by 32 bits'
    rounding of sums of up to 36 terms, 2e-6 of them."""
    buffer, counts, w_in, w_out = layer(torch.float32)
    dout = randn(4, *buffer.shape)
    leaves = [t.clone().requires_grad_() for t in (buffer, w_in, w_out)]
    (X.ffn(leaves[0], counts, leaves[1], leaves[2]) * dout).sum().backward()
    h = 2.0 ** -12
    for i, t in enumerate((buffer, w_in, w_out)):
        v = randn(5 + i, *t.shape).double()
        ends = []
        for sign in (1, -1):
            args = [buffer.double(), w_in.double(), w_out.double()]
            args[i] = args[i] + sign * h * v
            ends.append((plain(args[0], counts, args[1], args[2]) * dout).sum())
        terms = leaves[i].grad.double() * v
        assert ((ends[0] - ends[1]) / (2 * h) - terms.sum()).abs() <= 2e-5 * terms.abs().sum()


def test_only_what_is_asked_for():
    buffer, counts, w_in, w_out = layer(torch.bfloat16)
    whole = [t.clone().requires_grad_() for t in (buffer, w_in, w_out)]
    X.ffn(whole[0], counts, whole[1], whole[2]).float().sum().backward()
    for i in range(3):
        t = [buffer.clone(), w_in.clone(), w_out.clone()]
        t[i].requires_grad_()
        X.ffn(t[0], counts, t[1], t[2]).float().sum().backward()  # an expanded gradient
        assert torch.equal(t[i].grad, whole[i].grad)
    with torch.no_grad():
        assert not X.ffn(whole[0], counts, whole[1], whole[2]).requires_grad


@pytest.mark.parametrize("op", ["ffn", "dropout"])
def test_second_derivatives_are_refused(op):
    buffer, counts, w_in, w_out = layer(torch.float32)
    x = buffer.requires_grad_() if op == "ffn" else randn(1, 6, 8).requires_grad_()
    if op == "ffn":
        out = X.ffn(x, counts, w_in, w_out)
    else:
        out = X.dropout(x, 0.5, torch.tensor([1, 2], device="cuda"))
    g, = torch.autograd.grad((out ** 3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="twice|once_differentiable"):
        (g * x).sum().backward()


def test_ffn_tokens_has_no_gradient():
    _, _, w_in, w_out = layer(torch.float32)
    x = randn(1, 5, 24).requires_grad_()
    out, _, weights = X.ffn_tokens(x, randn(2, 5, 4), 2, w_in, w_out)
    with pytest.raises(RuntimeError, match="no gradient"):
        out.sum().backward()
    with torch.no_grad():
        assert torch.equal(X.ffn_tokens(x, randn(2, 5, 4), 2, w_in, w_out)[0], out)


@pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)
def test_dropout_gradients(dtype):
    x, r = (randn(i, 40, 70).to(dtype).requires_grad_() for i in (1, 2))
    rng = torch.tensor([7, 1000], device="cuda")
    dout = randn(3, 40, 70).to(dtype)
    X.dropout(x, 0.3, rng, r).backward(dout)
    want, slack = F.dropout(dout, rng.cpu(), 0.3)
    F.close(x.grad, want, dtype, slack)
    assert torch.equal(r.grad, dout)
    X.dropout(x.detach(), 0.3, rng, r).backward(dout)
    assert torch.equal(r.grad, 2 * dout)
    x.grad = None
    X.dropout(x, 0.3, rng).sum().backward()  # an expanded gradient
    assert torch.equal(x.grad != 0, F.kept(rng.cpu(), 40, 70, 0.3).cuda())


def test_stepped_numbers():
    """A generator stepped between the passes is refused; calls on states a
    call's words apart do not share a number."""
    x = randn(1, 64, 33).requires_grad_()
    rng = torch.tensor([7, 0], device="cuda")
    out = X.dropout(x, 0.5, rng)
    rng[1] += X.dropout_words(64, 33)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    ones = torch.ones(128, 33, device="cuda")
    start = torch.tensor([7, 0], device="cuda")
    whole = X.dropout(ones, 0.5, start)
    assert torch.equal(whole[64:], X.dropout(ones[:64], 0.5, rng))


def test_on_another_stream():
    buffer, counts, w_in, w_out = layer(torch.bfloat16, e=3, c=40, d=64, f=40)
    want = X.ffn(buffer, counts, w_in, w_out)
    x, logits = randn(5, 9, 64).bfloat16(), randn(6, 9, 3)
    want_tokens = X.ffn_tokens(x, logits, 2, w_in, w_out)
    rng = torch.tensor([1, 2], device="cuda")
    want_drop = X.dropout(x, 0.2, rng)
    side = torch.cuda.Stream()
    out, work = torch.empty_like(buffer), torch.empty(
        X.ffn_workspace(buffer.shape, 40, buffer.dtype), dtype=torch.uint8, device="cuda")
    tokens, twork = torch.empty_like(x), torch.empty(
        X.ffn_tokens_workspace(9, 2, 64, 40), dtype=torch.uint8, device="cuda")
    drop = torch.empty_like(x)
    torch.cuda.synchronize()
    X.ffn_tensors(buffer, counts, w_in, w_out, out, work, stream=side)
    X.ffn_tokens_tensors(x, logits, w_in, w_out, tokens, twork, k=2, stream=side)
    X.dropout_tensors(x, rng, drop, p=0.2, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(tokens, want_tokens[0])
    assert torch.equal(drop, want_drop)


@pytest.mark.parametrize("sizes", [(1, 4, 30, 64, 40), (3, 2, 13, 4101, 33), (8, 1, 400, 40, 24)],
                         ids=str)
def test_in_graphs(sizes):
    """Replays with other inputs, counts and random numbers, between eager
    calls, give the eager results' bits."""
    s, e, c, d, f = sizes
    dtype = torch.float16
    w_in, w_out = (randn(1, e, 2 * f, d) / d ** 0.5).to(dtype), (randn(2, e, d, f) / 5).to(dtype)
    buffer, dout = randn(3, s, e, c, d).to(dtype), randn(4, s, e, c, d).to(dtype)
    counts = torch.randint(0, c + 1, (s, e), device="cuda").int()
    x, logits = randn(5, 20, d).to(dtype), randn(6, 20, e)
    rng = torch.tensor([1, 0], device="cuda")
    k = min(2, e)

    def calls():
        pre = torch.zeros(s, e, c, 2 * f, dtype=dtype, device="cuda")
        out = torch.empty_like(buffer)
        work = torch.empty(X.ffn_workspace(buffer.shape, f, dtype, True), dtype=torch.uint8,
                           device="cuda")
        X.ffn_tensors(buffer, counts, w_in, w_out, out, work, pre=pre)
        grads = [torch.empty_like(t) for t in (buffer, w_in, w_out)]
        X.ffn_backward_tensors(dout, buffer, counts, w_in, w_out, pre, work, dbuffer=grads[0],
                               dw_in=grads[1], dw_out=grads[2])
        tokens = X.ffn_tokens(x, logits, k, w_in, w_out)
        return [out, pre, *grads, *tokens, X.dropout(x, 0.4, rng, x)]

    with torch.no_grad():
        calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = calls()
        for i in range(4):
            buffer.copy_(randn(10 + i, s, e, c, d))
            logits.copy_(randn(20 + i, 20, e))
            counts.copy_(torch.randint(0, c + 3, (s, e), device="cuda"))
            rng[1] += X.dropout_words(20, d)
            want = calls()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(held, want):
                assert torch.equal(a, b)


def test_a_captured_gradient():
    """Forward and gradient in one graph: replays draw new random numbers and
    give the eager results' bits. Every pass has leaves of its own."""
    values = layer(torch.bfloat16, e=3, c=40, d=72, f=40)
    counts, rng = values[1], torch.tensor([5, 0], device="cuda")
    dout = randn(7, 3 * 40, 72).bfloat16()

    def step(leaves):
        out = X.ffn(leaves[0], counts, *leaves[1:]).view(3 * 40, 72)
        out = X.dropout(out, 0.3, rng, leaves[0].view(3 * 40, 72))
        return [out.detach(), *torch.autograd.grad(out, leaves, dout)]

    def leaves():
        return [values[i].clone().requires_grad_() for i in (0, 2, 3)]

    own = leaves()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(leaves())
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(own)
    last = None
    for i in range(4):
        rng[1] += X.dropout_words(120, 72)
        want = step(leaves())
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
        assert last is None or not torch.equal(last, held[0])
        last = held[0].clone()


@pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)
def test_the_layer_in_parts_and_whole(dtype):
    """norm, route, dispatch, ffn, combine and dropout as a layer runs them; the
    few tokens' form gives the same rows. a's rounding to 16 bits and combine's
    rows' are the parts' alone: each within half a step of numbers whose
    products with weights of a size 1 add up to the row's own size or less, so
    three times four half steps of the largest value cover both."""
    t, e, k, d, f = 48, 8, 3, 64, 40
    x, weight = randn(1, t, d).to(dtype), torch.ones(d, dtype=dtype, device="cuda")
    router = randn(2, d, e) / d ** 0.5
    w_in, w_out = (randn(3, e, 2 * f, d) / d ** 0.5).to(dtype), (randn(4, e, d, f) / f ** 0.5).to(dtype)
    rng = torch.tensor([3, 4], device="cuda")
    leaves = [p.requires_grad_() for p in (x, router, w_in, w_out)]
    y, total, _, _ = X.norm(x, weight, x.detach())
    logits = y.float() @ router
    experts, weights, slots, counts, _, loss, _ = X.route(logits, k, capacity=t)
    sent = X.dispatch(y, experts, slots, counts, t)
    rows = X.combine(X.ffn(sent, counts, w_in, w_out), experts, slots, counts, weights)
    out = X.dropout(rows, 0.25, rng, total)
    (out.float().square().mean() + loss.sum()).backward()
    for p in leaves:
        assert p.grad.isfinite().all() and p.grad.abs().max() > 0
    with torch.no_grad():
        got, chosen, w = X.ffn_tokens(y, logits, k, w_in, w_out)
    assert torch.equal(chosen, experts)
    assert torch.allclose(w, weights, rtol=1e-5, atol=1e-8)
    step = F.ROUND[dtype][0] if dtype != torch.float32 else 64 * F.U
    assert (got.float() - rows.float()).abs().max() <= 12 * step * rows.float().abs().max()


def test_rows_from_several_ranks():
    """What an Alltoall brings, through the rank's experts as it lies, is each
    source's rows through them."""
    sources, e, c, d, f = 3, 2, 10, 40, 24
    buffer, counts, w_in, w_out = layer(torch.bfloat16, e, c, d, f, sources)
    got = X.ffn(buffer, counts, w_in, w_out)
    for s in range(sources):
        assert torch.equal(got[s], X.ffn(buffer[s].contiguous(), counts[s].contiguous(), w_in, w_out))
