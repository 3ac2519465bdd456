"""The operators together: a layer against its plain form, the example, other
streams and captured graphs."""
import os
import sys

import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed),
                       device="cuda")


def plain_layer(x, r, norm_w, router, weights, k, capacity, coef):
    """The layer in 64 bits, token by token; differentiable."""
    h = x + r
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * norm_w
    logits = y @ router
    p = torch.softmax(logits, 1)
    top, experts = torch.topk(p, k, dim=1)
    w = top / top.sum(1, keepdim=True)
    e = router.shape[1]
    hot = torch.zeros_like(p).scatter_(1, experts, 1.0)
    place = (hot.cumsum(0) - hot).gather(1, experts)
    out = []
    for t in range(len(x)):
        rows = [w[t, j] * torch.nn.functional.silu(y[t] @ weights[experts[t, j]])
                for j in range(k) if place[t, j] < capacity]
        out.append(sum(rows, torch.zeros_like(y[t])))
    n = len(x)
    loss = coef * e * ((hot.sum(0) / (n * k)).detach() * p.mean(0)).sum()
    return torch.stack(out), h, loss


def test_layer_and_its_gradients():
    """32-bit operators against the 64-bit layer. Every step's relative error is
    below 1e-6 and no value is the difference of much larger ones, so 1e-4 of a
    tensor's length bounds each; the choices agree since no two logits of a
    token are near enough to change places."""
    n, d, e, k, capacity, coef = 48, 40, 6, 2, 14, 0.5
    names = ("x", "r", "norm", "router", "experts")
    init = (randn(1, n, d), randn(2, n, d), 1 + 0.1 * randn(3, d), randn(4, d, e) / d ** 0.5,
            randn(5, e, d, d) / d ** 0.5)
    c, c2 = randn(6, n, d), randn(7, n, d)
    got = {m: t.clone().requires_grad_() for m, t in zip(names, init)}
    y, total, _, _ = X.norm(got["x"], got["norm"], got["r"])
    logits = y @ got["router"]
    experts, weights, slots, counts, _, loss, _ = X.route(logits, k, capacity=capacity, coef=coef)
    assert int((slots < 0).sum()) > 0  # some choices are past the capacity
    b = X.dispatch(y, experts, slots, counts, capacity)
    b = torch.stack([torch.nn.functional.silu(r @ w) for r, w in zip(b, got["experts"])])
    out = X.combine(b, experts, slots, counts, weights)
    ((out * c).sum() + (total * c2).sum() + 3 * loss.sum()).backward()

    want = {m: t.cpu().double().requires_grad_() for m, t in zip(names, init)}
    ref, h, ref_loss = plain_layer(*want.values(), k, capacity, coef)
    ((ref * c.cpu().double()).sum() + (h * c2.cpu().double()).sum() + 3 * ref_loss).backward()
    pairs = [(out, ref), (total, h), (loss, ref_loss.view(1))]
    pairs += [(got[m].grad, want[m].grad) for m in names]
    for g, w in pairs:
        assert (g.detach().cpu().double() - w.detach()).norm() <= 1e-4 * w.detach().norm()


def test_example():
    import expert_alltoall

    lines = []
    got = expert_alltoall.main(tokens=256, dim=256, num_experts=32, k=2, steps=20, candidates=64,
                               say=lines.append)
    assert len(lines) == 4
    t = got["times"]
    assert t["8-bit rows"] < t["16-bit rows"] and t["evened"] < t["8-bit rows"]
    # e4m3 has 4 significant bits: rows are within 2^-4 of themselves
    assert 0 < got["off"] < 2.0 ** -4
    first, last = got["dropped"]
    assert last < first


def step_buffers(n, d, e, k, cap):
    f = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    i = torch.int32
    return dict(out=f(n, d), total=f(n, d), q=f(n, d, t=torch.float8_e4m3fn),
                scale=f(n, -(-d // 64)), experts=f(n, k, t=i), weights=f(n, k), slots=f(n, k, t=i),
                counts=f(e, t=i), prob_sums=f(e), loss=f(1), rows=f(1, t=i), buffer=f(e, cap, d),
                back=f(n, d), db=f(e, cap, d), dw=f(n, k), dl=f(n, e), dx=f(n, d), dnorm=f(d),
                work=f(max(X.route_workspace(e), X.norm_workspace(d)), t=torch.uint8))


def step(x, r, w, logits, o, stream=None):
    """One pass through every operator, on the caller's buffers."""
    X.norm_tensors(x, w, o["out"], residual=r, total=o["total"], q=o["q"], scale=o["scale"],
                   group=64, stream=stream)
    X.route_tensors(logits, o["experts"], o["weights"], o["slots"], o["counts"], o["prob_sums"],
                    o["loss"], o["rows"], o["work"], capacity=o["buffer"].shape[1], stream=stream)
    X.dispatch_tensors(o["out"], o["experts"], o["slots"], o["counts"], o["buffer"], stream=stream)
    X.combine_tensors(o["buffer"], o["experts"], o["slots"], o["back"], weights=o["weights"],
                      stream=stream)
    X.combine_backward_tensors(o["back"], o["buffer"], o["experts"], o["slots"], o["counts"],
                               o["weights"], o["db"], o["dw"], stream=stream)
    X.route_backward_tensors(logits, o["experts"], o["counts"], o["rows"], o["dl"],
                             dweights=o["dw"], dloss=o["loss"], stream=stream)
    X.norm_backward_tensors(o["back"], o["total"], w, o["dx"], o["dnorm"], o["work"],
                            stream=stream)


SHAPE = dict(n=700, d=320, e=24, k=4, cap=120)


def inputs(seed):
    n, d, e = SHAPE["n"], SHAPE["d"], SHAPE["e"]
    return randn(seed, n, d), randn(seed + 1, n, d), randn(seed + 2, d), 2 * randn(seed + 3, n, e)


def bits(o):
    return {m: t.view(torch.uint8).clone() for m, t in o.items() if m != "work"}


def test_graph_replays():
    """A captured step, replayed with new inputs in place and eager work and
    synchronizations between the replays, gives the eager step's bits."""
    held, o = inputs(0), step_buffers(**SHAPE)
    step(*held, o)  # the library is loaded and warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*held, o)
    eager = step_buffers(**SHAPE)
    for seed in (10, 20, 30, 40):
        new = inputs(seed)
        for a, b in zip(held, new):
            a.copy_(b)
        for t in o.values():
            t.view(torch.uint8).fill_(7)
        graph.replay()
        if seed != 20:
            torch.cuda.synchronize()
        got = bits(o)
        step(*new, eager)
        want = bits(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(got[m], want[m]) for m in want)


def test_other_streams():
    """Two streams at once, the current one and a given one."""
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    ins = [inputs(50), inputs(60)]
    want = []
    for x in ins:
        o = step_buffers(**SHAPE)
        step(*x, o)
        want.append(bits(o))
    torch.cuda.synchronize()
    for _ in range(3):
        outs = [step_buffers(**SHAPE) for _ in ins]
        a.wait_stream(torch.cuda.current_stream())
        b.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(a):
            step(*ins[0], outs[0])
        step(*ins[1], outs[1], stream=b)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            got = bits(o)
            assert all(torch.equal(got[m], w[m]) for m in w)


def test_refusals_on_the_device():
    x, w = randn(1, 4, 8), randn(2, 8)
    out = torch.empty_like(x)
    with pytest.raises(ValueError, match="weight"):
        X.norm_tensors(x, w[:7], out)
    with pytest.raises(ValueError, match="out"):
        X.norm_tensors(x, w, out.bfloat16())
    with pytest.raises(ValueError, match="contiguous rows"):
        X.norm_tensors(x, w, torch.empty(8, 4, device="cuda").t())
    with pytest.raises(ValueError, match="scale"):
        X.norm_tensors(x, w, out, q=out.to(torch.float8_e4m3fn), scale=out[:, :3], group=32)
    with pytest.raises(X.binding.TacclError, match="group"):
        X.norm_tensors(x, w, out, group=48)
    with pytest.raises(X.binding.TacclError, match="stride"):
        X.norm_tensors(x[:1].expand(4, 8), w, out)
    i = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="counts"):
        X.dispatch_tensors(x, i, i, i[0, :1], torch.empty(2, 3, 8, device="cuda"))
    with pytest.raises(ValueError, match="slots"):
        X.combine_tensors(torch.empty(2, 3, 8, device="cuda"), i, i[:3], out)
    with pytest.raises(ValueError, match="buffer"):
        X.combine_tensors(torch.empty(2, 3, 8, device="cuda", dtype=torch.float64), i, i, out)
    with pytest.raises(ValueError, match="workspace"):
        X.norm_backward_tensors(x, x, w, out, w.clone(), torch.empty(9, dtype=torch.uint8))
    with pytest.raises(X.binding.TacclError, match="workspace too small"):
        X.norm_backward_tensors(x, x, w, out, w.clone(),
                                torch.empty(9, dtype=torch.uint8, device="cuda"))
