"""Router kernels at the widths and batches of their launch shapes, against a
64-bit form over whole tensors: one block and several, one tile and several per
block, 16, 32 and 64 lanes per token, choices ranked and one at a time.

Bounds as in test_gpu_route.py.
"""
import pytest
import torch

import expert_forms as F
from test_gpu_route import gen, logits_of, run

pytestmark = pytest.mark.gpu
U = F.U

SHAPES = [(9000, 256, 8), (9000, 600, 5), (700, 1024, 8), (400, 513, 3), (9000, 64, 12),
          (700, 300, 12), (9000, 1024, 16), (20000, 128, 6), (129, 256, 8), (8193, 32, 9),
          (50000, 16, 4)]


def wanted(x, k, mask, capacity, coef, renorm):
    x = x.cpu().double()
    n, e = x.shape
    live = torch.ones(n, dtype=torch.bool) if mask is None else mask.cpu() != 0
    p = torch.softmax(x, 1) * live[:, None]
    order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
    hot = torch.zeros(n, e, dtype=torch.int32).scatter_(1, order, 1) * live[:, None].int()
    place = (hot.cumsum(0, dtype=torch.int32) - hot).gather(1, order)
    taken = live[:, None] & (place < capacity if capacity else place >= 0)
    w = torch.softmax(x.gather(1, order), 1) if renorm else p.gather(1, order)
    rows, counts = int(live.sum()), hot.sum(0).int()
    loss = coef * e * (counts.double() / (rows * k) * p.sum(0) / rows).sum()
    return {"experts": torch.where(live[:, None], order, -1).int(),
            "slots": torch.where(taken, place, -1).int(), "weights": w * live[:, None],
            "counts": counts, "prob_sums": p.sum(0), "loss": loss.view(1), "rows": rows, "p": p}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,e,k", SHAPES)
def test_forward(n, e, k, dtype):
    for i, masked in enumerate((0, 5)):
        x = logits_of(n, e, dtype, n + e + i, 3 * i)
        mask = None
        if masked:
            mask = (torch.arange(n, device="cuda") % masked != 2).to(torch.uint8)
        cap, renorm = n * k // e + 1, i == 0
        got = run(x, k, mask=mask, capacity=cap, renorm=renorm)
        want = wanted(x, k, mask, cap, 0.01, renorm)
        for name in ("experts", "slots", "counts"):
            assert torch.equal(got[name].cpu(), want[name]), name
        assert int(got["rows"]) == want["rows"]
        near = (8 * F.logit_range(x, mask) + 40) * U
        chain = near + (100 + n / 256) * U
        F.close(got["weights"], want["weights"], torch.float32, near * want["weights"])
        F.close(got["prob_sums"], want["prob_sums"], torch.float32, chain * want["prob_sums"])
        F.close(got["loss"], want["loss"], torch.float32, 2 * chain * want["loss"].abs())


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("n,e,k", [(9000, 600, 5), (9000, 1024, 16), (20000, 300, 8),
                                   (40000, 16, 4), (33000, 256, 8)])
def test_backward(n, e, k, renorm):
    """Several tokens per group of lanes."""
    from paper_2111_04867_amd import experts as X

    coef = 0.3
    x = logits_of(n, e, torch.float32, n + e)
    mask = (torch.arange(n, device="cuda") % 5 != 2).to(torch.uint8)
    r = run(x, k, mask=mask, coef=coef, renorm=renorm)
    dw = torch.randn(n, k, generator=gen(9), device="cuda")
    out = torch.full((n, e), 3.0, device="cuda")
    X.route_backward_tensors(x, r["experts"], r["counts"], r["rows"], out, dweights=dw,
                             dloss=torch.full((1,), -2.0, device="cuda"), mask=mask, coef=coef,
                             renorm=renorm)
    want = wanted(x, k, mask, 0, coef, renorm)
    p, live = want["p"], mask.cpu() != 0
    g = (-2.0 * coef * e * want["counts"].double() / (want["rows"] ** 2 * k)).expand_as(p).clone()
    at = want["experts"].clamp_min(0).long()
    d = dw.cpu().double() * live[:, None]
    w = want["weights"]
    direct, size = torch.zeros_like(p), torch.zeros_like(p)
    if renorm:
        direct.scatter_add_(1, at, w * (d - (w * d).sum(1, keepdim=True)))
        size.scatter_add_(1, at, w * (d.abs() + (w * d).abs().sum(1, keepdim=True)))
    else:
        g.scatter_add_(1, at, d)
    dl = p * (g - (p * g).sum(1, keepdim=True)) + direct
    size += p * (g.abs() + (p * g).abs().sum(1, keepdim=True))
    F.close(out, dl, torch.float32, (8 * F.logit_range(x, mask) + 80) * U * size)
