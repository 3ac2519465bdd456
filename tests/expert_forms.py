"""Plain 64-bit forms of the expert-layer operators on the CPU, and the error
that 32-bit arithmetic with one final rounding may have (U: unit roundoff)."""
import torch

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# unit roundoff of the stored type and half its smallest step
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134),
         torch.float16: (2.0 ** -11, 2.0 ** -25)}
AMAX_MIN = 2.0 ** -100


def close(got, want, dtype, slack):
    """|got - want| within the stored type's rounding of `want` plus `slack`
    (the arithmetic's error, elementwise); the same NaNs and infinities."""
    g, w = got.detach().cpu().double(), want.double()
    assert g.shape == w.shape, (g.shape, w.shape)
    assert torch.equal(g.isnan(), w.isnan())
    big = torch.finfo(dtype).max
    fine = w.isfinite() & (w.abs() < big)
    rel, step = ROUND[dtype]
    slack = torch.as_tensor(slack, dtype=torch.float64).expand_as(w)
    off = (g - w).abs() - (rel * (1 + rel) * w.abs() + step + (1 + rel) * slack)
    worst = off[fine].max().item() if fine.any() else 0.0
    assert worst <= 0, f"off by {worst} more than allowed"
    inf = w.isinf()
    assert torch.equal(g[inf], w[inf])


# ---- norm -----------------------------------------------------------------------

def norm(x, weight, residual, eps):
    h = x.cpu().double()
    if residual is not None:
        h = h + residual.cpu().double()
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, h * r * weight.cpu().double()


def scales(y, group):
    n, d = y.shape
    group = group or d
    out = torch.empty(n, -(-d // group), dtype=torch.float64)
    for i in range(out.shape[1]):
        out[:, i] = y[:, i * group:(i + 1) * group].abs().amax(1).clamp_min(AMAX_MIN) / 448
    return out


def norm_backward(dout, h, weight, eps, dtotal):
    """(dx, dweight) and the sums of the terms' sizes."""
    h, dy, w = h.cpu().double(), dout.cpu().double(), weight.cpu().double()
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    a = dy * w
    t = torch.zeros_like(h) if dtotal is None else dtotal.cpu().double()
    dx = t + r * a - h * r ** 3 * (a * h).mean(1, keepdim=True)
    size = t.abs() + r * a.abs() + h.abs() * r ** 3 * (a * h).abs().mean(1, keepdim=True)
    return dx, (dy * h * r).sum(0), size, (dy * h * r).abs().sum(0)


# ---- route ----------------------------------------------------------------------

def probabilities(logits, mask):
    """(p, live): zero rows for masked tokens and rows of minus infinities."""
    x = logits.cpu().double()
    if mask is not None:
        x = torch.where(mask.cpu()[:, None] != 0, x, -torch.inf)
    top = torch.where(x.isnan(), -torch.inf, x).amax(1, keepdim=True)
    e = torch.exp(x - torch.where(top == -torch.inf, 0.0, top))
    s = e.sum(1, keepdim=True)
    live = s != 0
    return torch.where(live, e / torch.where(live, s, 1.0), 0.0), live[:, 0]


def route(logits, k, mask=None, capacity=0, coef=0.01, renorm=True):
    """Lists in token order, one token at a time."""
    n, e = logits.shape
    p, live = probabilities(logits, mask)
    x = logits.cpu().double().tolist()
    experts = torch.full((n, k), -1, dtype=torch.int32)
    slots = experts.clone()
    weights = torch.zeros(n, k, dtype=torch.float64)
    counts = [0] * e
    for t in range(n):
        if mask is not None and not mask[t]:
            continue
        order = sorted((i for i in range(e) if x[t][i] == x[t][i] and x[t][i] > -torch.inf),
                       key=lambda i: (-x[t][i], i))[:k]
        for j, i in enumerate(order):
            experts[t, j] = i
            slots[t, j] = counts[i] if not capacity or counts[i] < capacity else -1
            counts[i] += 1
            weights[t, j] = p[t, i]
        if renorm and order:
            top = torch.tensor([x[t][i] for i in order], dtype=torch.float64)
            weights[t, :len(order)] = torch.softmax(top, 0)
    sums, rows = p.sum(0), int(live.sum())
    loss = 0.0
    if rows:
        load = torch.tensor(counts, dtype=torch.float64)
        loss = (coef * e * (load / (rows * k) * sums / rows).sum()).item()
    return {"experts": experts, "slots": slots, "weights": weights,
            "counts": torch.tensor(counts, dtype=torch.int32), "prob_sums": sums, "loss": loss,
            "rows": rows}


def logit_range(logits, mask=None):
    x = logits.cpu().double()
    if mask is not None:
        x = x[mask.cpu() != 0]
    x = torch.where(x.isfinite(), x, torch.nan)
    if not x.numel():
        return 0.0
    spread = (x.nan_to_num(-torch.inf).amax(1) - x.nan_to_num(torch.inf).amin(1))
    spread = spread[spread.isfinite()]
    return min(spread.max().item(), 90.0) if spread.numel() else 0.0


def route_backward(logits, experts, counts, rows, k, dweights, dloss, mask, coef, renorm):
    """(dlogits, the sum of the terms' sizes)."""
    n, e = logits.shape
    p, live = probabilities(logits, mask)
    g = torch.zeros(n, e, dtype=torch.float64)
    if dloss is not None and rows:
        g += dloss * coef * e * counts.cpu().double() / (rows ** 2 * k)
    direct, size = torch.zeros(n, e, dtype=torch.float64), torch.zeros(n, e, dtype=torch.float64)
    if dweights is not None:
        for t in range(n):
            at = [int(i) for i in experts[t] if i >= 0]
            if not live[t] or not at:
                continue
            dw = dweights[t, :len(at)].cpu().double()
            if renorm:
                w = p[t, at] / p[t, at].sum()
                direct[t, at] = w * (dw - (w * dw).sum())
                size[t, at] = w * (dw.abs() + (w * dw).abs().sum())
            else:
                g[t, at] += dw
    dl = p * (g - (p * g).sum(1, keepdim=True)) + direct
    return dl, size + p * (g.abs() + (p * g).abs().sum(1, keepdim=True))


# ---- dispatch and combine ---------------------------------------------------------

def places(experts, slots, num_experts, capacity):
    """(t, j, expert, slot) of every choice that has a buffer row."""
    for t, (es, ss) in enumerate(zip(experts.tolist(), slots.tolist())):
        for j, (e, s) in enumerate(zip(es, ss)):
            if 0 <= e < num_experts and 0 <= s < capacity:
                yield t, j, e, s


def dispatch(x, experts, slots, num_experts, capacity):
    x = x.cpu()
    out = torch.zeros(num_experts, capacity, x.shape[1], dtype=x.dtype)
    for t, _, e, s in places(experts, slots, num_experts, capacity):
        out[e, s] = x[t]
    return out


def combine(buffer, experts, slots, weights):
    """(out, sum of the terms' sizes)."""
    b = buffer.cpu().double()
    out = torch.zeros(len(experts), b.shape[2], dtype=torch.float64)
    size = out.clone()
    for t, j, e, s in places(experts, slots, *b.shape[:2]):
        term = b[e, s] * (1.0 if weights is None else float(weights[t, j]))
        out[t] += term
        size[t] += term.abs()
    return out, size


def combine_backward(dout, buffer, experts, slots, weights):
    """(dbuffer, dweights, sum of the sizes of dweights' terms)."""
    b, d = buffer.cpu().double(), dout.cpu().double()
    db = torch.zeros_like(b)
    dw = torch.zeros(experts.shape, dtype=torch.float64)
    size = dw.clone()
    for t, j, e, s in places(experts, slots, *b.shape[:2]):
        db[e, s] = d[t] * float(weights[t, j])
        dw[t, j] = (d[t] * b[e, s]).sum()
        size[t, j] = (d[t] * b[e, s]).abs().sum()
    return db, dw, size
