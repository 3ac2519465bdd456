"""Timed cases of the expert-layer operators around an expert-parallel
Alltoall: norm, route, dispatch and combine, forward and backward.

A case is a plain dict:
  op          norm (root-mean-square norm after the residual's addition, with
              the 8-bit copy that travels), route (choices, slots, counts and
              balance loss from the router's logits), dispatch (token rows
              into the exchange buffer) or combine (rows back to tokens)
  backward    whether the pass is the gradient's
  tokens, dim rows and columns
  dtype       bf16, f16 or f32 (dispatch also f8: 8-bit rows with scales)
  group       columns per scale of an 8-bit row, 0 for one scale per row
  pad         columns between rows beyond the dim (row stride dim + pad)
  experts, k, capacity
              experts, choices per token, buffer rows per expert
  renorm      the chosen probabilities are divided by their sum
  masked      one token of so many is padding (0: none)

Inputs are made on the GPU from the seed: activations with a few large
columns, router logits with popular experts (so that some choices are past
the capacity and some buffer rows stay empty). Integer outputs have one right
value; ties go to the lowest index.
"""
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
         "f8": torch.float8_e4m3fn}
EPS, COEF = 1e-6, 0.01
F8_MAX, AMAX_MIN = 448.0, 2.0 ** -100

# no case moves more than the largest listed one (dispatch_train)
MOST_BYTES = 7.5e8


def _case(name, op, backward, tokens, dim=0, dtype="bf16", group=128, pad=0, experts=0, k=0,
          capacity=0, renorm=True, masked=0):
    return {"name": name, "op": op, "backward": backward, "tokens": tokens, "dim": dim,
            "dtype": dtype, "group": group, "pad": pad, "experts": experts, "k": k,
            "capacity": capacity, "renorm": renorm, "masked": masked}


def _capacity(tokens, k, experts):
    """A quarter more rows than an even load needs."""
    return max(1, -(-5 * tokens * k // (4 * experts)))


def listed():
    cap = _capacity
    return [
        # one new token per step in serving
        _case("norm_token", "norm", False, 1, 4096),
        # a long prompt
        _case("norm_prompt", "norm", False, 8192, 4096),
        # training at a smaller width
        _case("norm_train_back", "norm", True, 8192, 2048),
        # odd width, rows of a wider array
        _case("norm_odd_back", "norm", True, 3001, 1999, "f16", pad=33),
        # a serving batch of 16 tokens
        _case("route_batch", "route", False, 16, dtype="f32", experts=64, k=4,
              capacity=cap(16, 4, 64)),
        # a training batch
        _case("route_train", "route", False, 32768, dtype="f32", experts=256, k=8,
              capacity=cap(32768, 8, 256)),
        # gradients with padding tokens and an odd number of experts
        _case("route_odd_back", "route", True, 10007, dtype="bf16", experts=60, k=4,
              capacity=cap(10007, 4, 60), renorm=False, masked=7),
        # a serving batch, 8-bit rows
        _case("dispatch_batch", "dispatch", False, 32, 4096, "f8", experts=64, k=4,
              capacity=cap(32, 4, 64)),
        # a training batch, 8-bit rows
        _case("dispatch_train", "dispatch", False, 16384, 4096, "f8", experts=128, k=8,
              capacity=cap(16384, 8, 128)),
        # odd width in 32 bits
        _case("combine_odd", "combine", False, 509, 1111, "f32", experts=24, k=2,
              capacity=cap(509, 2, 24)),
        # a training batch and its gradients
        _case("combine_train", "combine", False, 8192, 4096, experts=64, k=8,
              capacity=cap(8192, 8, 64)),
        _case("combine_train_back", "combine", True, 8192, 2048, experts=128, k=6,
              capacity=cap(8192, 6, 128)),
    ]


def draw(rng):
    def between(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    while True:
        op = rng.choice(["norm", "route", "dispatch", "combine"])
        c = _case("", op, op != "dispatch" and rng.random() < 0.5, between(1, 32768))
        del c["name"]
        c["dtype"] = rng.choice(["bf16", "f16", "f32"])
        if op != "route":
            c["dim"] = between(64, 8192)
            if rng.random() < 0.5:
                c["dim"] = max(64, c["dim"] // 64 * 64)
        if op == "norm":
            c["group"] = rng.choice([0, 64, 128])
            c["pad"] = rng.choice([0, 0, 8, 33])
        else:
            c["experts"] = between(4, 256)
            c["k"] = rng.randint(1, min(8, c["experts"]))
            c["capacity"] = _capacity(c["tokens"], c["k"], c["experts"])
            c["renorm"] = rng.random() < 0.5
            c["masked"] = rng.choice([0, 0, 7])
        if op == "dispatch" and rng.random() < 0.5:
            c["dtype"], c["group"] = "f8", rng.choice([0, 64, 128])
        if work(c)["bytes"] <= MOST_BYTES:
            return c


def _groups(c):
    return -(-c["dim"] // c["group"]) if c["group"] else 1


def work(case):
    c = case
    t, d, e, k = c["tokens"], c["dim"], c["experts"], c["k"]
    size = TYPES[c["dtype"]].itemsize
    if c["op"] == "norm":
        if c["backward"]:
            return {"bytes": 4 * t * d * size + d * (size + 4), "flops": 10 * t * d}
        return {"bytes": 4 * t * d * size + t * d + 4 * t * _groups(c) + d * size,
                "flops": 8 * t * d}
    if c["op"] == "route":
        if c["backward"]:
            return {"bytes": 2 * t * e * size + 8 * t * k + 4 * e, "flops": 8 * t * e}
        return {"bytes": t * e * size + 12 * t * k + 8 * e, "flops": 5 * t * e}
    kept = (t - t // c["masked"] if c["masked"] else t) * k
    rows = e * c["capacity"]
    index = 8 * t * k
    if c["op"] == "dispatch":
        row = d * size + (4 * _groups(c) if c["dtype"] == "f8" else 0)
        return {"bytes": (t + rows) * row + index + 4 * e, "flops": 0}
    kept = min(kept, rows)
    if c["backward"]:
        return {"bytes": (t + kept + rows) * d * size + index + 8 * t * k + 4 * e,
                "flops": 3 * kept * d}
    return {"bytes": (t + kept) * d * size + index + 4 * t * k, "flops": 2 * kept * d}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _rows(gen, c, tokens, dtype):
    """Activations [tokens, dim] with some large columns, rows dim + pad apart."""
    x = _randn(gen, tokens, c["dim"] + c["pad"])
    x *= torch.exp(0.7 * _randn(gen, c["dim"] + c["pad"]))
    return x.to(dtype)[:, :c["dim"]]


def _logits(gen, c):
    """Router logits; a token's are near its neighbours', some experts popular."""
    e = c["experts"]
    return 1.5 * _randn(gen, c["tokens"], e) + 0.5 * _randn(gen, e)


def _mask(c):
    """uint8 [tokens], 0 for padding tokens, or None."""
    if not c["masked"]:
        return None
    at = torch.arange(c["tokens"], device="cuda")
    return (at % c["masked"] != c["masked"] - 1).to(torch.uint8)


def _f32(*shape):
    return torch.empty(*shape, dtype=torch.float32, device="cuda")


def _i32(*shape):
    return torch.empty(*shape, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, d, e, k, cap = c["tokens"], c["dim"], c["experts"], c["k"], c["capacity"]
    dtype = TYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "norm":
        s["weight"] = (1 + 0.1 * _randn(gen, d)).to(dtype)
        s["x"] = _rows(gen, c, t, dtype)
        s["residual"] = _rows(gen, c, t, dtype)
        if c["backward"]:
            s["dout"] = _rows(gen, c, t, dtype)
            s["dx"] = torch.empty(t, d, dtype=dtype, device="cuda")
            s["dweight"] = _f32(d)
            s["work"] = torch.empty(4 * 1024 * d, dtype=torch.uint8, device="cuda")
        else:
            s["out"] = torch.empty(t, d, dtype=dtype, device="cuda")
            s["total"] = torch.empty(t, d, dtype=dtype, device="cuda")
            s["q"] = torch.empty(t, d, dtype=TYPES["f8"], device="cuda")
            s["scale"] = _f32(t, _groups(c))
        return s
    logits, s["mask"] = _logits(gen, c), _mask(c)
    if c["op"] == "route":
        s["logits"] = logits.to(dtype)
        s["work"] = torch.empty(1 << 23, dtype=torch.uint8, device="cuda")
        if not c["backward"]:
            s["experts"], s["slots"], s["weights"] = _i32(t, k), _i32(t, k), _f32(t, k)
            s["counts"], s["prob_sums"], s["loss"], s["rows"] = _i32(e), _f32(e), _f32(1), _i32(1)
            return s
    r = _route(logits.to(dtype) if c["op"] == "route" else logits, s["mask"], c)
    s["experts"], s["slots"], s["counts"] = r["experts"], r["slots"], r["counts"]
    s["weights"], s["rows"] = r["weights"], r["rows"]
    if c["op"] == "route":
        s["dweights"] = _randn(gen, t, k)
        s["dloss"] = torch.ones(1, device="cuda")
        s["dlogits"] = torch.empty_like(s["logits"])
    elif c["op"] == "dispatch":
        x = _randn(gen, t, d)
        if c["dtype"] == "f8":
            s["x"] = (40 * x).to(dtype)
            s["scale"] = torch.rand(t, _groups(c), generator=gen, device="cuda") + 0.1
            s["out_scale"] = _f32(e, cap, _groups(c))
        else:
            s["x"] = x.to(dtype)
        s["out"] = torch.empty(e, cap, d, dtype=dtype, device="cuda")
    else:
        s["buffer"] = _randn(gen, e, cap, d).to(dtype)
        if c["backward"]:
            s["dout"] = _randn(gen, t, d).to(dtype)
            s["dbuffer"] = torch.empty(e, cap, d, dtype=dtype, device="cuda")
            s["dweights"] = _f32(t, k)
        else:
            s["out"] = torch.empty(t, d, dtype=dtype, device="cuda")
    return s


# --------------------------------------------------------------------------
# the operators' plain forms, in 32 bits
# --------------------------------------------------------------------------

def _norm(s, c):
    d, group = c["dim"], c["group"] or c["dim"]
    h = s["x"].float() + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
    full = torch.zeros(len(y), _groups(c) * group, device=y.device)
    full[:, :d] = y
    full = full.view(len(y), -1, group)
    scale = full.abs().amax(2).clamp_min(AMAX_MIN) / F8_MAX
    q = (full / scale[..., None]).view(len(y), -1)[:, :d]
    return {"out": y.to(s["x"].dtype), "total": h.to(s["x"].dtype),
            "q": q.to(torch.float8_e4m3fn), "scale": scale}


def _norm_backward(s, c):
    h, dy = s["x"].float(), s["dout"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    a = dy * s["weight"].float()
    dx = s["residual"].float() + r * a - h * (r * r * r * (a * h).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * h * r).sum(0)}


def _softmax(logits, mask):
    """(probabilities, rows that count): zeros in masked rows."""
    x = logits.float()
    if mask is not None:
        x = torch.where(mask[:, None] != 0, x, float("-inf"))
    top = x.amax(1, keepdim=True)
    live = top > float("-inf")
    p = torch.where(live, torch.exp(x - torch.where(live, top, 0.0)), 0.0)
    return x, p / p.sum(1, keepdim=True).clamp_min(1e-30), live


def _route(logits, mask, c):
    e, k, cap = c["experts"], c["k"], c["capacity"]
    x, p, live = _softmax(logits, mask)
    ranked, order = torch.sort(x, dim=1, descending=True, stable=True)
    there = ranked[:, :k] > float("-inf")
    experts = torch.where(there, order[:, :k], -1)
    weights = torch.where(there, p.gather(1, order[:, :k]), 0.0)
    if c["renorm"]:
        weights = weights / weights.sum(1, keepdim=True).clamp_min(1e-30)
    flat = torch.where(there, experts, e).reshape(-1)
    sums = torch.zeros(e + 1, dtype=torch.int64, device=x.device)
    sums.index_add_(0, flat, torch.ones_like(flat))
    by_expert, at = torch.sort(flat, stable=True)
    first = sums.cumsum(0) - sums
    slot = torch.empty_like(flat)
    slot[at] = torch.arange(len(flat), device=x.device) - first[by_expert]
    slots = torch.where(there & (slot.view(-1, k) < cap), slot.view(-1, k), -1)
    counts, prob_sums, rows = sums[:e], p.sum(0), live.sum()
    n = rows.float().clamp_min(1)
    loss = COEF * e * (counts.float() / (n * k) * (prob_sums / n)).sum()
    return {"experts": experts.int(), "slots": slots.int(), "weights": weights,
            "counts": counts.int(), "prob_sums": prob_sums, "loss": loss.view(1),
            "rows": rows.int().view(1)}


def _route_backward(s, c):
    e, k = c["experts"], c["k"]
    _, p, live = _softmax(s["logits"], s["mask"])
    n = s["rows"].float().clamp_min(1)
    g = (s["dloss"] * COEF * e * s["counts"].float() / (n * n * k)).expand_as(p)
    there = s["experts"] >= 0
    at = s["experts"].clamp_min(0).long()
    dw = torch.where(there, s["dweights"], 0.0)
    chosen = torch.zeros_like(p)
    if c["renorm"]:
        w = torch.where(there, p.gather(1, at), 0.0)
        w = w / w.sum(1, keepdim=True).clamp_min(1e-30)
        chosen.scatter_add_(1, at, w * (dw - (w * dw).sum(1, keepdim=True)))
        dl = p * (g - (p * g).sum(1, keepdim=True)) + chosen
    else:
        chosen.scatter_add_(1, at, dw)
        g = g + chosen
        dl = p * (g - (p * g).sum(1, keepdim=True))
    return {"dlogits": dl.to(s["logits"].dtype)}


def _at(s, c):
    """Buffer row of every choice [tokens, k]; the row past the buffer where it has none."""
    there = (s["experts"] >= 0) & (s["slots"] >= 0)
    return torch.where(there, s["experts"] * c["capacity"] + s["slots"],
                       c["experts"] * c["capacity"]).long()


def _spread(rows, at, c):
    """Rows [tokens, k, n] in a buffer [experts, capacity, n], zero elsewhere."""
    out = torch.zeros(c["experts"] * c["capacity"] + 1, rows.shape[2], dtype=rows.dtype,
                      device=rows.device)
    out[at.reshape(-1)] = rows.reshape(-1, rows.shape[2])
    return out[:-1].view(c["experts"], c["capacity"], -1)


def _dispatch(s, c):
    at, k = _at(s, c), c["k"]
    raw = s["x"].view(torch.uint8) if c["dtype"] == "f8" else s["x"]
    out = _spread(raw[:, None].expand(-1, k, -1), at, c).view(s["x"].dtype)
    if c["dtype"] != "f8":
        return {"out": out}
    return {"out": out, "scale": _spread(s["scale"][:, None].expand(-1, k, -1), at, c)}


def _chosen_rows(s, c):
    there = (s["experts"] >= 0) & (s["slots"] >= 0)
    rows = s["buffer"][s["experts"].clamp_min(0).long(), s["slots"].clamp_min(0).long()].float()
    return there, rows


def _combine(s, c):
    there, rows = _chosen_rows(s, c)
    w = torch.where(there, s["weights"], 0.0)
    return {"out": (rows * w[..., None]).sum(1).to(s["buffer"].dtype)}


def _combine_backward(s, c):
    there, rows = _chosen_rows(s, c)
    dout = s["dout"].float()[:, None]
    given = (dout * s["weights"][..., None]).to(s["buffer"].dtype)
    return {"dbuffer": _spread(given, _at(s, c), c),
            "dweights": torch.where(there, (dout * rows).sum(2), 0.0)}


PLAIN = {("norm", False): _norm, ("norm", True): _norm_backward, ("route", False):
         lambda s, c: _route(s["logits"], s["mask"], c), ("route", True): _route_backward,
         ("dispatch", False): _dispatch, ("combine", False): _combine,
         ("combine", True): _combine_backward}


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------

def _run_own(s, c):
    from paper_2111_04867_amd import experts as X

    if c["op"] == "norm":
        if c["backward"]:
            X.norm_backward_tensors(s["dout"], s["x"], s["weight"], s["dx"], s["dweight"],
                                    s["work"], eps=EPS, dtotal=s["residual"])
            return {"dx": s["dx"], "dweight": s["dweight"]}
        X.norm_tensors(s["x"], s["weight"], s["out"], eps=EPS, residual=s["residual"],
                       total=s["total"], q=s["q"], scale=s["scale"], group=c["group"])
        return {"out": s["out"], "total": s["total"], "q": s["q"], "scale": s["scale"]}
    if c["op"] == "route":
        if c["backward"]:
            X.route_backward_tensors(s["logits"], s["experts"], s["counts"], s["rows"],
                                     s["dlogits"], dweights=s["dweights"], dloss=s["dloss"],
                                     mask=s["mask"], coef=COEF, renorm=c["renorm"])
            return {"dlogits": s["dlogits"]}
        X.route_tensors(s["logits"], s["experts"], s["weights"], s["slots"], s["counts"],
                        s["prob_sums"], s["loss"], s["rows"], s["work"], mask=s["mask"],
                        capacity=c["capacity"], coef=COEF, renorm=c["renorm"])
        return {n: s[n] for n in ("experts", "slots", "weights", "counts", "prob_sums", "loss",
                                  "rows")}
    if c["op"] == "dispatch":
        X.dispatch_tensors(s["x"], s["experts"], s["slots"], s["counts"], s["out"],
                           scale=s.get("scale"), out_scale=s.get("out_scale"))
        return {"out": s["out"], "scale": s["out_scale"]} if "scale" in s else {"out": s["out"]}
    if c["backward"]:
        X.combine_backward_tensors(s["dout"], s["buffer"], s["experts"], s["slots"], s["counts"],
                                   s["weights"], s["dbuffer"], s["dweights"])
        return {"dbuffer": s["dbuffer"], "dweights": s["dweights"]}
    X.combine_tensors(s["buffer"], s["experts"], s["slots"], s["out"], weights=s["weights"])
    return {"out": s["out"]}


def run(state):
    c = state["case"]
    return _run_own(state, c) if own else PLAIN[c["op"], c["backward"]](state, c)


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def _exact_norm(s, c):
    x, w = s["x"].double(), s["weight"].double()
    if not c["backward"]:
        x = x + s["residual"].double()
    r = 1 / torch.sqrt(torch.linalg.vector_norm(x, dim=1) ** 2 / c["dim"] + EPS)
    if c["backward"]:
        dy = s["dout"].double()
        u = x * r[:, None]  # the normalised row: y = w u
        g = dy * w
        dx = s["residual"].double() + r[:, None] * (g - u * (g * u).mean(1)[:, None])
        return {"dx": dx, "dweight": torch.einsum("td,td->d", dy, u)}
    y = x * r[:, None] * w
    at = torch.arange(c["dim"], device=y.device) // (c["group"] or c["dim"])
    most = torch.zeros(len(y), _groups(c), dtype=torch.float64, device=y.device)
    most.scatter_reduce_(1, at.expand_as(y), y.abs(), "amax")
    scale = torch.clamp(most, min=AMAX_MIN) / F8_MAX
    return {"out": y, "total": x, "q": y / scale[:, at], "scale": scale}


def _exact_route(s, c):
    e, k = c["experts"], c["k"]
    x = s["logits"].double()
    out = torch.zeros(len(x), dtype=torch.bool, device=x.device)
    if s["mask"] is not None:
        out = s["mask"] == 0
    p = torch.softmax(x, 1).masked_fill(out[:, None], 0)
    n = max(1, int((~out).sum()))
    # the k chosen: expert indices break ties between equal logits
    rank = torch.argsort(x, dim=1, descending=True, stable=True)[:, :k]
    picked = p.gather(1, rank)
    weights = picked
    if c["renorm"]:
        weights = torch.softmax(x.gather(1, rank), 1).masked_fill(out[:, None], 0)
    load = torch.bincount(rank[~out].reshape(-1), minlength=e).double()
    if not c["backward"]:
        sums = p.sum(0)
        return {"experts": None, "slots": None, "weights": weights, "counts": None,
                "prob_sums": sums, "loss": (COEF * e / (n * n * k) * (load @ sums)).view(1),
                "rows": None}
    # through the softmax's Jacobian: loss = coef e/(n^2 k) sum load p + sum dw weights
    gp = (COEF * e / (n * n * k) * load).expand_as(p).clone()
    dw = s["dweights"].double().masked_fill(out[:, None], 0)
    if not c["renorm"]:
        gp.scatter_add_(1, rank, dw)
    dl = p * gp - p * (p * gp).sum(1, keepdim=True)
    if c["renorm"]:
        dl.scatter_add_(1, rank, weights * dw - weights * (weights * dw).sum(1, keepdim=True))
    return {"dlogits": dl}


def _exact_rows(s, c):
    """Row of the flat buffer of every choice, -1 without one, in 64 bits."""
    e, slot = s["experts"].long(), s["slots"].long()
    return torch.where((e >= 0) & (slot >= 0), e * c["capacity"] + slot, -1)


def _exact_dispatch(s, c):
    at = _exact_rows(s, c)
    token = torch.full((c["experts"] * c["capacity"] + 1,), -1, device=at.device)
    token[at.reshape(-1)] = torch.arange(len(at), device=at.device).repeat_interleave(c["k"])
    token = token[:-1]  # the last takes the choices without a row

    def rows(v):
        v = v.float()
        got = torch.where((token >= 0)[:, None], v[token.clamp_min(0)], 0.0)
        return got.view(c["experts"], c["capacity"], -1)

    return {"out": rows(s["x"]), "scale": rows(s["scale"])} if "scale" in s else {
        "out": rows(s["x"])}


def _exact_combine(s, c):
    at = _exact_rows(s, c)
    flat = s["buffer"].view(-1, c["dim"])
    if not c["backward"]:
        out = torch.zeros(len(at), c["dim"], dtype=torch.float64, device=at.device)
        for j in range(c["k"]):
            row = flat[at[:, j].clamp_min(0)].double() * s["weights"][:, j, None].double()
            out += torch.where(at[:, j, None] >= 0, row, 0.0)
        return {"out": out}
    dout = s["dout"].double()
    db = torch.zeros(len(flat) + 1, c["dim"], dtype=torch.float64, device=at.device)
    dw = torch.zeros(len(at), c["k"], dtype=torch.float64, device=at.device)
    for j in range(c["k"]):
        db[at[:, j]] = dout * s["weights"][:, j, None].double()
        dot = (dout * flat[at[:, j].clamp_min(0)].double()).sum(1)
        dw[:, j] = torch.where(at[:, j] >= 0, dot, 0.0)
    return {"dbuffer": db[:-1].view(c["experts"], c["capacity"], -1), "dweights": dw}


EXACT = {"norm": _exact_norm, "route": _exact_route, "dispatch": _exact_dispatch,
         "combine": _exact_combine}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed), case)
