"""Timed cases of the experts' own operators: the gated feed-forward of the
rows that an Alltoall brings, with its gradient, the whole expert layer of a
few tokens, and the dropout that adds the residual.

A case is a plain dict:
  op          ffn (rows [sources, experts, capacity, dim] through their
              experts), ffn_tokens (choice, experts and weighted sum of a few
              tokens) or dropout (residual + dropout of rows)
  backward    whether the pass is the gradient's
  dtype       bf16, f16 or f32
  tokens, dim rows and columns (ffn: dim alone)
  hidden      columns between the experts' two products
  experts, k  experts, choices per token
  sources, capacity
              ranks that rows come from, rows that each has per expert
  pad         columns between rows beyond the dim (row stride dim + pad)
  renorm      the chosen probabilities are divided by their sum
  masked      one token of so many is padding (0: none)
  p           share that dropout drops
  residual    whether dropout adds one

An expert has w_in [2 hidden, dim] (gate rows, then up rows) and w_out [dim,
hidden]: y = w_out (silu(gate x) * (up x)). Inputs are made on the GPU from
the seed: normalised rows, weights that keep their size, uneven loads (some
past the capacity, one expert without rows). Dropout's random numbers are
SplitMix64's outputs for a counter: row r, columns c and c + 1 (c even) take
the low and high half of word offset + r * ceil(dim / 2) + c / 2, and what is
below p * 2^32 is dropped.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GOLDEN, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB

# no drawn case does more than the largest listed ones
MOST_FLOPS, MOST_WEIGHTS, MOST_ROWS = 2.4e12, 2.5e9, 8e8


def _case(name, op, backward=False, dtype="bf16", tokens=0, dim=0, hidden=0, experts=0, k=0,
          sources=1, capacity=0, pad=0, renorm=True, masked=0, p=0.0, residual=False):
    return {"name": name, "op": op, "backward": backward, "dtype": dtype, "tokens": tokens,
            "dim": dim, "hidden": hidden, "experts": experts, "k": k, "sources": sources,
            "capacity": capacity, "pad": pad, "renorm": renorm, "masked": masked, "p": p,
            "residual": residual}


def listed():
    return [
        # one new token per step in serving
        _case("tokens_one", "ffn_tokens", tokens=1, dim=4096, hidden=1536, experts=64, k=4),
        # a serving batch: most experts are chosen by some token
        _case("tokens_batch", "ffn_tokens", tokens=16, dim=2048, hidden=1024, experts=128, k=8),
        # odd sizes with padding tokens
        _case("tokens_odd", "ffn_tokens", dtype="f16", tokens=37, dim=1111, hidden=777, experts=24,
              k=2, pad=5, masked=7, renorm=False),
        # a small layer in 32 bits, where latency counts
        _case("tokens_small", "ffn_tokens", dtype="f32", tokens=4, dim=512, hidden=256, experts=16,
              k=2),
        # a long prompt on one rank
        _case("ffn_prompt", "ffn", dim=4096, hidden=1536, experts=64, capacity=1280),
        # a rank's four experts, behind an Alltoall of 16 ranks
        _case("ffn_received", "ffn", dim=2048, hidden=1024, experts=4, sources=16, capacity=80),
        # a training batch's gradients, and their smaller form behind an Alltoall
        _case("ffn_train_back", "ffn", True, dim=2048, hidden=1024, experts=64, capacity=640),
        _case("ffn_received_back", "ffn", True, dtype="f32", dim=1024, hidden=512, experts=4,
              sources=4, capacity=64),
        # odd sizes
        _case("ffn_odd_back", "ffn", True, dtype="f16", dim=1111, hidden=515, experts=6,
              sources=3, capacity=101),
        # one token's rows
        _case("dropout_token", "dropout", dtype="f16", tokens=1, dim=4096, p=0.1, residual=True),
        # a training batch
        _case("dropout_train", "dropout", tokens=8192, dim=4096, p=0.1, residual=True),
        # the gradient's call at an odd width, rows of a wider array
        _case("dropout_odd", "dropout", dtype="f32", tokens=3001, dim=1999, p=0.3, pad=33),
    ]


def draw(rng):
    def between(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    def width(lo, hi):
        n = between(lo, hi)
        return n if rng.random() < 0.5 else max(lo, n // 64 * 64)

    while True:
        op = rng.choice(["ffn", "ffn", "ffn_tokens", "ffn_tokens", "dropout"])
        c = _case("", op, op == "ffn" and rng.random() < 0.5, rng.choice(["bf16", "f16", "f32"]))
        del c["name"]
        c["dim"] = width(64, 8192)
        if op == "dropout":
            c["tokens"], c["pad"] = between(1, 32768), rng.choice([0, 0, 8, 33])
            c["p"], c["residual"] = rng.choice([0.05, 0.1, 0.3, 0.5]), rng.random() < 0.5
        else:
            c["hidden"], c["experts"] = width(32, 4096), between(1, 128)
        if op == "ffn":
            c["sources"] = rng.choice([1, 1, 2, 4, 8, 16])
            c["capacity"] = between(1, 2048)
        if op == "ffn_tokens":
            c["tokens"], c["pad"] = between(1, 64), rng.choice([0, 0, 5, 8])
            c["k"] = rng.randint(1, min(8, c["experts"]))
            c["renorm"], c["masked"] = rng.random() < 0.5, rng.choice([0, 0, 7])
        size = TYPES[c["dtype"]].itemsize
        rows = c["tokens"] + c["sources"] * c["experts"] * c["capacity"]
        if (work(c)["flops"] <= MOST_FLOPS * (0.1 if size == 4 else 1)
                and 3 * c["experts"] * c["dim"] * c["hidden"] * size <= MOST_WEIGHTS
                and rows * (c["dim"] + c["hidden"]) * size <= MOST_ROWS):
            return c


def _loads(c):
    """Tokens of every (source, expert), in no order: none, then from a
    quarter of the capacity to half again as much."""
    n = c["sources"] * c["experts"]
    out = [round(c["capacity"] * (0.25 + 1.2 * (i + 0.5) / n)) for i in range(n)]
    return [0] + out[1:] if n > 2 else out


def _distinct(c):
    """Experts that some token chooses, if all are as likely."""
    t = c["tokens"] - (c["tokens"] // c["masked"] if c["masked"] else 0)
    return c["experts"] * (1 - (1 - c["k"] / c["experts"]) ** t)


def work(case):
    c = case
    t, d, f, e, k = c["tokens"], c["dim"], c["hidden"], c["experts"], c["k"]
    size = TYPES[c["dtype"]].itemsize
    if c["op"] == "dropout":
        return {"bytes": (3 if c["residual"] else 2) * t * d * size + 16, "flops": 3 * t * d}
    if c["op"] == "ffn_tokens":
        kept = (t - t // c["masked"] if c["masked"] else t) * k
        return {"bytes": _distinct(c) * 3 * d * f * size + 2 * t * d * size + 4 * t * e + 8 * t * k,
                "flops": 6 * kept * d * f}
    rows = c["sources"] * e * c["capacity"]
    full = sum(min(n, c["capacity"]) for n in _loads(c))
    weights = 3 * e * d * f * size
    if c["backward"]:
        return {"bytes": 2 * weights + full * (2 * d + 2 * f) * size + rows * d * size,
                "flops": 12 * full * d * f}
    return {"bytes": weights + full * d * size + rows * d * size, "flops": 6 * full * d * f}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _weights(gen, dtype, experts, rows, cols):
    """[experts, rows, cols], of a size that keeps a row's size."""
    w = torch.empty(experts, rows, cols, dtype=dtype, device="cuda")
    for e in range(experts):
        w[e] = _randn(gen, rows, cols) / cols ** 0.5
    return w


def _padded(gen, c, dtype):
    return _randn(gen, c["tokens"], c["dim"] + c["pad"]).to(dtype)[:, :c["dim"]]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, d, f, e, k = c["tokens"], c["dim"], c["hidden"], c["experts"], c["k"]
    dtype = TYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "dropout":
        s["x"] = _padded(gen, c, dtype)
        s["residual"] = _padded(gen, c, dtype) if c["residual"] else None
        s["rng"] = torch.randint(0, 1 << 40, (2,), generator=gen, device="cuda")
        s["out"] = torch.empty(t, d, dtype=dtype, device="cuda")
        return s
    s["w_in"] = _weights(gen, dtype, e, 2 * f, d)
    s["w_out"] = _weights(gen, dtype, e, d, f)
    if c["op"] == "ffn_tokens":
        s["x"] = _padded(gen, c, dtype)
        s["logits"] = 1.5 * _randn(gen, t, e) + 0.5 * _randn(gen, e)
        s["mask"] = None
        if c["masked"]:
            at = torch.arange(t, device="cuda")
            s["mask"] = (at % c["masked"] != c["masked"] - 1).to(torch.uint8)
        s["out"] = torch.empty(t, d, dtype=dtype, device="cuda")
        s["experts"] = torch.empty(t, k, dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty(t, k, device="cuda")
        s["work"] = torch.empty((1 << 20) + 8 * t * min(e, t * k) * (f + 8) + 256 * t * d,
                                dtype=torch.uint8, device="cuda")
        return s
    shape = (c["sources"], e, c["capacity"])
    rows = shape[0] * shape[1] * shape[2]
    loads = torch.tensor(_loads(c), dtype=torch.int32, device="cuda")
    loads = loads[torch.randperm(len(loads), generator=gen, device="cuda")]
    s["counts"] = loads.view(shape[0], e)
    there = torch.arange(c["capacity"], device="cuda") < s["counts"][..., None]

    def filled(n):  # rows from the count on are zero, as dispatch leaves them
        return (_randn(gen, *shape, n) * there[..., None]).to(dtype)

    s["buffer"] = filled(d)
    size = dtype.itemsize
    if c["backward"]:
        s["dout"], s["pre"] = filled(d), filled(2 * f)
        s["dbuffer"] = torch.empty_like(s["buffer"])
        s["dw_in"], s["dw_out"] = torch.empty_like(s["w_in"]), torch.empty_like(s["w_out"])
        s["work"] = torch.empty((1 << 20) + rows * (3 * (f + 8) * size + 64) + 64 * e,
                                dtype=torch.uint8, device="cuda")
    else:
        s["out"] = torch.empty_like(s["buffer"])
        s["work"] = torch.empty((1 << 20) + rows * ((f + 8) * size + 64) + 64 * e,
                                dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------------------------
# the operators' plain forms, in 32 bits
# --------------------------------------------------------------------------

def _silu(g):
    return g * torch.sigmoid(g)


def _there(s, c):
    """[sources, experts, capacity, 1]: rows below their count."""
    return (torch.arange(c["capacity"], device="cuda") < s["counts"][..., None])[..., None]


def _expert_rows(rows, there, e, c):
    """Expert e's rows of all sources in 32 bits, zero from the counts on."""
    got = torch.where(there[:, e], rows[:, e].float(), 0.0)
    return got.reshape(c["sources"] * c["capacity"], -1)


def _ffn(s, c):
    there, f = _there(s, c), c["hidden"]
    out = torch.empty_like(s["buffer"])
    for e in range(c["experts"]):
        h = _expert_rows(s["buffer"], there, e, c) @ s["w_in"][e].float().t()
        y = (_silu(h[:, :f]) * h[:, f:]) @ s["w_out"][e].float().t()
        out[:, e] = y.view(c["sources"], c["capacity"], -1).to(out.dtype)
    return {"out": out}


def _ffn_backward(s, c):
    there, f = _there(s, c), c["hidden"]
    dbuffer, dw_in, dw_out = (torch.empty_like(s[n]) for n in ("buffer", "w_in", "w_out"))
    for e in range(c["experts"]):
        x, dy, pre = (_expert_rows(s[n], there, e, c) for n in ("buffer", "dout", "pre"))
        g, u = pre[:, :f], pre[:, f:]
        sig = torch.sigmoid(g)
        da = dy @ s["w_out"][e].float()
        dpre = torch.cat([da * u * sig * (1 + g * (1 - sig)), da * g * sig], 1)
        dx = dpre @ s["w_in"][e].float()
        dbuffer[:, e] = dx.view(c["sources"], c["capacity"], -1).to(dbuffer.dtype)
        dw_out[e] = (dy.t() @ (g * sig * u)).to(dw_out.dtype)
        dw_in[e] = (dpre.t() @ x).to(dw_in.dtype)
    return {"dbuffer": dbuffer, "dw_in": dw_in, "dw_out": dw_out}


def _choices(s, c):
    x = s["logits"]
    if s["mask"] is not None:
        x = torch.where(s["mask"][:, None] != 0, x, float("-inf"))
    top = x.amax(1, keepdim=True)
    live = top > float("-inf")
    p = torch.where(live, torch.exp(x - torch.where(live, top, 0.0)), 0.0)
    p = p / p.sum(1, keepdim=True).clamp_min(1e-30)
    ranked, order = torch.sort(x, dim=1, descending=True, stable=True)
    there = ranked[:, :c["k"]] > float("-inf")
    experts = torch.where(there, order[:, :c["k"]], -1)
    weights = torch.where(there, p.gather(1, order[:, :c["k"]]), 0.0)
    if c["renorm"]:
        weights = weights / weights.sum(1, keepdim=True).clamp_min(1e-30)
    return experts, weights


def _ffn_tokens(s, c):
    experts, weights = _choices(s, c)
    x, f, t, k = s["x"].float(), c["hidden"], c["tokens"], c["k"]
    out = torch.zeros(t, c["dim"], device=x.device)
    if t * k <= c["experts"]:  # the weights of every choice
        for i in range(t):
            at = experts[i].clamp_min(0)
            h = s["w_in"][at].float() @ x[i]
            y = s["w_out"][at].float() @ (_silu(h[:, :f]) * h[:, f:])[..., None]
            out[i] = (y[..., 0] * weights[i][:, None]).sum(0)
    else:  # every expert on all tokens
        for e in range(c["experts"]):
            w = torch.where(experts == e, weights, 0.0).sum(1, keepdim=True)
            h = x @ s["w_in"][e].float().t()
            out += w * ((_silu(h[:, :f]) * h[:, f:]) @ s["w_out"][e].float().t())
    return {"out": out.to(s["x"].dtype), "experts": experts.int(), "weights": weights}


def _signed(n):
    return n - (1 << 64) if n >> 63 else n


def _shifted(z, n):
    """z >> n of unsigned 64-bit numbers."""
    return (z >> n) & ((1 << (64 - n)) - 1)


def _kept(rng, c):
    t, half = c["tokens"], -(-c["dim"] // 2)
    at = torch.arange(t * half, device="cuda") + rng[1] + 1
    z = rng[0] + at * _signed(GOLDEN)
    z = (z ^ _shifted(z, 30)) * _signed(MIX1)
    z = (z ^ _shifted(z, 27)) * _signed(MIX2)
    z = z ^ _shifted(z, 31)
    field = torch.stack([z & 0xFFFFFFFF, _shifted(z, 32)], 1).view(t, 2 * half)[:, :c["dim"]]
    return field >= math.ceil(c["p"] * 2 ** 32)


def _dropout(s, c):
    y = torch.where(_kept(s["rng"], c), s["x"].float() * (1 / (1 - c["p"])), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"out": y.to(s["x"].dtype)}


PLAIN = {("ffn", False): _ffn, ("ffn", True): _ffn_backward, ("ffn_tokens", False): _ffn_tokens,
         ("dropout", False): _dropout}


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------

def _run_own(s, c):
    from paper_2111_04867_amd import experts as X

    if c["op"] == "dropout":
        X.dropout_tensors(s["x"], s["rng"], s["out"], p=c["p"], residual=s["residual"])
        return {"out": s["out"]}
    if c["op"] == "ffn_tokens":
        X.ffn_tokens_tensors(s["x"], s["logits"], s["w_in"], s["w_out"], s["out"], s["work"],
                             k=c["k"], mask=s["mask"], renorm=c["renorm"], experts=s["experts"],
                             weights=s["weights"])
        return {n: s[n] for n in ("out", "experts", "weights")}
    if c["backward"]:
        X.ffn_backward_tensors(s["dout"], s["buffer"], s["counts"], s["w_in"], s["w_out"],
                               s["pre"], s["work"], dbuffer=s["dbuffer"], dw_in=s["dw_in"],
                               dw_out=s["dw_out"])
        return {n: s[n] for n in ("dbuffer", "dw_in", "dw_out")}
    X.ffn_tensors(s["buffer"], s["counts"], s["w_in"], s["w_out"], s["out"], s["work"])
    return {"out": s["out"]}


def run(state):
    c = state["case"]
    return _run_own(state, c) if own else PLAIN[c["op"], c["backward"]](state, c)


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def _gated(rows, w_in, w_out):
    """One expert's rows, in 64 bits."""
    gate, up = w_in.double().chunk(2)
    g = torch.mm(rows, gate.T)
    return torch.mm(g / (1 + torch.exp(-g)) * torch.mm(rows, up.T), w_out.double().T)


def _exact_ffn(s, c):
    held = s["counts"].clamp(max=c["capacity"]).tolist()
    shape = s["buffer"].shape
    if not c["backward"]:
        out = torch.zeros(shape, dtype=torch.float64, device="cuda")
        for e in range(c["experts"]):
            for i, n in enumerate(h[e] for h in held):
                out[i, e, :n] = _gated(s["buffer"][i, e, :n].double(), s["w_in"][e], s["w_out"][e])
        return {"out": out}
    out = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda")
           for n in ("dbuffer", "dw_in", "dw_out")}
    for e in range(c["experts"]):
        w_in, w_out = s["w_in"][e].double(), s["w_out"][e].double()
        for i, n in enumerate(h[e] for h in held):
            x, dy, pre = (s[a][i, e, :n].double() for a in ("buffer", "dout", "pre"))
            g, u = pre.chunk(2, 1)
            ex = torch.exp(-g)
            act = g / (1 + ex)
            slope = (1 + ex + g * ex) / (1 + ex) ** 2  # of g / (1 + exp(-g))
            da = torch.mm(dy, w_out)
            dpre = torch.cat((da * u * slope, da * act), 1)
            out["dbuffer"][i, e, :n] = torch.mm(dpre, w_in)
            out["dw_in"][e] += torch.mm(dpre.T, x)
            out["dw_out"][e] += torch.mm(dy.T, act * u)
    return out


def _exact_tokens(s, c):
    logits, k = s["logits"].double(), c["k"]
    rank = torch.argsort(logits, dim=1, descending=True, stable=True)[:, :k]
    picked = logits.gather(1, rank)
    if c["renorm"]:
        weights = torch.softmax(picked, 1)
    else:
        weights = torch.exp(picked - torch.logsumexp(logits, 1, keepdim=True))
    if s["mask"] is not None:
        weights[s["mask"] == 0] = 0
    out = torch.zeros(c["tokens"], c["dim"], dtype=torch.float64, device="cuda")
    for e in range(c["experts"]):
        t, j = torch.nonzero((rank == e) & (weights > 0), as_tuple=True)
        if len(t):
            out[t] += weights[t, j][:, None] * _gated(s["x"][t].double(), s["w_in"][e],
                                                      s["w_out"][e])
    return {"out": out, "experts": None, "weights": weights}


def _exact_dropout(s, c):
    # the generator on numpy's unsigned numbers, its words seen as 32-bit halves
    import numpy as np

    seed, offset = (np.uint64(v) for v in s["rng"].tolist())
    half = -(-c["dim"] // 2)
    with np.errstate(over="ignore"):
        z = seed + (offset + np.uint64(1) + np.arange(c["tokens"] * half, dtype=np.uint64)
                    ) * np.uint64(GOLDEN)
        z = (z ^ z >> np.uint64(30)) * np.uint64(MIX1)
        z = (z ^ z >> np.uint64(27)) * np.uint64(MIX2)
        z ^= z >> np.uint64(31)
    drops = z.view(np.uint32).reshape(c["tokens"], 2 * half)[:, :c["dim"]] < c["p"] * 2 ** 32
    y = s["x"].double() / (1 - c["p"])
    y[torch.from_numpy(drops).cuda()] = 0
    return {"out": y if s["residual"] is None else y + s["residual"].double()}


EXACT = {"ffn": _exact_ffn, "ffn_tokens": _exact_tokens, "dropout": _exact_dropout}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed), case)
