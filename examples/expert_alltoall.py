"""An expert-parallel layer and the Alltoall schedule that carries its rows.

Sixteen ranks behind a switch share the layer's experts. On every rank the
token rows are normalised (and copied to 8 bits), routed to k experts and
dispatched into the rank's send buffer, whose parts for the other ranks are the
chunks of an Alltoall plan. The plan's candidate schedules are evaluated for
the chunk's size, with 16-bit rows and with 8-bit ones. The received rows go
through the experts and back, and are combined into tokens; a few training
steps on the balance loss then even the loads, so that a smaller capacity (and
chunk) drops the same share of the choices.

One GPU plays all ranks in turn; the exchange is a transposition.

    python examples/expert_alltoall.py
"""
import os
import sys
from dataclasses import replace

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2111_04867_amd import experts as X  # noqa: E402
from paper_2111_04867_amd.binding import Plan  # noqa: E402
from workloads import generate, named  # noqa: E402


def exchange(buffers, ranks):
    """What an Alltoall leaves on every rank: [dst][src, experts / ranks, capacity, n]."""
    sent = torch.stack([b.view(ranks, -1, *b.shape[1:]) for b in buffers])
    return list(sent.transpose(0, 1).contiguous())


def back(received, ranks):
    """The Alltoall the other way: buffers [experts, capacity, n] on every source."""
    sent = torch.stack(received).transpose(0, 1).contiguous()
    return [b.view(-1, *b.shape[2:]) for b in sent]


GROUP = 128  # columns per scale of an 8-bit row


def rows_in_floats(q, scale):
    """8-bit rows with their scales as bfloat16."""
    wide = scale.repeat_interleave(GROUP, dim=-1)[..., :q.shape[-1]]
    return (q.float() * wide).bfloat16()


def experts_of(rank, received, weights):
    """Rows [src, local experts, capacity, n] through the rank's experts."""
    local = received.shape[1]
    rows = received.transpose(0, 1).reshape(local, -1, received.shape[-1])
    own = weights[rank * local:(rank + 1) * local]
    out = torch.stack([torch.nn.functional.silu(r @ w) for r, w in zip(rows, own)])
    return out.view(local, received.shape[0], -1, out.shape[-1]).transpose(0, 1).contiguous()


def layer(hidden, residual, model, k, capacity, ranks, eight_bits=False):
    """(tokens out, residual out, balance loss, counts) of every rank."""
    sent, scales, kept = [], [], []
    for x, r in zip(hidden, residual):
        y, total, q, scale = X.norm(x, model["norm"], r, group=GROUP, quantize=eight_bits)
        logits = (y @ model["router"]).float()
        experts, weights, slots, counts, _, loss, _ = X.route(logits, k, capacity=capacity)
        if eight_bits:
            e = model["router"].shape[1]
            buffer = torch.empty(e, capacity, y.shape[1], dtype=q.dtype, device=q.device)
            sc = torch.empty(e, capacity, scale.shape[1], device=q.device)
            X.dispatch_tensors(q, experts, slots, counts, buffer, scale=scale, out_scale=sc)
            scales.append(sc)
        else:
            buffer = X.dispatch(y, experts, slots, counts, capacity)
        sent.append(buffer)
        kept.append((total, experts, weights, slots, counts, loss))
    received = exchange(sent, ranks)
    if eight_bits:
        received = [rows_in_floats(q, s) for q, s in zip(received, exchange(scales, ranks))]
    done = [experts_of(d, rows, model["experts"]) for d, rows in enumerate(received)]
    out = [X.combine(b, experts, slots, counts, weights)
           for b, (_, experts, weights, slots, counts, _) in zip(back(done, ranks), kept)]
    return (out, [t[0] for t in kept], torch.stack([t[5] for t in kept]).mean(),
            torch.stack([t[4] for t in kept]))


def best_schedule(chunk_bytes, candidates, seed=1):
    """Smallest makespan (us) of `candidates` schedules of the 16-rank Alltoall."""
    plan = Plan.from_workload(replace(named("switch16_a2a"), chunk_bytes=chunk_bytes))
    routes, prio = generate(seed, 0, candidates, plan.route_options(), plan.prio_stride)
    makespan, valid = plan.eval(routes, prio)
    return makespan[valid == 1].min() / 1000


def dropped(counts, capacity):
    """Share of the choices past the capacity."""
    return ((counts - capacity).clamp_min(0).sum() / counts.sum()).item()


def main(tokens=1024, dim=1024, num_experts=64, k=4, steps=30, candidates=2048, ranks=16,
         say=print):
    gen = torch.Generator(device="cuda").manual_seed(0)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    model = {"norm": torch.ones(dim, device="cuda").bfloat16(),
             "router": (randn(dim, num_experts) * (0.5 + randn(num_experts).abs()) / dim ** 0.5)
             .bfloat16().requires_grad_(),
             "experts": (randn(num_experts, dim, dim) / dim ** 0.5).bfloat16()}
    hidden = [randn(tokens, dim).bfloat16() for _ in range(ranks)]
    residual = [randn(tokens, dim).bfloat16() for _ in range(ranks)]
    even = tokens * k // num_experts
    capacity = 2 * even

    with torch.no_grad():
        out, _, _, counts = layer(hidden, residual, model, k, capacity, ranks)
        out8 = layer(hidden, residual, model, k, capacity, ranks, eight_bits=True)[0]
    off = max(((a.float() - b.float()).norm() / b.float().norm()).item() for a, b in zip(out8, out))
    times = {}
    for name, row in (("16-bit rows", 2 * dim), ("8-bit rows", dim + 4 * -(-dim // GROUP))):
        chunk = X.chunk_bytes(num_experts, capacity, row, ranks)
        times[name] = best_schedule(chunk, candidates)
        say(f"{name}: chunks of {chunk} bytes, best of {candidates} schedules "
            f"{times[name]:.1f} us")
    say(f"8-bit rows change the layer's output by {off:.3f} of its length")

    # training steps on the balance loss alone, as one term of a model's loss
    first = dropped(counts, even * 5 // 4)
    for _ in range(steps):
        _, _, loss, counts = layer(hidden, residual, model, k, capacity, ranks)
        loss.backward()
        with torch.no_grad():
            g = model["router"].grad
            model["router"] -= 0.3 * g / g.norm() * dim ** 0.5 / steps ** 0.5
            model["router"].grad = None
    last = dropped(counts, even * 5 // 4)
    chunk = X.chunk_bytes(num_experts, even * 5 // 4, dim + 4 * -(-dim // GROUP), ranks)
    times["evened"] = best_schedule(chunk, candidates)
    say(f"choices past 1.25 times the even load: {first:.3f} before and {last:.3f} after {steps} "
        f"steps; with that capacity {times['evened']:.1f} us")
    return {"times": times, "off": off, "dropped": (first, last)}


if __name__ == "__main__":
    main()
