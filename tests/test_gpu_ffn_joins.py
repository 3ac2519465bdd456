"""Tiles that several blocks share: in the sizes of eight wavefronts (128 x 256
and 256 x 256), for every product of the feed-forward and its gradient, and in
smaller ones for odd rows and 32 bits.

Which tiles are shared is read from the workspace that a call leaves: how many
parts of each came (the counters), and how far the parts' sums reach, which
tells the tiles' size. So a case that a change of the rules empties fails.
"""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
SOURCES = pytest.mark.parametrize("sources", [1, 4])

UP, DOWN = 0, 1                       # counters of the forward's products
GRAD, DX, DW_IN, DW_OUT = 0, 1, 2, 3  # and of the gradient's
SMALL, MEDIUM, WIDE, LARGE = (4 * n for n in (64 * 64, 128 * 128, 128 * 256, 256 * 256))
# (bytes of a tile's sums)
COUNTERS = 1024                       # of a product

# rows of an expert in the buffer, columns, hidden columns, rows below the
# counts; {product: (tiles shared, parts)} and the bytes of sums, of the forward
# and the gradient
ROWS = (4864, 2304, 2304, (4864, 4700, 4864),
        {UP: (2, 4), DOWN: (1, 4)}, 8 * LARGE, {GRAD: (1, 4), DX: (1, 4)}, 4 * LARGE)
WEIGHTS = (4096, 11008, 768, (1500,),
           {}, 0, {DX: (2, 3), DW_IN: (2, 4), DW_OUT: (2, 4)}, 8 * LARGE)
CASES = [ROWS, WEIGHTS,
         (1600, 3328, 1600, (1600, 896),
          {UP: (4, 4), DOWN: (4, 3)}, 16 * WIDE, {DX: (4, 4)}, 16 * WIDE),
         (1600, 1600, 3328, (1600, 896),
          {UP: (30, 3)}, 90 * LARGE, {GRAD: (4, 3)}, 12 * WIDE)]
# with the least workspace, and the bytes that it has for sums
LEAST = [ROWS[:4] + ({UP: (2, 3), DOWN: (1, 4)}, 6 * LARGE, ROWS[6], ROWS[7]),
         WEIGHTS[:6] + ({DX: (2, 2), DW_IN: (2, 2), DW_OUT: (2, 4)}, 4 * LARGE)]
# through registers (any 16-bit type), and in 32 bits
ODD = (5504, 2049, 321, (5504, 5504),
       {UP: (4, 2)}, 8 * MEDIUM, {DW_OUT: (102, 5)}, 510 * MEDIUM)
WORDS = (13184, 800, 320, (13184,),
         {UP: (3, 3)}, 9 * MEDIUM, {GRAD: (6, 3), DW_IN: (130, 3), DW_OUT: (65, 7)}, 845 * SMALL)


def make(dtype, sources, slots, d, f, rows, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    e, c = len(rows), slots // sources
    counts = torch.zeros(sources, e, dtype=torch.int32)
    for j, n in enumerate(rows):  # uneven over the sources, one without rows if they allow
        for i in reversed(range(sources)):
            counts[i, j] = min(c, n)
            n -= min(c, n)
        assert n == 0
    counts = counts.cuda()
    past = torch.arange(c, device="cuda") >= counts[..., None]

    def filled(n):
        x = randn(sources, e, c, n).to(dtype)
        x[past] = float("nan")
        return x

    return {"counts": counts, "past": past, "buffer": filled(d), "dout": filled(d),
            "pre": filled(2 * f), "w_in": (randn(e, 2 * f, d) / d ** 0.5).to(dtype),
            "w_out": (randn(e, d, f) / f ** 0.5).to(dtype)}


def workspace(m, backward, least):
    """Bytes 0x5A that a call may write and 256 behind them; where the counters
    and the sums begin."""
    shape, f = m["buffer"].shape, m["w_out"].shape[2]
    rows = shape[0] * shape[1] * shape[2]

    def room(base, per_row):
        return -(-min(64 << 20, base + per_row * rows) // 256) * 256

    n = X.ffn_workspace(shape, f, m["buffer"].dtype, backward)
    sums = n - room(3 << 19, 8192)
    if least:
        n = sums + room(3 << 18, 64)
    return torch.full((n + 256,), 0x5A, dtype=torch.uint8, device="cuda"), n, sums


def shared(work, n, sums):
    """{product: (tiles, parts)}, bytes of sums."""
    assert (work[n:] == 0x5A).all()
    done = work[sums - 4 * 4 * COUNTERS:sums].view(torch.int32).view(4, COUNTERS).cpu()
    got = {}
    for i, counters in enumerate(done):
        came = counters[counters != 0]
        if len(came):
            assert (came == came[0]).all() and (counters[:len(came)] != 0).all()
            got[i] = (len(came), int(came[0]))
    written = torch.nonzero(work[sums:n].view(torch.int32) != 0x5A5A5A5A)
    return got, 4 * (int(written.max()) + 1) if len(written) else 0


def forward(m, least=False):
    out, pre = torch.full_like(m["buffer"], float("nan")), torch.full_like(m["pre"], 7.0)
    work, n, sums = workspace(m, False, least)
    X.ffn_tensors(m["buffer"], m["counts"], m["w_in"], m["w_out"], out, work[:n], pre=pre)
    return [out, pre], shared(work, n, sums)


def backward(m, least=False):
    got = {n: torch.full_like(m[k], float("nan"))
           for n, k in (("dbuffer", "buffer"), ("dw_in", "w_in"), ("dw_out", "w_out"))}
    work, n, sums = workspace(m, True, least)
    X.ffn_backward_tensors(m["dout"], m["buffer"], m["counts"], m["w_in"], m["w_out"], m["pre"],
                           work[:n], **got)
    return list(got.values()), shared(work, n, sums)


def check(m, dtype, case, least=False):
    there, past = ~m["past"].cpu(), m["past"]
    (out, pre), seen = forward(m, least)
    assert seen == case[4:6]
    want, slack, want_pre, pre_slack = F.ffn(m["buffer"], m["counts"], m["w_in"], m["w_out"],
                                             "cuda")
    F.close(out, want, dtype, slack)
    F.close(pre.cpu()[there], want_pre[there], dtype, pre_slack[there])
    assert not out[past].any() and (pre[past] == 7).all()
    got, seen = backward(m, least)
    assert seen == case[6:8]
    for g, (w, slack) in zip(got, F.ffn_backward(m["dout"], m["buffer"], m["counts"], m["w_in"],
                                                 m["w_out"], m["pre"], "cuda")):
        F.close(g, w, dtype, slack)
    assert not got[0][past].any()
    # the same bits whichever part comes last
    first = [out, pre, *got]
    for _ in range(2):
        for a, b in zip(first, forward(m, least)[0] + backward(m, least)[0]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@TYPES
@SOURCES
@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c[:3]))
def test_joins(dtype, sources, case):
    check(make(dtype, sources, *case[:4], seed=1), dtype, case)


@SOURCES
@pytest.mark.parametrize("dtype,case", [(torch.bfloat16, ODD), (torch.float16, ODD),
                                        (torch.float32, WORDS)], ids=["bf16", "f16", "f32"])
def test_joins_of_smaller_tiles(dtype, case, sources):
    check(make(dtype, sources, *case[:4], seed=3), dtype, case)


@TYPES
@SOURCES
@pytest.mark.parametrize("case", LEAST, ids=lambda c: str(c[:3]))
def test_joins_in_the_least_workspace(dtype, sources, case):
    """Nothing is written behind it; of the second case the sums fill it."""
    m = make(dtype, sources, *case[:4], seed=2)
    check(m, dtype, case, least=True)
    if case[0] == WEIGHTS[0]:
        work, n, sums = workspace(m, True, True)
        assert n - sums == case[7]
