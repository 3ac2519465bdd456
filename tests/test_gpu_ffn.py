"""The experts' feed-forward and its gradient against the 64-bit form.

The slack of every result is worked out with the form (expert_forms.py); rows
past the counts hold NaN on the way in, so a result that took one in is NaN.
"""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X
from paper_2111_04867_amd.binding import TacclError

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)

# sources, experts, capacity, dim, hidden: single values, sizes that are no whole
# 16 bytes, tiles that end inside, more than one step and tile
CASES = [(1, 1, 1, 1, 1), (1, 2, 5, 8, 8), (1, 3, 70, 64, 40), (2, 4, 33, 72, 136),
         (3, 5, 40, 111, 77), (1, 2, 300, 256, 128), (16, 4, 9, 128, 64), (1, 1, 129, 520, 264),
         (1, 2, 60, 1111, 515), (5, 1, 64, 200, 330)]
# few tiles with many steps, which blocks share: along the dim, along the rows
LONG = [(1, 2, 40, 4104, 32), (3, 2, 13, 4101, 33), (1, 1, 3000, 64, 32), (8, 1, 400, 41, 23),
        (2, 3, 1100, 40, 24)]
# enough tiles for the larger ones, whole chunks or not, rows of one source or more
LARGE = [(1, 130, 260, 264, 136), (2, 128, 140, 512, 264), (4, 16, 300, 1032, 520),
         (2, 16, 256, 1024, 512), (1, 24, 300, 777, 333), (1, 20, 512, 1024, 512),
         (2, 8, 300, 1024, 510)]
# a last turn of few tiles, which blocks share; so, in 32 bits, and by registers
LAST = [(1, 4, 1100, 1032, 1024), (2, 8, 310, 2048, 512), (1, 6, 700, 2049, 255),
        (3, 7, 150, 1025, 1023)]


def make(dtype, s, e, c, d, f, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    counts = torch.randint(0, c + c // 3 + 2, (s, e), generator=gen, device="cuda").int()
    flat = counts.view(-1)
    if len(flat) > 1:
        flat[1] = 0
    if len(flat) > 2:
        flat[2] = -5
        flat[0] = c
    past = torch.arange(c, device="cuda") >= counts[..., None]

    def rows(n):
        x = randn(s, e, c, n).to(dtype)
        x[past] = float("nan")
        return x

    return {"counts": counts, "past": past, "buffer": rows(d), "dout": rows(d), "pre": rows(2 * f),
            "w_in": (randn(e, 2 * f, d) / d ** 0.5).to(dtype),
            "w_out": (randn(e, d, f) / f ** 0.5).to(dtype)}


def workspace(m, backward):
    f = m["w_out"].shape[2]
    n = X.ffn_workspace(m["buffer"].shape, f, m["buffer"].dtype, backward)
    # the bytes behind it have to stay as they are
    return torch.full((n + 256,), 0x5A, dtype=torch.uint8, device="cuda"), n


def forward(m):
    out = torch.full_like(m["buffer"], float("nan"))
    pre = torch.full_like(m["pre"], 7.0)
    work, n = workspace(m, False)
    X.ffn_tensors(m["buffer"], m["counts"], m["w_in"], m["w_out"], out, work[:n], pre=pre)
    assert (work[n:] == 0x5A).all()
    return out, pre


def backward(m, *, only=None):
    got = {n: torch.full_like(m[k], float("nan"))
           for n, k in (("dbuffer", "buffer"), ("dw_in", "w_in"), ("dw_out", "w_out"))
           if only is None or n == only}
    work, n = workspace(m, True)
    X.ffn_backward_tensors(m["dout"], m["buffer"], m["counts"], m["w_in"], m["w_out"], m["pre"],
                           work[:n], **got)
    assert (work[n:] == 0x5A).all()
    return got


def check_forward(m, dtype, device="cpu"):
    out, pre = forward(m)
    want, slack, want_pre, pre_slack = F.ffn(m["buffer"], m["counts"], m["w_in"], m["w_out"], device)
    F.close(out, want, dtype, slack)
    past = m["past"].cpu()
    assert (out.cpu()[past] == 0).all() and (pre.cpu()[past] == 7).all()
    F.close(pre.cpu()[~past], want_pre[~past], dtype, pre_slack[~past])


def check_backward(m, dtype, device="cpu"):
    got = backward(m)
    want = F.ffn_backward(m["dout"], m["buffer"], m["counts"], m["w_in"], m["w_out"], m["pre"],
                          device)
    for name, (w, slack) in zip(("dbuffer", "dw_in", "dw_out"), want):
        F.close(got[name], w, dtype, slack)
    assert (got["dbuffer"].cpu()[m["past"].cpu()] == 0).all()


@TYPES
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(dtype, case):
    check_forward(make(dtype, *case), dtype)


@TYPES
@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(dtype, case):
    check_backward(make(dtype, *case, seed=1), dtype)


@TYPES
@pytest.mark.parametrize("case", LONG, ids=str)
def test_shared_steps(dtype, case):
    """The same bits whichever part comes last."""
    m = make(dtype, *case, seed=3)
    check_forward(m, dtype)
    check_backward(m, dtype)
    first = [*forward(m), *backward(m).values()]
    for _ in range(3):
        for a, b in zip(first, [*forward(m), *backward(m).values()]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@TYPES
@pytest.mark.parametrize("case", LARGE, ids=str)
def test_large_tiles(dtype, case):
    m = make(dtype, *case, seed=2)
    check_forward(m, dtype, "cuda")
    check_backward(m, dtype, "cuda")


@TYPES
@pytest.mark.parametrize("case", LAST, ids=str)
def test_shared_last_tiles(dtype, case):
    m = make(dtype, *case, seed=4)
    check_forward(m, dtype, "cuda")
    check_backward(m, dtype, "cuda")
    first = [*forward(m), *backward(m).values()]
    for a, b in zip(first, [*forward(m), *backward(m).values()]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@TYPES
@pytest.mark.parametrize("case", [LONG[1], LAST[0], LAST[1]], ids=str)
def test_the_least_workspace(dtype, case, monkeypatch):
    """Of the sums' bytes the least that is taken: nothing is written behind it."""
    m = make(dtype, *case, seed=5)
    rows, full = case[0] * case[1] * case[2], X.ffn_workspace
    less = min(64 << 20, (3 << 19) + 8192 * rows) - min(64 << 20, (3 << 18) + 64 * rows)
    # both are rounded up to 256
    monkeypatch.setattr(X, "ffn_workspace", lambda *a: full(*a) - (less - 256) // 256 * 256)
    check_forward(m, dtype, "cuda")
    check_backward(m, dtype, "cuda")
    monkeypatch.setattr(X, "ffn_workspace", lambda *a: full(*a) - less - 512)
    with pytest.raises(TacclError, match="workspace too small"):
        forward(m)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_misaligned_arrays(dtype):
    """Sizes in whole chunks, arrays an element off."""
    m = make(dtype, 2, 3, 40, 64, 48, seed=4)

    def off(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:]
        return flat.copy_(t.reshape(-1)).view(t.shape)

    want = [*forward(m), *backward(m).values()]
    for name in ("buffer", "dout", "pre", "w_in", "w_out"):
        m[name] = off(m[name])
    out, pre = off(m["buffer"]), torch.full_like(m["pre"], 7.0)
    work, n = workspace(m, False)
    X.ffn_tensors(m["buffer"], m["counts"], m["w_in"], m["w_out"], out, work[:n], pre=pre)
    # the same products in the same order of steps
    for a, b in zip([out, pre, *backward(m).values()], want):
        assert torch.allclose(a.float(), b.float(), rtol=2 * F.ROUND[dtype][0], atol=1e-3)


@TYPES
def test_out_in_place(dtype):
    m = make(dtype, 2, 3, 50, 72, 40, seed=5)
    want, _ = forward(m)
    work, n = workspace(m, False)
    X.ffn_tensors(m["buffer"], m["counts"], m["w_in"], m["w_out"], m["buffer"], work[:n])
    assert torch.equal(m["buffer"], want)


@pytest.mark.parametrize("name", ["dbuffer", "dw_in", "dw_out"])
@pytest.mark.parametrize("case", [(2, 3, 50, 72, 40), (4, 16, 300, 1032, 520)], ids=str)
def test_one_gradient_alone(name, case):
    m = make(torch.bfloat16, *case, seed=6)
    whole = backward(m)
    assert torch.equal(backward(m, only=name)[name], whole[name])


def test_no_rows():
    """All counts zero: zeros, and nothing is read."""
    m = make(torch.bfloat16, 2, 3, 30, 64, 32, seed=7)
    m["counts"].zero_()
    for n in ("buffer", "dout", "pre"):
        m[n].fill_(float("nan"))
    out, pre = forward(m)
    assert (out == 0).all() and (pre == 7).all()
    for g in backward(m).values():
        assert (g == 0).all()


def test_infinities_stay_in_their_rows():
    """A row of infinities or NaN reaches its own results and the weights'
    gradients, not other rows."""
    m = make(torch.float32, 1, 2, 70, 64, 32, seed=8)
    m["counts"][:] = torch.tensor([70, 40])
    for n in ("buffer", "dout", "pre"):
        m[n].copy_(torch.randn(m[n].shape, device="cuda"))
    want, want_back = forward(m)[0], backward(m)["dbuffer"]
    for n in ("buffer", "dout", "pre"):
        m[n][0, 0, 3] = float("inf")
        m[n][0, 1, 5, 2] = float("nan")
    got, back = forward(m)[0], backward(m)["dbuffer"]
    rows = torch.ones(1, 2, 70, dtype=torch.bool, device="cuda")
    rows[0, 0, 3] = rows[0, 1, 5] = False
    for a, b in ((got, want), (back, want_back)):
        assert torch.equal(a[rows], b[rows])
        assert a[0, 0, 3].isnan().any() and a[0, 1, 5].isnan().any()


def test_offsets_past_32_bits():
    """Rows that lie more than 2^32 bytes into the buffer, read and zeroed."""
    s, e, c, d, f = 2, 2, 80000, 8192, 32
    gen = torch.Generator(device="cuda").manual_seed(9)
    buffer = torch.zeros(s, e, c, d, dtype=torch.float16, device="cuda")
    counts = torch.tensor([[3, 1], [0, 70]], dtype=torch.int32, device="cuda")
    for i in range(s):
        for j in range(e):
            n = int(counts[i, j])
            buffer[i, j, :n] = torch.randn(n, d, generator=gen, device="cuda").half()
    w_in = (torch.randn(e, 2 * f, d, generator=gen, device="cuda") / 90).half()
    w_out = (torch.randn(e, d, f, generator=gen, device="cuda") / 6).half()
    out = torch.full_like(buffer, 9.0)
    work = torch.empty(X.ffn_workspace(buffer.shape, f, buffer.dtype), dtype=torch.uint8,
                       device="cuda")
    X.ffn_tensors(buffer, counts, w_in, w_out, out, work)
    small = F.ffn(buffer[:, :, :70], counts, w_in, w_out)
    F.close(out[:, :, :70], small[0], torch.float16, small[1])
    assert not out[:, :, 70:].any()
