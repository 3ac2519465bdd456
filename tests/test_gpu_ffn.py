"""The experts' feed-forward and its gradient against the 64-bit form.

The slack of every result is worked out with the form (expert_forms.py); rows
past the counts hold NaN on the way in, so a result that took one in is NaN.
"""
import pytest
import torch

import expert_forms as F
from paper_2111_04867_amd import experts as X

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", F.TYPES.values(), ids=F.TYPES)

# sources, experts, capacity, dim, hidden: single values, sizes that are no whole
# 16 bytes, tiles that end inside, more than one step and tile
CASES = [(1, 1, 1, 1, 1), (1, 2, 5, 8, 8), (1, 3, 70, 64, 40), (2, 4, 33, 72, 136),
         (3, 5, 40, 111, 77), (1, 2, 300, 256, 128), (16, 4, 9, 128, 64), (1, 1, 129, 520, 264),
         (1, 2, 60, 1111, 515), (5, 1, 64, 200, 330)]
# enough tiles for the large ones
LARGE = [(1, 130, 260, 264, 136), (2, 128, 140, 512, 264)]


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


def check_forward(m, dtype):
    out, pre = forward(m)
    want, slack, want_pre, pre_slack = F.ffn(m["buffer"], m["counts"], m["w_in"], m["w_out"])
    F.close(out, want, dtype, slack)
    past = m["past"].cpu()
    assert (out.cpu()[past] == 0).all() and (pre.cpu()[past] == 7).all()
    F.close(pre.cpu()[~past], want_pre[~past], dtype, pre_slack[~past])


def check_backward(m, dtype):
    got = backward(m)
    want = F.ffn_backward(m["dout"], m["buffer"], m["counts"], m["w_in"], m["w_out"], m["pre"])
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("case", LARGE, ids=str)
def test_large_tiles(dtype, case):
    m = make(dtype, *case, seed=2)
    check_forward(m, dtype)
    check_backward(m, dtype)
