"""Entry points of the experts' operators without a GPU: layout of the argument
structs, sizes and the refusals that come before any device work."""
import ctypes as ct
import os
import subprocess

import pytest
import torch

from paper_2111_04867_amd import binding as B
from paper_2111_04867_amd import experts as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_P, _I32, _I64, _F64 = ct.c_void_p, ct.c_int32, ct.c_int64, ct.c_double


def _struct(name, fields):
    return type(name, (ct.Structure,), {"_fields_": fields})


_SIZES = [("capacity", _I64), ("sources", _I32), ("num_experts", _I32), ("cols", _I32),
          ("hidden", _I32), ("dtype", _I32)]
_Ffn = _struct("_Ffn", _SIZES + [
    ("buffer", _P), ("counts", _P), ("w_in", _P), ("w_out", _P), ("out", _P), ("pre", _P),
    ("workspace", _P), ("workspace_bytes", _I64)])
_FfnBackward = _struct("_FfnBackward", _SIZES + [
    ("dout", _P), ("buffer", _P), ("counts", _P), ("w_in", _P), ("w_out", _P), ("pre", _P),
    ("dbuffer", _P), ("dw_in", _P), ("dw_out", _P), ("workspace", _P), ("workspace_bytes", _I64)])
_FfnTokens = _struct("_FfnTokens", [
    ("tokens", _I64), ("cols", _I32), ("hidden", _I32), ("num_experts", _I32), ("k", _I32),
    ("first_expert", _I32), ("local_experts", _I32), ("dtype", _I32), ("logits_dtype", _I32),
    ("renorm", _I32), ("x", _P), ("x_stride", _I64), ("logits", _P), ("logits_stride", _I64),
    ("mask", _P), ("w_in", _P), ("w_out", _P), ("out", _P), ("out_stride", _I64), ("experts", _P),
    ("weights", _P), ("workspace", _P), ("workspace_bytes", _I64)])
_Dropout = _struct("_Dropout", [
    ("rows", _I64), ("cols", _I32), ("dtype", _I32), ("p", _F64), ("x", _P), ("residual", _P),
    ("x_stride", _I64), ("residual_stride", _I64), ("rng", _P), ("out", _P), ("out_stride", _I64)])
STRUCTS = {"taccl_ffn_t": _Ffn, "taccl_ffn_backward_t": _FfnBackward,
           "taccl_ffn_tokens_t": _FfnTokens, "taccl_dropout_t": _Dropout}


def test_structs_match_the_header(tmp_path):
    lines = []
    for name, cls in STRUCTS.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for f, _ in cls._fields_:
            lines.append(f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "taccl.h"\n'
                   "int main(void) {" + "\n".join(lines) + " return 0; }")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = dict(line.rsplit(" ", 1) for line in
               subprocess.run([str(exe)], capture_output=True, text=True).stdout.splitlines())
    for name, cls in STRUCTS.items():
        assert int(got[name]) == ct.sizeof(cls), name
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


def status(name, args):
    fn = getattr(B.lib(), name)
    fn.argtypes, fn.restype = [ct.c_void_p, ct.c_void_p], ct.c_int
    st = fn(None if args is None else ct.addressof(args), None)
    return st, B.lib().taccl_last_error().decode()


INVALID, LIMIT = B.ERR_INVALID_ARGUMENT, B.ERR_LIMIT
_FFN = dict(capacity=10, sources=2, num_experts=4, cols=64, hidden=32, dtype=1, buffer=4096,
            counts=4096, w_in=4096, w_out=4096, workspace=4096, workspace_bytes=1 << 30)
GOOD = {
    "taccl_ffn": dict(_FFN, out=4096, pre=4096),
    "taccl_ffn_backward": dict(_FFN, dout=4096, pre=4096, dbuffer=4096, dw_in=4096, dw_out=4096),
    "taccl_ffn_tokens": dict(tokens=4, cols=64, hidden=32, num_experts=8, k=2, first_expert=0,
                             local_experts=8, dtype=1, logits_dtype=0, x=4096, x_stride=64,
                             logits=4096, logits_stride=8, w_in=4096, w_out=4096, out=4096,
                             out_stride=64, experts=4096, weights=4096, workspace=4096,
                             workspace_bytes=1 << 30),
    "taccl_dropout": dict(rows=4, cols=64, dtype=1, p=0.5, x=4096, x_stride=64, rng=4096, out=4096,
                          out_stride=64),
}
BAD = [(n, c, w) for n in ("taccl_ffn", "taccl_ffn_backward") for c, w in [
    (dict(capacity=0), INVALID), (dict(capacity=-3), INVALID), (dict(capacity=1 << 21), LIMIT),
    (dict(capacity=1 << 62), LIMIT), (dict(sources=0), INVALID), (dict(sources=1025), LIMIT),
    (dict(num_experts=0), INVALID), (dict(num_experts=1025), LIMIT),
    (dict(num_experts=1024, capacity=1 << 20), LIMIT),
    (dict(cols=0), INVALID), (dict(hidden=0), INVALID), (dict(cols=65537), LIMIT),
    (dict(hidden=65537), LIMIT), (dict(cols=65536, hidden=65536, num_experts=64), LIMIT),
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(buffer=None), INVALID),
    (dict(buffer=4097), INVALID), (dict(counts=4098), INVALID), (dict(w_in=None), INVALID),
    (dict(w_out=4099), INVALID), (dict(pre=4097), INVALID), (dict(workspace=None), INVALID),
    (dict(workspace=4104), INVALID), (dict(workspace_bytes=100), INVALID)]]
BAD += [
    ("taccl_ffn", dict(out=None), INVALID), ("taccl_ffn", dict(out=4097), INVALID),
    ("taccl_ffn_backward", dict(dout=None), INVALID),
    ("taccl_ffn_backward", dict(pre=None), INVALID),
    ("taccl_ffn_backward", dict(dbuffer=None, dw_in=None, dw_out=None), INVALID),
    ("taccl_ffn_backward", dict(dw_in=4097), INVALID),
    ("taccl_ffn_tokens", dict(tokens=-1), INVALID), ("taccl_ffn_tokens", dict(tokens=65), LIMIT),
    ("taccl_ffn_tokens", dict(k=0), INVALID), ("taccl_ffn_tokens", dict(k=9), INVALID),
    ("taccl_ffn_tokens", dict(num_experts=64, logits_stride=64, k=17), LIMIT),
    ("taccl_ffn_tokens", dict(num_experts=1025, logits_stride=1025), LIMIT),
    ("taccl_ffn_tokens", dict(local_experts=0), INVALID),
    ("taccl_ffn_tokens", dict(first_expert=-1, local_experts=2), INVALID),
    ("taccl_ffn_tokens", dict(first_expert=1), INVALID),
    ("taccl_ffn_tokens", dict(first_expert=2147483647, local_experts=8), INVALID),
    ("taccl_ffn_tokens", dict(cols=0), INVALID), ("taccl_ffn_tokens", dict(hidden=70000), LIMIT),
    ("taccl_ffn_tokens", dict(dtype=4), INVALID),
    ("taccl_ffn_tokens", dict(logits_dtype=-1), INVALID),
    ("taccl_ffn_tokens", dict(x_stride=63), INVALID),
    ("taccl_ffn_tokens", dict(logits_stride=7), INVALID),
    ("taccl_ffn_tokens", dict(out_stride=0), INVALID), ("taccl_ffn_tokens", dict(x=None), INVALID),
    ("taccl_ffn_tokens", dict(logits=4098), INVALID),
    ("taccl_ffn_tokens", dict(weights=4097), INVALID),
    ("taccl_ffn_tokens", dict(workspace_bytes=64), INVALID),
    ("taccl_dropout", dict(rows=-1), INVALID), ("taccl_dropout", dict(rows=1 << 22), LIMIT),
    ("taccl_dropout", dict(cols=0), INVALID), ("taccl_dropout", dict(cols=(1 << 20) + 1), LIMIT),
    ("taccl_dropout", dict(p=-0.1), INVALID), ("taccl_dropout", dict(p=1.0001), INVALID),
    ("taccl_dropout", dict(p=float("nan")), INVALID), ("taccl_dropout", dict(dtype=3), INVALID),
    ("taccl_dropout", dict(rng=4100), INVALID), ("taccl_dropout", dict(rng=None), INVALID),
    ("taccl_dropout", dict(residual=4096), INVALID), ("taccl_dropout", dict(x=4097), INVALID),
    ("taccl_dropout", dict(out_stride=63), INVALID),
]


@pytest.mark.parametrize("name,change,want", BAD, ids=[f"{n}-{c}" for n, c, _ in BAD])
def test_refusals(name, change, want):
    st, message = status(name, STRUCTS[name + "_t"](**{**GOOD[name], **change}))
    assert st == want, (st, message)
    assert message.startswith(name + ":")


@pytest.mark.parametrize("name", GOOD)
def test_null_arguments(name):
    assert status(name, None) == (INVALID, name + ": null arguments")


def test_nothing_to_do():
    """No rows: success without a device."""
    assert status("taccl_dropout", _Dropout(rows=0, cols=4, p=0.5))[0] == B.OK
    assert status("taccl_ffn_tokens", _FfnTokens(tokens=0, cols=4, hidden=4, num_experts=4, k=1,
                                                 local_experts=4))[0] == B.OK


def test_workspace_sizes():
    shape, f = (4, 100, 64), 32
    size = X.ffn_workspace(shape, f, torch.bfloat16)
    assert size >= 400 * f * 2 and size % 256 == 0
    assert X.ffn_workspace((2, *shape), f, torch.bfloat16) >= 2 * 400 * f * 2 + 4 * 800
    assert X.ffn_workspace(shape, f, torch.bfloat16, True) >= size + 400 * 2 * f * 2
    assert X.ffn_workspace(shape, f, torch.float32) >= 400 * f * 4
    for bad in ((0, 10, 8), (4, 0, 8), (4, 1 << 40, 8), (1 << 40, 4, 8), (2000, 4, 4, 8)):
        assert X.ffn_workspace(bad, f, torch.bfloat16) == 0
    assert X.ffn_workspace(shape, f, torch.float64) == 0
    assert X.ffn_workspace(shape, 0, torch.float32) == 0
    assert X.ffn_tokens_workspace(16, 4, 64, 32) >= 16 * 4 * 32 * 4
    for bad in ((65, 1, 8, 8), (-1, 1, 8, 8), (1, 0, 8, 8), (1, 17, 8, 8), (1, 1, 0, 8),
                (1, 1, 8, 1 << 40)):
        assert X.ffn_tokens_workspace(*bad) == 0
    assert X.dropout_words(3, 5) == 9 and X.dropout_words(0, 8) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x, w = torch.zeros(2, 4, 8), torch.zeros(2, 8, 6)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA tensor"):
        X.ffn_tensors(x, i, torch.zeros(2, 12, 8), w, x, x)
    with pytest.raises(ValueError, match="CUDA tensor"):
        X.ffn_backward_tensors(x, x, i, w, w, x, x)
    with pytest.raises(ValueError, match="buffer must be a CUDA tensor"):
        X.ffn_tensors(None, i, w, w, x, x)
    with pytest.raises(ValueError, match="matrix"):
        X.ffn_tokens_tensors(x, x, w, w, x, x, k=1)
    with pytest.raises(ValueError, match="CUDA"):
        X.ffn_tokens_tensors(x[0], x[0], w, w, x[0], x, k=1)
    with pytest.raises(ValueError, match="CUDA"):
        X.dropout_tensors(x[0], torch.zeros(2, dtype=torch.int64), x[0], p=0.5)
    with pytest.raises(TypeError, match="takes 6 arguments"):
        X._calls.dropout(x)
