"""Expert-layer entry points without a GPU: the argument structs' layout, sizes
and the refusals that come before any device work."""
import ctypes as ct
import os
import re
import subprocess

import pytest
import torch

from paper_2111_04867_amd import binding as B
from paper_2111_04867_amd import experts as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_P, _I32, _I64, _F32 = ct.c_void_p, ct.c_int32, ct.c_int64, ct.c_float


def _struct(name, fields):
    return type(name, (ct.Structure,), {"_fields_": fields})


# the argument structs of include/taccl.h, in their order
_Norm = _struct("_Norm", [
    ("rows", _I64), ("cols", _I32), ("dtype", _I32), ("eps", _F32), ("group", _I32), ("x", _P),
    ("residual", _P), ("x_stride", _I64), ("residual_stride", _I64), ("weight", _P), ("out", _P),
    ("total", _P), ("out_stride", _I64), ("total_stride", _I64), ("q", _P), ("scale", _P),
    ("q_stride", _I64), ("scale_stride", _I64)])
_NormBackward = _struct("_NormBackward", [
    ("rows", _I64), ("cols", _I32), ("dtype", _I32), ("eps", _F32), ("dout", _P), ("h", _P),
    ("dtotal", _P), ("dout_stride", _I64), ("h_stride", _I64), ("dtotal_stride", _I64),
    ("weight", _P), ("dx", _P), ("dx_stride", _I64), ("dweight", _P), ("workspace", _P),
    ("workspace_bytes", _I64)])
_Route = _struct("_Route", [
    ("tokens", _I64), ("num_experts", _I32), ("k", _I32), ("dtype", _I32), ("renorm", _I32),
    ("coef", _F32), ("capacity", _I64), ("logits", _P), ("logits_stride", _I64), ("mask", _P),
    ("experts", _P), ("weights", _P), ("slots", _P), ("counts", _P), ("prob_sums", _P),
    ("loss", _P), ("rows", _P), ("workspace", _P), ("workspace_bytes", _I64)])
_RouteBackward = _struct("_RouteBackward", [
    ("tokens", _I64), ("num_experts", _I32), ("k", _I32), ("dtype", _I32), ("renorm", _I32),
    ("coef", _F32), ("logits", _P), ("logits_stride", _I64), ("mask", _P), ("experts", _P),
    ("counts", _P), ("rows", _P), ("dweights", _P), ("dloss", _P), ("dlogits", _P),
    ("dlogits_stride", _I64)])
_Dispatch = _struct("_Dispatch", [
    ("tokens", _I64), ("capacity", _I64), ("num_experts", _I32), ("k", _I32), ("cols", _I32),
    ("element_bytes", _I32), ("scale_cols", _I32), ("x", _P), ("x_stride", _I64), ("scale", _P),
    ("scale_stride", _I64), ("experts", _P), ("slots", _P), ("counts", _P), ("out", _P),
    ("out_scale", _P)])
_Combine = _struct("_Combine", [
    ("tokens", _I64), ("capacity", _I64), ("num_experts", _I32), ("k", _I32), ("cols", _I32),
    ("dtype", _I32), ("buffer", _P), ("experts", _P), ("slots", _P), ("weights", _P), ("out", _P),
    ("out_stride", _I64)])
_CombineBackward = _struct("_CombineBackward", [
    ("tokens", _I64), ("capacity", _I64), ("num_experts", _I32), ("k", _I32), ("cols", _I32),
    ("dtype", _I32), ("dout", _P), ("dout_stride", _I64), ("buffer", _P), ("experts", _P),
    ("slots", _P), ("counts", _P), ("weights", _P), ("dbuffer", _P), ("dweights", _P)])


STRUCTS = {"taccl_norm_t": _Norm, "taccl_norm_backward_t": _NormBackward,
           "taccl_route_t": _Route, "taccl_route_backward_t": _RouteBackward,
           "taccl_dispatch_t": _Dispatch, "taccl_combine_t": _Combine,
           "taccl_combine_backward_t": _CombineBackward}


def test_structs_match_the_header(tmp_path):
    """Every field of the structs above lies where a C compiler puts it."""
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


def test_workspace_sizes():
    assert X.norm_workspace(100) == 4096 * 100 and X.norm_workspace(0) == 0
    assert X.route_workspace(64) == 4 * 256 * 129 and X.route_workspace(-1) == 0


def status(name, args):
    fn = getattr(B.lib(), name)
    fn.argtypes, fn.restype = [ct.c_void_p, ct.c_void_p], ct.c_int
    st = fn(None if args is None else ct.addressof(args), None)
    return st, B.lib().taccl_last_error().decode()


INVALID, LIMIT = B.ERR_INVALID_ARGUMENT, B.ERR_LIMIT
# arguments that pass every check, by name (pointers that nothing reads)
GOOD = {
    "taccl_norm": dict(rows=4, cols=64, dtype=1, eps=1e-6, group=64, x=4096, x_stride=64,
                       weight=4096, out=4096, out_stride=64, q=4096, scale=4096, q_stride=64,
                       scale_stride=1),
    "taccl_norm_backward": dict(rows=4, cols=64, dtype=0, eps=1e-6, dout=4096, h=4096,
                                dout_stride=64, h_stride=64, weight=4096, dx=4096, dx_stride=64,
                                dweight=4096, workspace=4096, workspace_bytes=4096 * 64),
    "taccl_route": dict(tokens=4, num_experts=8, k=2, dtype=0, logits=4096, logits_stride=8,
                        experts=4096, weights=4096, slots=4096, counts=4096, prob_sums=4096,
                        loss=4096, rows=4096, workspace=4096, workspace_bytes=1 << 20),
    "taccl_route_backward": dict(tokens=4, num_experts=8, k=2, dtype=0, logits=4096,
                                 logits_stride=8, experts=4096, counts=4096, rows=4096,
                                 dlogits=4096, dlogits_stride=8),
    "taccl_dispatch": dict(tokens=4, capacity=3, num_experts=8, k=2, cols=64, element_bytes=2,
                           x=4096, x_stride=64, experts=4096, slots=4096, counts=4096, out=4096),
    "taccl_combine": dict(tokens=4, capacity=3, num_experts=8, k=2, cols=64, dtype=1, buffer=4096,
                          experts=4096, slots=4096, out=4096, out_stride=64),
    "taccl_combine_backward": dict(tokens=4, capacity=3, num_experts=8, k=2, cols=64, dtype=1,
                                   dout=4096, dout_stride=64, buffer=4096, experts=4096,
                                   slots=4096, counts=4096, weights=4096, dbuffer=4096,
                                   dweights=4096),
}
BAD = [
    ("taccl_norm", dict(rows=-1), INVALID), ("taccl_norm", dict(rows=(1 << 21) + 1), LIMIT),
    ("taccl_norm", dict(cols=0), INVALID), ("taccl_norm", dict(cols=16385), LIMIT),
    ("taccl_norm", dict(dtype=3), INVALID), ("taccl_norm", dict(dtype=-1), INVALID),
    ("taccl_norm", dict(eps=-1.0), INVALID), ("taccl_norm", dict(eps=float("nan")), INVALID),
    ("taccl_norm", dict(group=48), INVALID), ("taccl_norm", dict(group=512), INVALID),
    ("taccl_norm", dict(scale=None), INVALID), ("taccl_norm", dict(q=None), INVALID),
    ("taccl_norm", dict(out=None, q=None, scale=None), INVALID),
    ("taccl_norm", dict(x=None), INVALID), ("taccl_norm", dict(weight=None), INVALID),
    ("taccl_norm", dict(x=4097), INVALID), ("taccl_norm", dict(scale=4098), INVALID),
    ("taccl_norm", dict(x_stride=63), INVALID), ("taccl_norm", dict(out_stride=-64), INVALID),
    ("taccl_norm", dict(q_stride=0), INVALID), ("taccl_norm", dict(scale_stride=0), INVALID),
    ("taccl_norm", dict(residual=4096), INVALID), ("taccl_norm", dict(total=4096), INVALID),
    ("taccl_norm_backward", dict(dweight=None), INVALID),
    ("taccl_norm_backward", dict(dx=4098), INVALID),
    ("taccl_norm_backward", dict(dtotal=4096), INVALID),
    ("taccl_norm_backward", dict(workspace=None), INVALID),
    ("taccl_norm_backward", dict(workspace_bytes=4096 * 64 - 1), INVALID),
    ("taccl_norm_backward", dict(cols=20000), LIMIT),
    ("taccl_route", dict(num_experts=0), INVALID), ("taccl_route", dict(k=0), INVALID),
    ("taccl_route", dict(k=9), INVALID), ("taccl_route", dict(num_experts=1025), LIMIT),
    ("taccl_route", dict(num_experts=64, k=17), LIMIT),
    ("taccl_route", dict(tokens=1 << 22), LIMIT), ("taccl_route", dict(capacity=-1), INVALID),
    ("taccl_route", dict(logits=None), INVALID), ("taccl_route", dict(slots=None), INVALID),
    ("taccl_route", dict(logits_stride=7), INVALID), ("taccl_route", dict(loss=4097), INVALID),
    ("taccl_route", dict(workspace_bytes=100), INVALID),
    ("taccl_route_backward", dict(rows=None), INVALID),
    ("taccl_route_backward", dict(dweights=4097), INVALID),
    ("taccl_route_backward", dict(dlogits_stride=4), INVALID),
    ("taccl_dispatch", dict(element_bytes=8), INVALID),
    ("taccl_dispatch", dict(capacity=0), INVALID), ("taccl_dispatch", dict(capacity=1 << 31), LIMIT),
    ("taccl_dispatch", dict(cols=0), INVALID), ("taccl_dispatch", dict(cols=(1 << 20) + 1), LIMIT),
    ("taccl_dispatch", dict(counts=None), INVALID), ("taccl_dispatch", dict(x=4097), INVALID),
    ("taccl_dispatch", dict(x_stride=8), INVALID),
    ("taccl_dispatch", dict(scale_cols=-1), INVALID),
    ("taccl_dispatch", dict(scale_cols=1), INVALID),
    ("taccl_dispatch", dict(scale_cols=2, scale=4096, scale_stride=1, out_scale=4096), INVALID),
    ("taccl_combine", dict(buffer=None), INVALID), ("taccl_combine", dict(weights=4099), INVALID),
    ("taccl_combine", dict(out_stride=1), INVALID), ("taccl_combine", dict(dtype=7), INVALID),
    ("taccl_combine_backward", dict(weights=None), INVALID),
    ("taccl_combine_backward", dict(dbuffer=4097), INVALID),
    ("taccl_combine_backward", dict(num_experts=2000), LIMIT),
]


@pytest.mark.parametrize("name,change,want", BAD, ids=[f"{n}-{c}" for n, c, _ in BAD])
def test_refusals(name, change, want):
    cls = STRUCTS[name + "_t"]
    st, message = status(name, cls(**{**GOOD[name], **change}))
    assert st == want, (st, message)
    assert message.startswith(name + ":")


@pytest.mark.parametrize("name", GOOD)
def test_null_arguments(name):
    st, message = status(name, None)
    assert st == INVALID and message == name + ": null arguments"


def test_nothing_to_do():
    """No rows: success without a device."""
    assert status("taccl_norm", _Norm(rows=0, cols=4, out=4096))[0] == B.OK
    assert status("taccl_combine", _Combine(tokens=0, capacity=1, num_experts=1, k=1,
                                              cols=4))[0] == B.OK
    assert status("taccl_route_backward", _RouteBackward(tokens=0, num_experts=4, k=1))[0] == B.OK


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x, w = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises(ValueError, match="CUDA"):
        X.norm_tensors(x, w, torch.empty(4, 8))
    with pytest.raises(ValueError, match="matrix"):
        X.norm_tensors(torch.zeros(4, 8, dtype=torch.float64), w, x)
    with pytest.raises(ValueError, match="matrix"):
        X.norm_tensors(torch.zeros(8), w, x)
    i = torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        X.route_tensors(x, i, torch.zeros(4, 2), i, i[0], w, w[:1], i[0, :1], w)
    with pytest.raises(ValueError, match=r"\[experts, capacity, dim\]"):
        X.dispatch_tensors(x, i, i, i[0], x)
    with pytest.raises(ValueError, match=r"\[experts, capacity, dim\]"):
        X.combine_tensors(torch.zeros(2, 3, 8), i, i, x)


def test_chunk_bytes():
    assert X.chunk_bytes(64, 40, 4224, 16) == 4 * 40 * 4224
    assert X.chunk_bytes(64, 40, 4096, 16, chunks_per_pair=2) == 2 * 40 * 4096
    with pytest.raises(ValueError):
        X.chunk_bytes(60, 40, 4096, 16)
    with pytest.raises(ValueError):
        X.chunk_bytes(16, 1, 7, 16, chunks_per_pair=2)


def test_header_states_the_limits():
    text = open(os.path.join(ROOT, "include", "taccl.h")).read()
    assert re.search(r"1 <= cols <= 16384", text) and re.search(r"tokens <= 2\^21", text)


def test_binding_refuses_what_is_no_tensor():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="x must be a CUDA tensor"):
        X.norm_tensors([1.0], x)
    with pytest.raises(ValueError, match="buffer must be a CUDA tensor"):
        X.combine_tensors(None, x, x, x)
    with pytest.raises(TypeError, match="takes 10 arguments"):
        X._calls.norm(x)
