"""Expert layer around an expert-parallel Alltoall (include/taccl.h).

An Alltoall plan moves chunks of one size between ranks; these operators make
the chunks and take them back: `norm` gives the token rows (also in 8 bits),
`route` the experts, places and loads with the loss that keeps them even,
`dispatch` the send buffer [experts, capacity, dim], whose rows for one rank's
experts are that rank's chunks (`chunk_bytes` is their size), and `combine`
the tokens from the rows that come back.

`*_tensors` run the library's kernels on the caller's CUDA tensors, on
`stream` (default: torch's current stream) of the current device, without
allocating; a tensor made on another stream has to be ready on this one, as
for any kernel. `norm`, `route`, `dispatch` and `combine` allocate their
results and are differentiable. There is no fallback: without the library they
raise.
"""
import ctypes as ct

import torch

from . import binding

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_P, _I32, _I64, _F32 = ct.c_void_p, ct.c_int32, ct.c_int64, ct.c_float


def _struct(name, fields):
    return type(name, (ct.Structure,), {"_fields_": fields})


# argument structs of include/taccl.h, in their order
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

_calls = {}


def _bind(name):
    fn = getattr(binding.lib(), name)
    fn.argtypes, fn.restype = [_P, _P], ct.c_int
    _calls[name] = fn
    return fn


def _call(name, args, device, stream):
    """The library's call on `stream`, or on the current one of `device`."""
    fn = _calls.get(name) or _bind(name)
    status = fn(ct.addressof(args), torch._C._cuda_getCurrentRawStream(device)
                if stream is None else stream.cuda_stream)
    if status:
        binding._check(status)


def _size(name, arg):
    fn = getattr(binding.lib(), name)
    fn.argtypes, fn.restype = [_I32], _I64
    return fn(arg)


def norm_workspace(cols):
    """Bytes of norm_backward_tensors' workspace."""
    return _size("taccl_norm_workspace", int(cols))


def route_workspace(num_experts):
    """Bytes of route_tensors' workspace."""
    return _size("taccl_route_workspace", int(num_experts))


def _wrong(t, name, what, shape, dtype):
    return ValueError(f"{name} must be a {what} {list(shape)} of {dtype}, got {list(t.shape)} of "
                      f"{t.dtype} with strides {t.stride()} on {t.device}")


def _rows(t, name, shape, dtype, device):
    """(pointer, row stride) of a matrix on `device` with a contiguous last axis."""
    if t.dtype is dtype and t.get_device() == device and t.shape == shape:
        stride = t.stride()
        if stride[1] == 1 or shape[1] <= 1:
            return t.data_ptr(), stride[0]
    raise _wrong(t, name, "CUDA tensor with contiguous rows", shape, dtype)


def _flat(t, name, shape, dtype, device):
    """Pointer of a contiguous tensor on `device`."""
    if t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise _wrong(t, name, "contiguous CUDA tensor", shape, dtype)


def _on_device(t, name):
    """Index of the tensor's device, which has to be the current one."""
    device = t.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        raise ValueError(f"{name} must be a CUDA tensor on the current device, is on {t.device}")
    return device


def _matrix(t, name):
    """(shape, type, its code, device) of the tensor that a call's others go by."""
    dtype = t.dtype
    code = _DTYPES.get(dtype)
    if code is None or t.dim() != 2:
        raise ValueError(f"{name} must be a matrix of {', '.join(str(d) for d in _DTYPES)}, got "
                         f"{list(t.shape)} of {dtype}")
    return t.shape, dtype, code, _on_device(t, name)


def _code(dtype, name):
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"{name} is of {dtype}, must be one of {', '.join(map(str, _DTYPES))}")
    return code


def _bytes(t, name, device):
    if t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor on the current device")
    return t.data_ptr(), t.numel() * t.element_size()


# ---- norm -----------------------------------------------------------------------

def norm_tensors(x, weight, out=None, *, eps=1e-6, residual=None, total=None, q=None, scale=None,
                 group=128, stream=None):
    """taccl_norm: h = x + residual; out = weight * h / sqrt(mean(h^2) + eps);
    total = h; q (float8_e4m3fn) = out / scale, scale [rows, ceil(cols /
    group)] in 32 bits (group 0: one column). Outputs that are None are left
    out."""
    shape, dtype, code, device = _matrix(x, "x")
    n, d = shape
    p, stride = _rows(x, "x", shape, dtype, device)
    r = o = h = f = s = None
    r_stride = o_stride = h_stride = f_stride = s_stride = 0
    if residual is not None:
        r, r_stride = _rows(residual, "residual", shape, dtype, device)
    if out is not None:
        o, o_stride = _rows(out, "out", shape, dtype, device)
    if total is not None:
        h, h_stride = _rows(total, "total", shape, dtype, device)
    if q is not None:
        f, f_stride = _rows(q, "q", shape, torch.float8_e4m3fn, device)
    if scale is not None:
        s, s_stride = _rows(scale, "scale", (n, -(-d // group) if group else 1), torch.float32,
                            device)
    w = _flat(weight, "weight", (d,), dtype, device)
    _call("taccl_norm", _Norm(n, d, code, eps, group, p, r, stride, r_stride, w, o, h, o_stride,
                              h_stride, f, s, f_stride, s_stride), device, stream)


def norm_backward_tensors(dout, h, weight, dx, dweight, workspace, *, eps=1e-6, dtotal=None,
                          stream=None):
    """taccl_norm_backward: dx (of x and of residual) and dweight (32 bits)
    from dout, the stored total h and the gradient dtotal that reaches h
    directly."""
    shape, dtype, code, device = _matrix(h, "h")
    n, d = shape
    g, g_stride = _rows(dout, "dout", shape, dtype, device)
    p, stride = _rows(h, "h", shape, dtype, device)
    t, t_stride = (None, 0) if dtotal is None else _rows(dtotal, "dtotal", shape, dtype, device)
    o, o_stride = _rows(dx, "dx", shape, dtype, device)
    w, w_bytes = _bytes(workspace, "workspace", device)
    _call("taccl_norm_backward",
          _NormBackward(n, d, code, eps, g, p, t, g_stride, stride, t_stride,
                        _flat(weight, "weight", (d,), dtype, device), o, o_stride,
                        _flat(dweight, "dweight", (d,), torch.float32, device), w, w_bytes),
          device, stream)


# ---- route ----------------------------------------------------------------------

def route_tensors(logits, experts, weights, slots, counts, prob_sums, loss, rows, workspace, *,
                  mask=None, capacity=0, coef=0.01, renorm=True, stream=None):
    """taccl_route: experts int32, weights float32 and slots int32
    [tokens, k], counts int32 and prob_sums float32 [experts], loss float32
    [1] and rows int32 [1] from logits [tokens, experts]; mask uint8 [tokens]."""
    (n, e), dtype, code, device = _matrix(logits, "logits")
    p, stride = _rows(logits, "logits", (n, e), dtype, device)
    if experts.dim() != 2:
        raise ValueError("experts must be a matrix [tokens, k]")
    shape = (n, experts.shape[1])
    m = None if mask is None else _flat(mask, "mask", (n,), torch.uint8, device)
    w, w_bytes = _bytes(workspace, "workspace", device)
    _call("taccl_route",
          _Route(n, e, shape[1], code, 1 if renorm else 0, coef, capacity, p, stride, m,
                 _flat(experts, "experts", shape, torch.int32, device),
                 _flat(weights, "weights", shape, torch.float32, device),
                 _flat(slots, "slots", shape, torch.int32, device),
                 _flat(counts, "counts", (e,), torch.int32, device),
                 _flat(prob_sums, "prob_sums", (e,), torch.float32, device),
                 _flat(loss, "loss", (1,), torch.float32, device),
                 _flat(rows, "rows", (1,), torch.int32, device), w, w_bytes), device, stream)


def route_backward_tensors(logits, experts, counts, rows, dlogits, *, dweights=None, dloss=None,
                           mask=None, coef=0.01, renorm=True, stream=None):
    """taccl_route_backward: dlogits from dweights [tokens, k] and dloss [1]
    (float32; None: zero). counts and rows may be summed over ranks."""
    (n, e), dtype, code, device = _matrix(logits, "logits")
    p, stride = _rows(logits, "logits", (n, e), dtype, device)
    o, o_stride = _rows(dlogits, "dlogits", (n, e), dtype, device)
    if experts.dim() != 2:
        raise ValueError("experts must be a matrix [tokens, k]")
    shape = (n, experts.shape[1])
    _call("taccl_route_backward",
          _RouteBackward(n, e, shape[1], code, 1 if renorm else 0, coef, p, stride,
                         None if mask is None else _flat(mask, "mask", (n,), torch.uint8, device),
                         _flat(experts, "experts", shape, torch.int32, device),
                         _flat(counts, "counts", (e,), torch.int32, device),
                         _flat(rows, "rows", (1,), torch.int32, device),
                         None if dweights is None else
                         _flat(dweights, "dweights", shape, torch.float32, device),
                         None if dloss is None else
                         _flat(dloss, "dloss", (1,), torch.float32, device),
                         o, o_stride), device, stream)


# ---- dispatch and combine ---------------------------------------------------------

def chunk_bytes(num_experts, capacity, row_bytes, ranks, chunks_per_pair=1):
    """Bytes of an Alltoall chunk that carries one rank's share of a dispatch
    buffer: num_experts / ranks experts of `capacity` rows each, split over
    chunks_per_pair chunks."""
    total = num_experts * capacity * row_bytes
    if num_experts % ranks or total % (ranks * chunks_per_pair):
        raise ValueError(f"{num_experts} experts of {capacity} rows of {row_bytes} bytes do not "
                         f"split into {chunks_per_pair} chunks for each of {ranks} ranks")
    return total // (ranks * chunks_per_pair)


def _choices(experts, slots, device):
    """(tokens, k, pointers) of the choices."""
    if experts.dim() != 2:
        raise ValueError("experts must be a matrix [tokens, k]")
    shape = experts.shape
    return shape, _flat(experts, "experts", shape, torch.int32, device), \
        _flat(slots, "slots", shape, torch.int32, device)


def _buffer(t, name):
    """(shape, device) of a buffer."""
    if t.dim() != 3 or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be a contiguous CUDA tensor [experts, capacity, dim], got "
                         f"{list(t.shape)} with strides {t.stride()} on {t.device}")
    return t.shape, _on_device(t, name)


def dispatch_tensors(x, experts, slots, counts, out, *, scale=None, out_scale=None, stream=None):
    """taccl_dispatch: out[experts[t, j], slots[t, j]] = x[t], zero from
    counts on; scale [tokens, n] float32 goes to out_scale [experts, capacity,
    n] alike. x of any type of 1, 2 or 4 bytes."""
    (e, c, d), device = _buffer(out, "out")
    (n, k), pe, ps = _choices(experts, slots, device)
    p, stride = _rows(x, "x", (n, d), out.dtype, device)
    s = o = None
    s_cols = s_stride = 0
    if scale is not None:
        if out_scale is None or scale.dim() != 2:
            raise ValueError("scale must be a matrix and come with out_scale")
        s_cols = scale.shape[1]
        s, s_stride = _rows(scale, "scale", (n, s_cols), torch.float32, device)
        o = _flat(out_scale, "out_scale", (e, c, s_cols), torch.float32, device)
    _call("taccl_dispatch",
          _Dispatch(n, c, e, k, d, x.element_size(), s_cols, p, stride, s, s_stride, pe, ps,
                    _flat(counts, "counts", (e,), torch.int32, device), out.data_ptr(), o),
          device, stream)


def combine_tensors(buffer, experts, slots, out, *, weights=None, stream=None):
    """taccl_combine: out[t] = sum over j of weights[t, j] *
    buffer[experts[t, j], slots[t, j]] (weights None: 1)."""
    shape, device = _buffer(buffer, "buffer")
    e, c, d = shape
    (n, k), pe, ps = _choices(experts, slots, device)
    dtype = buffer.dtype
    code = _code(dtype, "buffer")
    o, o_stride = _rows(out, "out", (n, d), dtype, device)
    w = None if weights is None else _flat(weights, "weights", (n, k), torch.float32, device)
    _call("taccl_combine",
          _Combine(n, c, e, k, d, code, buffer.data_ptr(), pe, ps, w, o, o_stride),
          device, stream)


def combine_backward_tensors(dout, buffer, experts, slots, counts, weights, dbuffer, dweights, *,
                             stream=None):
    """taccl_combine_backward: dbuffer (zero from counts on) and dweights."""
    shape, device = _buffer(buffer, "buffer")
    e, c, d = shape
    (n, k), pe, ps = _choices(experts, slots, device)
    dtype = buffer.dtype
    code = _code(dtype, "buffer")
    g, g_stride = _rows(dout, "dout", (n, d), dtype, device)
    _call("taccl_combine_backward",
          _CombineBackward(n, c, e, k, d, code, g, g_stride, buffer.data_ptr(), pe, ps,
                           _flat(counts, "counts", (e,), torch.int32, device),
                           _flat(weights, "weights", (n, k), torch.float32, device),
                           _flat(dbuffer, "dbuffer", shape, dtype, device),
                           _flat(dweights, "dweights", (n, k), torch.float32, device)),
          device, stream)


# ---- differentiable forms ---------------------------------------------------------

def _workspace(n, like):
    return torch.empty(n, dtype=torch.uint8, device=like.device)


def _gradient_rows(g):
    """A gradient as the kernels take it (autograd may hand over expanded ones)."""
    return g if g.dim() != 2 or g.stride(1) == 1 and g.stride(0) >= g.shape[1] else g.contiguous()


class _NormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps, group, quantize):
        ctx.set_materialize_grads(False)
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        total = x if residual is None else torch.empty_like(out)
        q = scale = None
        if quantize:
            n, d = x.shape
            q = torch.empty(n, d, dtype=torch.float8_e4m3fn, device=x.device)
            scale = torch.empty(n, -(-d // group) if group else 1, device=x.device)
        norm_tensors(x, weight, out, eps=eps, residual=residual,
                     total=None if residual is None else total, q=q, scale=scale, group=group)
        ctx.save_for_backward(total, weight)
        ctx.eps, ctx.has_residual = eps, residual is not None
        if quantize:
            ctx.mark_non_differentiable(q, scale)
        return out, (total if residual is not None else None), q, scale

    @staticmethod
    def backward(ctx, dout, dtotal, _q, _scale):
        h, weight = ctx.saved_tensors
        if dout is None:
            dout = torch.zeros(h.shape, dtype=h.dtype, device=h.device)
        dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
        dweight = torch.empty(h.shape[1], device=h.device)
        norm_backward_tensors(_gradient_rows(dout), h, weight, dx, dweight,
                              _workspace(norm_workspace(h.shape[1]), h), eps=ctx.eps,
                              dtotal=None if dtotal is None else _gradient_rows(dtotal))
        return dx, dweight.to(weight.dtype), dx if ctx.has_residual else None, None, None, None


def norm(x, weight, residual=None, *, eps=1e-6, group=128, quantize=False):
    """(out, total, q, scale) of norm_tensors; total is None without a
    residual, q and scale (no gradient) without `quantize`."""
    return _NormFn.apply(x, weight, residual, eps, group, quantize)


class _RouteFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, mask, capacity, coef, renorm):
        ctx.set_materialize_grads(False)
        n, e = logits.shape

        def new(dtype, *shape):
            return torch.empty(*shape, dtype=dtype, device=logits.device)

        experts, slots = new(torch.int32, n, k), new(torch.int32, n, k)
        weights, counts = new(torch.float32, n, k), new(torch.int32, e)
        prob_sums, loss, rows = new(torch.float32, e), new(torch.float32, 1), new(torch.int32, 1)
        route_tensors(logits, experts, weights, slots, counts, prob_sums, loss, rows,
                      _workspace(route_workspace(e), logits), mask=mask, capacity=capacity,
                      coef=coef, renorm=renorm)
        ctx.save_for_backward(logits, experts, counts, rows)
        ctx.mask, ctx.coef, ctx.renorm = mask, coef, renorm
        ctx.mark_non_differentiable(experts, slots, counts, prob_sums, rows)
        return experts, weights, slots, counts, prob_sums, loss, rows

    @staticmethod
    def backward(ctx, _experts, dweights, _slots, _counts, _sums, dloss, _rows_):
        logits, experts, counts, rows = ctx.saved_tensors
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        route_backward_tensors(logits, experts, counts, rows, dlogits,
                               dweights=None if dweights is None else dweights.contiguous(),
                               dloss=None if dloss is None else dloss.contiguous(),
                               mask=ctx.mask, coef=ctx.coef, renorm=ctx.renorm)
        return dlogits, None, None, None, None, None


def route(logits, k, *, mask=None, capacity=0, coef=0.01, renorm=True):
    """(experts, weights, slots, counts, prob_sums, loss, rows) of
    route_tensors; gradients flow from weights and loss to the logits."""
    return _RouteFn.apply(logits, k, mask, capacity, coef, renorm)


class _DispatchFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, experts, slots, counts, capacity):
        out = torch.empty(len(counts), capacity, x.shape[1], dtype=x.dtype, device=x.device)
        dispatch_tensors(x, experts, slots, counts, out)
        ctx.save_for_backward(experts, slots)
        return out

    @staticmethod
    def backward(ctx, dout):
        experts, slots = ctx.saved_tensors
        dx = torch.empty(len(experts), dout.shape[2], dtype=dout.dtype, device=dout.device)
        combine_tensors(dout.contiguous(), experts, slots, dx)
        return dx, None, None, None, None


def dispatch(x, experts, slots, counts, capacity):
    """Buffer [experts, capacity, dim] of dispatch_tensors."""
    return _DispatchFn.apply(x, experts, slots, counts, capacity)


class _CombineFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, buffer, experts, slots, counts, weights):
        out = torch.empty(len(experts), buffer.shape[2], dtype=buffer.dtype, device=buffer.device)
        combine_tensors(buffer, experts, slots, out, weights=weights)
        ctx.save_for_backward(buffer, experts, slots, counts, weights)
        return out

    @staticmethod
    def backward(ctx, dout):
        buffer, experts, slots, counts, weights = ctx.saved_tensors
        dbuffer, dweights = torch.empty_like(buffer), torch.empty_like(weights)
        combine_backward_tensors(_gradient_rows(dout), buffer, experts, slots, counts, weights,
                                 dbuffer, dweights)
        return dbuffer, None, None, None, dweights


def combine(buffer, experts, slots, counts, weights):
    """Tokens [tokens, dim] of combine_tensors; gradients flow to the buffer
    and the weights."""
    return _CombineFn.apply(buffer, experts, slots, counts, weights)
