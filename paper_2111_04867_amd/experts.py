"""Expert layer around an expert-parallel Alltoall (include/taccl.h).

An Alltoall plan moves chunks of one size between ranks; these operators make
the chunks and take them back: `norm` gives the token rows (also in 8 bits),
`route` the experts, places and loads with the loss that keeps them even,
`dispatch` the send buffer [experts, capacity, dim], whose rows for one rank's
experts are that rank's chunks (`chunk_bytes` is their size), `ffn` the rows
through the experts, as they arrive from every rank, and `combine` the tokens
from the rows that come back; `dropout` adds them to the residual. `ffn_tokens`
is the whole layer of a few tokens.

`*_tensors` run the library's kernels on the caller's CUDA tensors, on
`stream` (default: torch's current stream) of the current device, without
allocating; a tensor made on another stream has to be ready on this one, as
for any kernel. `norm`, `route`, `dispatch`, `ffn`, `combine` and `dropout`
allocate their results and are differentiable, once: a second derivative
raises. `ffn_tokens` allocates its results and has no gradient. There is no
fallback: without the library they raise.

All calls can be captured into a graph. For a gradient torch asks that no
autograd graph of an earlier pass over the same leaves is alive when a pass is
captured (it adds to a leaf's gradient on the stream of the first one, which is
not the captured one): drop the earlier results first, or capture over leaves of
its own.
"""
import ctypes as ct

import torch
from torch.autograd.function import once_differentiable

from . import binding

try:
    from . import _experts as _calls
except ImportError as e:
    raise ImportError("paper_2111_04867_amd/_experts.so is missing or does not load: build it with "
                      f"__graft_entry__.build() ({e})") from e


def _address(name):
    return ct.cast(getattr(binding.lib(), "taccl_" + name), ct.c_void_p).value


_calls.bind(torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream,
            *(_address(n) for n in ("norm", "norm_backward", "route", "route_backward", "dispatch",
                                    "combine", "combine_backward", "ffn", "ffn_backward",
                                    "ffn_tokens", "dropout")))


def _size(name, *args, types=None):
    fn = getattr(binding.lib(), name)
    fn.argtypes, fn.restype = types or [ct.c_int32] * len(args), ct.c_int64
    return fn(*args)


def norm_workspace(cols):
    """Bytes of norm_backward_tensors' workspace."""
    return _size("taccl_norm_workspace", int(cols))


def route_workspace(num_experts):
    """Bytes of route_tensors' workspace."""
    return _size("taccl_route_workspace", int(num_experts))


_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _fits(*sizes):
    return all(0 <= n < 1 << 31 for n in sizes)


def ffn_workspace(shape, hidden, dtype, backward=False):
    """Bytes of ffn_tensors' workspace (backward: ffn_backward_tensors') for
    rows of `shape` [experts, capacity, dim] or [sources, experts, capacity,
    dim]; 0 for sizes that they refuse."""
    s, e, c = (1, *shape[:2]) if len(shape) == 3 else shape[:3]
    if not _fits(s, e, c, hidden):
        return 0
    return _size("taccl_ffn_workspace", s, e, c, hidden, _DTYPES.get(dtype, -1), int(backward),
                 types=[ct.c_int32, ct.c_int32, ct.c_int64] + [ct.c_int32] * 3)


def ffn_tokens_workspace(tokens, k, dim, hidden):
    """Bytes of ffn_tokens_tensors' workspace; 0 for sizes that it refuses."""
    if not _fits(tokens, k, dim, hidden):
        return 0
    return _size("taccl_ffn_tokens_workspace", tokens, k, dim, hidden,
                 types=[ct.c_int64] + [ct.c_int32] * 3)


def dropout_words(rows, cols):
    """Random numbers that a call of dropout uses: what to add to rng[1]
    before the next one."""
    return rows * ((cols + 1) // 2)


def chunk_bytes(num_experts, capacity, row_bytes, ranks, chunks_per_pair=1):
    """Bytes of an Alltoall chunk that carries one rank's share of a dispatch
    buffer: num_experts / ranks experts of `capacity` rows each, split over
    chunks_per_pair chunks."""
    total = num_experts * capacity * row_bytes
    if num_experts % ranks or total % (ranks * chunks_per_pair):
        raise ValueError(f"{num_experts} experts of {capacity} rows of {row_bytes} bytes do not "
                         f"split into {chunks_per_pair} chunks for each of {ranks} ranks")
    return total // (ranks * chunks_per_pair)


# ---- on the caller's tensors --------------------------------------------------------
# The tensors are checked (ValueError) and the library called (TacclError) in
# pyext/experts.cpp. All have to be on the current device; matrices may have
# rows further apart than their length.

def norm_tensors(x, weight, out=None, *, eps=1e-6, residual=None, total=None, q=None, scale=None,
                 group=128, stream=None):
    """taccl_norm: h = x + residual; out = weight * h / sqrt(mean(h^2) + eps);
    total = h; q (float8_e4m3fn) = out / scale, scale [rows, ceil(cols /
    group)] in 32 bits (group 0: one column). Outputs that are None are left
    out."""
    st = _calls.norm(x, weight, out, eps, residual, total, q, scale, group,
                     stream and stream.cuda_stream)
    if st:
        binding._check(st)


def norm_backward_tensors(dout, h, weight, dx, dweight, workspace, *, eps=1e-6, dtotal=None,
                          stream=None):
    """taccl_norm_backward: dx (of x and of residual) and dweight (32 bits)
    from dout, the stored total h and the gradient dtotal that reaches h
    directly."""
    st = _calls.norm_backward(dout, h, weight, dx, dweight, workspace, eps, dtotal,
                              stream and stream.cuda_stream)
    if st:
        binding._check(st)


def route_tensors(logits, experts, weights, slots, counts, prob_sums, loss, rows, workspace, *,
                  mask=None, capacity=0, coef=0.01, renorm=True, stream=None):
    """taccl_route: experts int32, weights float32 and slots int32
    [tokens, k], counts int32 and prob_sums float32 [experts], loss float32
    [1] and rows int32 [1] from logits [tokens, experts]; mask uint8 or bool [tokens]."""
    st = _calls.route(logits, experts, weights, slots, counts, prob_sums, loss, rows, workspace,
                      mask, capacity, coef, renorm, stream and stream.cuda_stream)
    if st:
        binding._check(st)


def route_backward_tensors(logits, experts, counts, rows, dlogits, *, dweights=None, dloss=None,
                           mask=None, coef=0.01, renorm=True, stream=None):
    """taccl_route_backward: dlogits from dweights [tokens, k] and dloss [1]
    (float32; None: zero). counts and rows may be summed over ranks."""
    st = _calls.route_backward(logits, experts, counts, rows, dlogits, dweights, dloss, mask, coef,
                               renorm, stream and stream.cuda_stream)
    if st:
        binding._check(st)


def dispatch_tensors(x, experts, slots, counts, out, *, scale=None, out_scale=None, stream=None):
    """taccl_dispatch: out[experts[t, j], slots[t, j]] = x[t], zero from
    counts on; scale [tokens, n] float32 goes to out_scale [experts, capacity,
    n] alike. x of any type of 1, 2 or 4 bytes."""
    st = _calls.dispatch(x, experts, slots, counts, out, scale, out_scale,
                         stream and stream.cuda_stream)
    if st:
        binding._check(st)


def combine_tensors(buffer, experts, slots, out, *, weights=None, stream=None):
    """taccl_combine: out[t] = sum over j of weights[t, j] *
    buffer[experts[t, j], slots[t, j]] (weights None: 1)."""
    st = _calls.combine(buffer, experts, slots, out, weights, stream and stream.cuda_stream)
    if st:
        binding._check(st)


def combine_backward_tensors(dout, buffer, experts, slots, counts, weights, dbuffer, dweights, *,
                             stream=None):
    """taccl_combine_backward: dbuffer (zero from counts on) and dweights."""
    st = _calls.combine_backward(dout, buffer, experts, slots, counts, weights, dbuffer, dweights,
                                 stream and stream.cuda_stream)
    if st:
        binding._check(st)


def ffn_tensors(buffer, counts, w_in, w_out, out, workspace, *, pre=None, stream=None):
    """taccl_ffn: out = w_out[e] (silu(g) * u) with (g, u) = w_in[e] x for the
    rows x of buffer [experts, capacity, dim] or [sources, experts, capacity,
    dim] below counts int32 [experts] or [sources, experts], zero from there
    on; w_in [experts, 2 hidden, dim], w_out [experts, dim, hidden]. pre [...,
    2 hidden] keeps g and u for the gradient. out may be buffer."""
    st = _calls.ffn(buffer, counts, w_in, w_out, out, workspace, pre,
                    stream and stream.cuda_stream)
    if st:
        binding._check(st)


def ffn_backward_tensors(dout, buffer, counts, w_in, w_out, pre, workspace, *, dbuffer=None,
                         dw_in=None, dw_out=None, stream=None):
    """taccl_ffn_backward: the gradients that are given, dbuffer (zero from
    counts on), dw_in and dw_out."""
    st = _calls.ffn_backward(dout, buffer, counts, w_in, w_out, pre, workspace, dbuffer, dw_in,
                             dw_out, stream and stream.cuda_stream)
    if st:
        binding._check(st)


def ffn_tokens_tensors(x, logits, w_in, w_out, out, workspace, *, k, mask=None, renorm=True,
                       first_expert=0, experts=None, weights=None, stream=None):
    """taccl_ffn_tokens: route's choices of up to 64 tokens x [tokens, dim] by
    logits [tokens, experts] and, in out, the weighted sum over them of ffn
    with the weights w_in and w_out of the experts from first_expert on; the
    choices go to experts int32 and weights float32 [tokens, k]."""
    st = _calls.ffn_tokens(x, logits, w_in, w_out, out, workspace, k, mask, renorm, first_expert,
                           experts, weights, stream and stream.cuda_stream)
    if st:
        binding._check(st)


def dropout_tensors(x, rng, out, *, p, residual=None, stream=None):
    """taccl_dropout: out = residual + (kept ? x / (1 - p) : 0), by the random
    numbers of rng int64 [2] (seed and offset, on the device)."""
    st = _calls.dropout(x, rng, out, p, residual, stream and stream.cuda_stream)
    if st:
        binding._check(st)


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
    @once_differentiable
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
        ctx.save_for_backward(logits, experts, counts, rows, mask)
        ctx.coef, ctx.renorm = coef, renorm
        ctx.mark_non_differentiable(experts, slots, counts, prob_sums, rows)
        return experts, weights, slots, counts, prob_sums, loss, rows

    @staticmethod
    @once_differentiable
    def backward(ctx, _experts, dweights, _slots, _counts, _sums, dloss, _rows_):
        logits, experts, counts, rows, mask = ctx.saved_tensors
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        route_backward_tensors(logits, experts, counts, rows, dlogits,
                               dweights=None if dweights is None else dweights.contiguous(),
                               dloss=None if dloss is None else dloss.contiguous(),
                               mask=mask, coef=ctx.coef, renorm=ctx.renorm)
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
    @once_differentiable
    def backward(ctx, dout):
        experts, slots = ctx.saved_tensors
        dx = torch.empty(len(experts), dout.shape[2], dtype=dout.dtype, device=dout.device)
        combine_tensors(dout.contiguous(), experts, slots, dx)
        return dx, None, None, None, None


def dispatch(x, experts, slots, counts, capacity):
    """Buffer [experts, capacity, dim] of dispatch_tensors. `capacity` is
    route's, or less; for a larger buffer give counts.clamp(max=route's), here
    and to combine, or the rows between hold whatever the memory held."""
    return _DispatchFn.apply(x, experts, slots, counts, capacity)


class _CombineFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, buffer, experts, slots, counts, weights):
        out = torch.empty(len(experts), buffer.shape[2], dtype=buffer.dtype, device=buffer.device)
        combine_tensors(buffer, experts, slots, out, weights=weights)
        ctx.save_for_backward(buffer, experts, slots, counts, weights)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        buffer, experts, slots, counts, weights = ctx.saved_tensors
        dbuffer = torch.empty_like(buffer)
        if weights is None:
            dispatch_tensors(_gradient_rows(dout), experts, slots, counts, dbuffer)
            return dbuffer, None, None, None, None
        dweights = torch.empty_like(weights)
        combine_backward_tensors(_gradient_rows(dout), buffer, experts, slots, counts, weights,
                                 dbuffer, dweights)
        return dbuffer, None, None, None, dweights


def combine(buffer, experts, slots, counts, weights):
    """Tokens [tokens, dim] of combine_tensors; gradients flow to the buffer
    and the weights (None: 1)."""
    return _CombineFn.apply(buffer, experts, slots, counts, weights)


class _FfnFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, buffer, counts, w_in, w_out, recorded):
        hidden = w_out.shape[2]
        out = torch.empty_like(buffer)
        pre = None
        if recorded and any(ctx.needs_input_grad):
            pre = torch.empty(*buffer.shape[:-1], 2 * hidden, dtype=buffer.dtype,
                              device=buffer.device)
        ffn_tensors(buffer, counts, w_in, w_out, out,
                    _workspace(ffn_workspace(buffer.shape, hidden, buffer.dtype), buffer), pre=pre)
        ctx.save_for_backward(buffer, counts, w_in, w_out, pre)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        buffer, counts, w_in, w_out, pre = ctx.saved_tensors
        want = ctx.needs_input_grad
        given = [torch.empty_like(t) if need else None
                 for t, need in ((buffer, want[0]), (w_in, want[2]), (w_out, want[3]))]
        size = ffn_workspace(buffer.shape, w_out.shape[2], buffer.dtype, True)
        ffn_backward_tensors(dout.contiguous(), buffer, counts, w_in, w_out, pre,
                             _workspace(size, buffer), dbuffer=given[0], dw_in=given[1],
                             dw_out=given[2])
        return given[0], None, given[1], given[2], None


def ffn(buffer, counts, w_in, w_out):
    """Rows of ffn_tensors; gradients flow to the buffer and the weights. What
    they need is kept only where autograd records the call."""
    # asked for here: within forward gradients are off, and needs_input_grad
    # tells what the tensors want under no_grad too
    return _FfnFn.apply(buffer, counts, w_in, w_out, torch.is_grad_enabled())


class _FfnTokensFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, logits, k, w_in, w_out, mask, renorm, first_expert):
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        experts = torch.empty(len(x), k, dtype=torch.int32, device=x.device)
        weights = torch.empty(len(x), k, device=x.device)
        size = ffn_tokens_workspace(len(x), k, x.shape[1], w_out.shape[2])
        ffn_tokens_tensors(x, logits, w_in, w_out, out, _workspace(size, x), k=k, mask=mask,
                           renorm=renorm, first_expert=first_expert, experts=experts,
                           weights=weights)
        ctx.mark_non_differentiable(experts)
        return out, experts, weights

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("ffn_tokens has no gradient: take route, dispatch, ffn and combine")


def ffn_tokens(x, logits, k, w_in, w_out, *, mask=None, renorm=True, first_expert=0):
    """(out, experts, weights) of ffn_tokens_tensors, without a gradient."""
    return _FfnTokensFn.apply(x, logits, k, w_in, w_out, mask, renorm, first_expert)


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, rng, p, residual):
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dropout_tensors(x, rng, out, p=p, residual=residual)
        ctx.save_for_backward(rng)
        ctx.p = p
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        rng, = ctx.saved_tensors
        dx = None
        if ctx.needs_input_grad[0]:
            dx = torch.empty(dout.shape, dtype=dout.dtype, device=dout.device)
            dropout_tensors(_gradient_rows(dout), rng, dx, p=ctx.p)
        return dx, None, None, dout if ctx.needs_input_grad[3] else None


def dropout(x, p, rng, residual=None):
    """Rows of dropout_tensors; gradients flow to x and the residual. The
    gradient draws the same numbers again, so rng has to stay as it is until
    then (a changed one raises): give every call its own, `rng + offset`, or
    step a shared one between the training steps."""
    return _DropoutFn.apply(x, rng, p, residual)
