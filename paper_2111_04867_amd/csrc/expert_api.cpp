// C ABI of the expert-layer operators: checks of arguments and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <string>

#include "expert.h"
#include "ffn.h"
#include "plan.h"

namespace taccl {
namespace {

// The first failed check of a call is its error.
struct Check {
  const char *call;
  taccl_status_t st = TACCL_OK;

  void that(bool ok, taccl_status_t status, const char *what) {
    if (!ok && st == TACCL_OK) st = fail(status, std::string(call) + ": " + what);
  }
  void invalid(bool bad, const char *what) { that(!bad, TACCL_ERR_INVALID_ARGUMENT, what); }
  void limit(bool bad, const char *what) { that(!bad, TACCL_ERR_LIMIT, what); }

  // a pointer that has to be there, aligned to its elements
  void array(const void *p, int64_t align, const char *name) {
    if (!p) invalid(true, (std::string("null ") + name).c_str());
    else optional(p, align, name);
  }
  void optional(const void *p, int64_t align, const char *name) {
    if ((uintptr_t)p % (uintptr_t)align) invalid(true, (std::string("misaligned ") + name).c_str());
  }
  // rows `stride` elements apart (a single row has no stride)
  void stride(int64_t stride, int64_t cols, int64_t rows, const char *name) {
    if (rows > 1 && stride < cols)
      invalid(true, (std::string(name) + "'s stride is below the row's length").c_str());
  }
  void rows(int64_t n) {
    invalid(n < 0, "negative number of rows");
    limit(n > kMaxRows, "more than 2^21 rows");
  }
  void dtype(int32_t d) { invalid(d < TACCL_F32 || d > TACCL_F16, "unknown type"); }
  void experts(int32_t e, int32_t k) {
    invalid(e < 1 || k < 1, "num_experts and k must be at least 1");
    limit(e > kMaxExperts, "more than 1024 experts");
    limit(k > kMaxChoices, "more than 16 choices per token");
  }
  void workspace(const void *p, int64_t bytes, int64_t need) {
    array(p, 16, "workspace");
    invalid(bytes < need, "workspace too small");
  }
};

int64_t size_of(int32_t dtype) { return dtype == TACCL_F32 ? 4 : 2; }

// the buffer that dispatch and combine share
template <class A>
void check_buffer(Check &c, const A &a) {
  c.rows(a.tokens);
  c.experts(a.num_experts, a.k);
  c.invalid(a.capacity < 1, "capacity must be at least 1");
  c.limit(a.capacity > INT32_MAX, "capacity of 2^31 or more");
  c.invalid(a.cols < 1, "cols must be at least 1");
  c.limit(a.cols > kExchangeMaxCols, "more than 2^20 columns");
  if (a.tokens == 0) return;
  c.array(a.experts, 4, "experts");
  c.array(a.slots, 4, "slots");
}

// the sizes that taccl_ffn and its gradient share, and the workspace's
struct FfnSizes {
  int64_t sources, experts, capacity, cols, hidden;
  int32_t dtype;
};
void check_ffn_sizes(Check &c, const FfnSizes &z) {
  c.dtype(z.dtype);
  c.invalid(z.sources < 1 || z.experts < 1, "sources and num_experts must be at least 1");
  c.limit(z.sources > kFfnMaxSources, "more than 1024 sources");
  c.limit(z.experts > kMaxExperts, "more than 1024 experts");
  c.invalid(z.capacity < 1, "capacity must be at least 1");
  c.limit(z.capacity > kMaxRows || z.sources * z.capacity > kMaxRows,
          "more than 2^21 rows of an expert");
  c.limit(z.sources * z.experts * z.capacity > INT32_MAX, "2^31 rows or more");
  c.invalid(z.cols < 1 || z.hidden < 1, "cols and hidden must be at least 1");
  c.limit(z.cols > kFfnMaxCols || z.hidden > kFfnMaxCols, "more than 65536 columns");
  if (c.st) return;
  // blocks of the largest grid (the gradient's last one, of the smallest tiles),
  // whose threads have to stay below 2^32
  auto tiles = [](int64_t n) { return (n + 63) / 64; };
  const int64_t rows = (z.sources * z.capacity + 31) / 32, wide = tiles(2 * z.hidden);
  const int64_t all = rows * (wide + tiles(z.cols)) + tiles(z.cols) * 2 * wide;
  c.limit(z.experts * all >= 1 << 23, "2^23 tiles or more");
}
template <class A>
void check_ffn(Check &c, const A &a, bool backward) {
  const FfnSizes z{a.sources, a.num_experts, a.capacity, a.cols, a.hidden, a.dtype};
  check_ffn_sizes(c, z);
  if (c.st) return;
  const int64_t size = size_of(a.dtype);
  c.array(a.buffer, size, "buffer");
  c.array(a.counts, 4, "counts");
  c.array(a.w_in, size, "w_in");
  c.array(a.w_out, size, "w_out");
  c.workspace(a.workspace, a.workspace_bytes,
              ffn_space(z.sources, z.experts, z.capacity, z.hidden, z.dtype, backward).least);
}

taccl_status_t launched(hipError_t e, const char *call) {
  if (e == hipSuccess) return TACCL_OK;
  return fail(TACCL_ERR_HIP, std::string(call) + ": kernel launch: " + hipGetErrorString(e));
}

// CUs of the current device (asked for once per device)
taccl_status_t device_cus(const char *call, int *cus) {
  static std::atomic<int> known[64];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess && dev >= 0 && dev < 64 && (*cus = known[dev].load()) > 0) return TACCL_OK;
  if (e == hipSuccess) e = hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess)
    return fail(TACCL_ERR_HIP, std::string(call) + ": " + hipGetErrorString(e));
  if (dev < 64) known[dev].store(*cus);
  return TACCL_OK;
}

}  // namespace
}  // namespace taccl

using namespace taccl;

extern "C" {

taccl_status_t taccl_norm(const taccl_norm_t *a, taccl_stream_t stream) {
  Check c{"taccl_norm"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  c.rows(a->rows);
  c.dtype(a->dtype);
  c.invalid(a->cols < 1, "cols must be at least 1");
  c.limit(a->cols > kNormMaxCols, "more than 16384 columns");
  c.invalid(!(a->eps >= 0), "eps must be at least 0");
  c.invalid(a->group != 0 && a->group != 32 && a->group != 64 && a->group != 128 && a->group != 256,
            "group must be 0, 32, 64, 128 or 256");
  if (c.st || a->rows == 0) return c.st;  // empty arrays may be null
  c.invalid((a->q != nullptr) != (a->scale != nullptr), "q and scale come together");
  c.invalid(!a->out && !a->total && !a->q, "no output");
  const int64_t size = size_of(a->dtype), cols = a->cols;
  c.array(a->x, size, "x");
  c.optional(a->residual, size, "residual");
  c.array(a->weight, size, "weight");
  c.optional(a->out, size, "out");
  c.optional(a->total, size, "total");
  c.optional(a->scale, 4, "scale");
  c.stride(a->x_stride, cols, a->rows, "x");
  if (a->residual) c.stride(a->residual_stride, cols, a->rows, "residual");
  if (a->out) c.stride(a->out_stride, cols, a->rows, "out");
  if (a->total) c.stride(a->total_stride, cols, a->rows, "total");
  if (a->q) {
    c.stride(a->q_stride, cols, a->rows, "q");
    c.stride(a->scale_stride, a->group ? (cols + a->group - 1) / a->group : 1, a->rows, "scale");
  }
  if (c.st) return c.st;
  return launched(launch_norm(*a, (hipStream_t)stream), c.call);
}

int64_t taccl_norm_workspace(int32_t cols) {
  return cols < 1 ? 0 : (int64_t)sizeof(float) * kNormMaxBlocks * cols;
}

taccl_status_t taccl_norm_backward(const taccl_norm_backward_t *a, taccl_stream_t stream) {
  Check c{"taccl_norm_backward"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  c.rows(a->rows);
  c.dtype(a->dtype);
  c.invalid(a->cols < 1, "cols must be at least 1");
  c.limit(a->cols > kNormMaxCols, "more than 16384 columns");
  c.invalid(!(a->eps >= 0), "eps must be at least 0");
  if (c.st) return c.st;
  const int64_t size = size_of(a->dtype), cols = a->cols;
  c.array(a->dweight, 4, "dweight");
  c.array(a->weight, size, "weight");
  c.workspace(a->workspace, a->workspace_bytes, taccl_norm_workspace(a->cols));
  if (a->rows > 0) {
    c.array(a->dout, size, "dout");
    c.array(a->h, size, "h");
    c.optional(a->dtotal, size, "dtotal");
    c.array(a->dx, size, "dx");
    c.stride(a->dout_stride, cols, a->rows, "dout");
    c.stride(a->h_stride, cols, a->rows, "h");
    if (a->dtotal) c.stride(a->dtotal_stride, cols, a->rows, "dtotal");
    c.stride(a->dx_stride, cols, a->rows, "dx");
  }
  if (c.st) return c.st;
  int cus = 0;
  if (taccl_status_t st = device_cus(c.call, &cus)) return st;
  return launched(launch_norm_backward(*a, cus, (hipStream_t)stream), c.call);
}

int64_t taccl_route_workspace(int32_t num_experts) {
  // per block a row of sums (4 bytes each), one of counts (2) and the tokens that
  // count (4), and the word of the loss (8): it lies in the 2 bytes per column to spare
  const int64_t wide = ((int64_t)num_experts + 7) / 8 * 8;
  return num_experts < 1 ? 0 : kRouteMaxBlocks * (8 * wide + 4);
}

taccl_status_t taccl_route(const taccl_route_t *a, taccl_stream_t stream) {
  Check c{"taccl_route"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  c.rows(a->tokens);
  c.dtype(a->dtype);
  c.experts(a->num_experts, a->k);
  c.invalid(a->k > a->num_experts, "more choices than experts");
  c.invalid(a->capacity < 0, "negative capacity");
  if (c.st) return c.st;
  c.array(a->counts, 4, "counts");
  c.array(a->prob_sums, 4, "prob_sums");
  c.array(a->loss, 4, "loss");
  c.array(a->rows, 4, "rows");
  c.workspace(a->workspace, a->workspace_bytes, taccl_route_workspace(a->num_experts));
  if (a->tokens > 0) {
    c.array(a->logits, size_of(a->dtype), "logits");
    c.array(a->experts, 4, "experts");
    c.array(a->weights, 4, "weights");
    c.array(a->slots, 4, "slots");
    c.stride(a->logits_stride, a->num_experts, a->tokens, "logits");
  }
  if (c.st) return c.st;
  return launched(launch_route(*a, (hipStream_t)stream), c.call);
}

taccl_status_t taccl_route_backward(const taccl_route_backward_t *a, taccl_stream_t stream) {
  Check c{"taccl_route_backward"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  c.rows(a->tokens);
  c.dtype(a->dtype);
  c.experts(a->num_experts, a->k);
  c.invalid(a->k > a->num_experts, "more choices than experts");
  if (c.st || a->tokens == 0) return c.st;
  c.array(a->logits, size_of(a->dtype), "logits");
  c.array(a->experts, 4, "experts");
  c.array(a->counts, 4, "counts");
  c.array(a->rows, 4, "rows");
  c.optional(a->dweights, 4, "dweights");
  c.optional(a->dloss, 4, "dloss");
  c.array(a->dlogits, size_of(a->dtype), "dlogits");
  c.stride(a->logits_stride, a->num_experts, a->tokens, "logits");
  c.stride(a->dlogits_stride, a->num_experts, a->tokens, "dlogits");
  if (c.st) return c.st;
  int cus = 0;
  if (taccl_status_t st = device_cus(c.call, &cus)) return st;
  return launched(launch_route_backward(*a, cus, (hipStream_t)stream), c.call);
}

taccl_status_t taccl_dispatch(const taccl_dispatch_t *a, taccl_stream_t stream) {
  Check c{"taccl_dispatch"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  check_buffer(c, *a);
  const int64_t size = a->element_bytes;
  c.invalid(size != 1 && size != 2 && size != 4, "element_bytes must be 1, 2 or 4");
  c.invalid(a->scale_cols < 0, "negative scale_cols");
  c.limit(a->scale_cols > kExchangeMaxCols, "more than 2^20 columns of scales");
  if (c.st) return c.st;
  c.array(a->counts, 4, "counts");
  c.array(a->out, size, "out");
  if (a->scale_cols) c.array(a->out_scale, 4, "out_scale");
  if (a->tokens > 0) {
    c.array(a->x, size, "x");
    c.stride(a->x_stride, a->cols, a->tokens, "x");
    if (a->scale_cols) {
      c.array(a->scale, 4, "scale");
      c.stride(a->scale_stride, a->scale_cols, a->tokens, "scale");
    }
  }
  if (c.st) return c.st;
  int cus = 0;
  if (taccl_status_t st = device_cus(c.call, &cus)) return st;
  return launched(launch_dispatch(*a, cus, (hipStream_t)stream), c.call);
}

taccl_status_t taccl_combine(const taccl_combine_t *a, taccl_stream_t stream) {
  Check c{"taccl_combine"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  check_buffer(c, *a);
  c.dtype(a->dtype);
  if (c.st || a->tokens == 0) return c.st;
  c.array(a->buffer, size_of(a->dtype), "buffer");
  c.optional(a->weights, 4, "weights");
  c.array(a->out, size_of(a->dtype), "out");
  c.stride(a->out_stride, a->cols, a->tokens, "out");
  if (c.st) return c.st;
  return launched(launch_combine(*a, (hipStream_t)stream), c.call);
}

taccl_status_t taccl_combine_backward(const taccl_combine_backward_t *a, taccl_stream_t stream) {
  Check c{"taccl_combine_backward"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  check_buffer(c, *a);
  c.dtype(a->dtype);
  if (c.st) return c.st;
  const int64_t size = size_of(a->dtype);
  c.array(a->counts, 4, "counts");
  c.array(a->dbuffer, size, "dbuffer");
  if (a->tokens > 0) {
    c.array(a->dout, size, "dout");
    c.array(a->buffer, size, "buffer");
    c.array(a->weights, 4, "weights");
    c.array(a->dweights, 4, "dweights");
    c.stride(a->dout_stride, a->cols, a->tokens, "dout");
  }
  if (c.st) return c.st;
  int cus = 0;
  if (taccl_status_t st = device_cus(c.call, &cus)) return st;
  return launched(launch_combine_backward(*a, cus, (hipStream_t)stream), c.call);
}

taccl_status_t taccl_ffn(const taccl_ffn_t *a, taccl_stream_t stream) {
  Check c{"taccl_ffn"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  check_ffn(c, *a, false);
  if (c.st) return c.st;
  c.array(a->out, size_of(a->dtype), "out");
  c.optional(a->pre, size_of(a->dtype), "pre");
  if (c.st) return c.st;
  int cus = 0;
  if (taccl_status_t st = device_cus(c.call, &cus)) return st;
  return launched(launch_ffn(*a, cus, (hipStream_t)stream), c.call);
}

int64_t taccl_ffn_workspace(int32_t sources, int32_t num_experts, int64_t capacity, int32_t hidden,
                            int32_t dtype, int32_t backward) {
  Check c{"taccl_ffn_workspace"};
  check_ffn_sizes(c, FfnSizes{sources, num_experts, capacity, 1, hidden, dtype});
  return c.st ? 0 : ffn_space(sources, num_experts, capacity, hidden, dtype, backward != 0).bytes;
}

taccl_status_t taccl_ffn_backward(const taccl_ffn_backward_t *a, taccl_stream_t stream) {
  Check c{"taccl_ffn_backward"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  check_ffn(c, *a, true);
  if (c.st) return c.st;
  const int64_t size = size_of(a->dtype);
  c.array(a->dout, size, "dout");
  c.array(a->pre, size, "pre");
  c.optional(a->dbuffer, size, "dbuffer");
  c.optional(a->dw_in, size, "dw_in");
  c.optional(a->dw_out, size, "dw_out");
  c.invalid(!a->dbuffer && !a->dw_in && !a->dw_out, "no output");
  if (c.st) return c.st;
  int cus = 0;
  if (taccl_status_t st = device_cus(c.call, &cus)) return st;
  return launched(launch_ffn_backward(*a, cus, (hipStream_t)stream), c.call);
}

int64_t taccl_ffn_tokens_workspace(int64_t tokens, int32_t k, int32_t cols, int32_t hidden) {
  if (tokens < 0 || tokens > kFfnTokens || k < 1 || k > kMaxChoices || cols < 1 ||
      cols > kFfnMaxCols || hidden < 1 || hidden > kFfnMaxCols)
    return 0;
  return ffn_tokens_space(tokens, k, cols, hidden);
}

taccl_status_t taccl_ffn_tokens(const taccl_ffn_tokens_t *a, taccl_stream_t stream) {
  Check c{"taccl_ffn_tokens"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  c.invalid(a->tokens < 0, "negative number of tokens");
  c.limit(a->tokens > kFfnTokens, "more than 64 tokens");
  c.dtype(a->dtype);
  c.dtype(a->logits_dtype);
  c.experts(a->num_experts, a->k);
  c.invalid(a->k > a->num_experts, "more choices than experts");
  c.invalid(a->local_experts < 1, "no experts of its own");
  c.invalid(a->first_expert < 0 ||
                a->first_expert > (int64_t)a->num_experts - a->local_experts,
            "the experts of its own are not among the logits'");
  c.invalid(a->cols < 1 || a->hidden < 1, "cols and hidden must be at least 1");
  c.limit(a->cols > kFfnMaxCols || a->hidden > kFfnMaxCols, "more than 65536 columns");
  if (c.st || a->tokens == 0) return c.st;
  const int64_t size = size_of(a->dtype);
  c.array(a->x, size, "x");
  c.stride(a->x_stride, a->cols, a->tokens, "x");
  c.array(a->logits, size_of(a->logits_dtype), "logits");
  c.stride(a->logits_stride, a->num_experts, a->tokens, "logits");
  c.array(a->w_in, size, "w_in");
  c.array(a->w_out, size, "w_out");
  c.array(a->out, size, "out");
  c.stride(a->out_stride, a->cols, a->tokens, "out");
  c.optional(a->experts, 4, "experts");
  c.optional(a->weights, 4, "weights");
  c.workspace(a->workspace, a->workspace_bytes,
              ffn_tokens_space(a->tokens, a->k, a->cols, a->hidden));
  if (c.st) return c.st;
  int cus = 0;
  if (taccl_status_t st = device_cus(c.call, &cus)) return st;
  return launched(launch_ffn_tokens(*a, cus, (hipStream_t)stream), c.call);
}

taccl_status_t taccl_dropout(const taccl_dropout_t *a, taccl_stream_t stream) {
  Check c{"taccl_dropout"};
  c.invalid(!a, "null arguments");
  if (c.st) return c.st;
  c.rows(a->rows);
  c.dtype(a->dtype);
  c.invalid(a->cols < 1, "cols must be at least 1");
  c.limit(a->cols > kDropoutMaxCols, "more than 2^20 columns");
  c.invalid(!(a->p >= 0 && a->p <= 1), "p must be from 0 to 1");
  if (c.st || a->rows == 0) return c.st;
  const int64_t size = size_of(a->dtype);
  c.array(a->x, size, "x");
  c.optional(a->residual, size, "residual");
  c.array(a->rng, 8, "rng");
  c.array(a->out, size, "out");
  c.stride(a->x_stride, a->cols, a->rows, "x");
  if (a->residual) c.stride(a->residual_stride, a->cols, a->rows, "residual");
  c.stride(a->out_stride, a->cols, a->rows, "out");
  if (c.st) return c.st;
  return launched(launch_dropout(*a, (hipStream_t)stream), c.call);
}

}  // extern "C"
