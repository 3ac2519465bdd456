// C ABI of the expert-layer operators: checks of arguments and launches.
#include <hip/hip_runtime.h>

#include <atomic>
#include <string>

#include "expert.h"
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

}  // extern "C"
