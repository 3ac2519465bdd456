// Token rows into the expert buffer that an Alltoall sends (dispatch) and
// back (combine), with combine's gradient.
//
//   dispatch: out[e_j, s_j] = x[t];  combine: out[t] = sum_j w_j buf[e_j, s_j]
//   gradient: dbuf[e_j, s_j] = w_j dout[t],  dw_j = <dout[t], buf[e_j, s_j]>
//
// All three are bound by memory: a token's row is read (or written) once and
// each of its k buffer rows written (or read) once, in 16-byte units. A row
// whose length is no multiple of a unit has its last unit moved back to the
// row's end, so that it overlaps the one before and holds the same values.
//
// Measured, against 5.09 TB/s of a large copy:
//   dispatch of 16384 rows of 4096 bytes and 32 scales to 8 of 128 experts, 1280
//   rows each (762 MB): 148 us, 5.1 TB/s;
//   combine of 8192 x 8 rows of 4096 bf16, less those past the capacity (537 MB
//   by the counters): 111 us, 4.9 TB/s;
//   its gradient, 8192 x 6 rows of 2048 bf16 alike (453 MB): 94 us, 4.8 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "elem.h"
#include "expert.h"

namespace taccl {

namespace {

constexpr int kThreads = 256;

typedef uint32_t Bits16 __attribute__((ext_vector_type(4)));
typedef Bits16 Bits16u __attribute__((aligned(1)));

// Units of a row: `unit` bytes each (16, or an element in a shorter row)
struct RowUnits {
  int64_t bytes;
  int32_t unit, n;
};
RowUnits row_units(int64_t bytes, int element) {
  const int unit = bytes >= 16 ? 16 : element;
  return {bytes, unit, (int32_t)((bytes + unit - 1) / unit)};
}

__device__ __forceinline__ int64_t unit_at(const RowUnits &r, int u) {
  const int64_t at = (int64_t)u * r.unit;
  return at + r.unit > r.bytes ? r.bytes - r.unit : at;
}

// Row of choice (t, j) in the buffer, -1 without one
__device__ __forceinline__ int64_t choice_row(int e, int s, int E, int64_t C) {
  return (uint32_t)e < (uint32_t)E && s >= 0 && s < C ? (int64_t)e * C + s : -1;
}

__device__ __forceinline__ void store_unit(uint8_t *p, Bits16 v, int unit) {
  if (unit == 16) *(Bits16u *)p = v;
  else if (unit == 4) *(uint32_t *)p = v[0];
  else if (unit == 2) *(uint16_t *)p = (uint16_t)v[0];
  else *p = (uint8_t)v[0];
}
__device__ __forceinline__ Bits16 load_unit(const uint8_t *p, int unit) {
  Bits16 v = {0, 0, 0, 0};
  if (unit == 16) v = *(const Bits16u *)p;
  else if (unit == 4) v[0] = *(const uint32_t *)p;
  else if (unit == 2) v[0] = *(const uint16_t *)p;
  else v[0] = *p;
  return v;
}

// Rows of expert e from its count on, zeroed by block `part` of `parts`. They
// lie in one piece of memory, so the piece is dealt out by units: row by row
// the address arithmetic of a store took longer than the store.
__device__ __forceinline__ void zero_rows(uint8_t *out, const RowUnits &r, const int32_t *counts,
                                          int64_t C, int e, int part, int parts) {
  const int64_t from = min((int64_t)max(counts[e], 0), C);  // any 32-bit count
  const int64_t n = (C - from) * r.bytes;
  uint8_t *p = out + (e * C + from) * r.bytes;
  int64_t i = (int64_t)part * kThreads + threadIdx.x;
  const int64_t step = (int64_t)parts * kThreads;
  if (n < 16) {
    if (i < n) p[i] = 0;
    return;
  }
  const Bits16 zero = {0, 0, 0, 0};
  const int64_t units = n / 16;
  for (; i + 3 * step < units; i += 4 * step) {
#pragma unroll
    for (int j = 0; j < 4; j++) *(Bits16u *)(p + 16 * (i + j * step)) = zero;
  }
  for (; i < units; i += step) *(Bits16u *)(p + 16 * i) = zero;
  if (part == 0 && threadIdx.x == 0) *(Bits16u *)(p + n - 16) = zero;
}

// The rows of token t's choices, the same in all `lanes` threads of its group.
// From 16 threads on (kMaxChoices) thread j reads choice j and hands the row to
// the others: every thread reading every choice made most of a short row's
// memory instructions (18934 rows of 704 bytes to 7 experts each: 41 us, 33 so;
// combine of 32768 x 7 rows of 352 bf16: 48 and 42 us).
template <int kK, class A>
__device__ __forceinline__ void choice_rows(const A &a, int64_t t, int lanes, int64_t *rows) {
  if (lanes < kMaxChoices) {
#pragma unroll
    for (int j = 0; j < kK; j++)
      rows[j] = j < a.k ? choice_row(a.experts[t * a.k + j], a.slots[t * a.k + j], a.num_experts,
                                     a.capacity)
                        : -1;
    return;
  }
  const int lane = threadIdx.x & (min(lanes, 64) - 1), first = (threadIdx.x & 63) - lane;
  int64_t own = -1;
  if (lane < a.k)
    own = choice_row(a.experts[t * a.k + lane], a.slots[t * a.k + lane], a.num_experts, a.capacity);
#pragma unroll
  for (int j = 0; j < kK; j++) rows[j] = __shfl(own, first + j);
}

// The weights of token t's choices alike (1 without weights, 0 past the k-th)
template <int kK>
__device__ __forceinline__ void choice_weights(const float *weights, int k, int64_t t, int lanes,
                                               float *w) {
  if (lanes < kMaxChoices) {
#pragma unroll
    for (int j = 0; j < kK; j++) w[j] = j >= k ? 0.0f : weights ? weights[t * k + j] : 1.0f;
    return;
  }
  const int lane = threadIdx.x & (min(lanes, 64) - 1), first = (threadIdx.x & 63) - lane;
  const float own = lane >= k ? 0.0f : weights ? weights[t * k + lane] : 1.0f;
#pragma unroll
  for (int j = 0; j < kK; j++) w[j] = __shfl(own, first + j);
}

struct DispatchArgs {
  taccl_dispatch_t a;
  RowUnits row, scale;
  int lanes;        // threads per token row, a power of two up to kThreads
  int token_blocks;  // blocks that take tokens; the rest zero rows
  int parts;
};

template <int kK>
__global__ __launch_bounds__(kThreads) void dispatch_kernel(DispatchArgs g) {
  constexpr int kUnits = 4;  // units of a row on their way per thread
  const taccl_dispatch_t &a = g.a;
  if ((int)blockIdx.x >= g.token_blocks) {
    const int b = blockIdx.x - g.token_blocks, e = b % a.num_experts, part = b / a.num_experts;
    zero_rows((uint8_t *)a.out, g.row, a.counts, a.capacity, e, part, g.parts);
    if (g.scale.n)
      zero_rows((uint8_t *)a.out_scale, g.scale, a.counts, a.capacity, e, part, g.parts);
    return;
  }
  const int per = kThreads / g.lanes, lane = threadIdx.x & (g.lanes - 1);
  const int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / g.lanes;
  if (t >= a.tokens) return;
  int64_t to[kK];
  choice_rows<kK>(a, t, g.lanes, to);
  const uint8_t *x = (const uint8_t *)a.x + t * a.x_stride * a.element_bytes;
  uint8_t *out = (uint8_t *)a.out;
  // the scales' first units are on their way while the row is written
  const uint8_t *scale = (const uint8_t *)(a.scale + t * a.scale_stride);
  Bits16 first = {0, 0, 0, 0};
  if (lane < g.scale.n) first = load_unit(scale + unit_at(g.scale, lane), g.scale.unit);
  if (g.row.unit == 16) {
    for (int u0 = lane; u0 < g.row.n; u0 += kUnits * g.lanes) {
      Bits16 v[kUnits];
#pragma unroll
      for (int i = 0; i < kUnits; i++)
        if (u0 + i * g.lanes < g.row.n)
          v[i] = *(const Bits16u *)(x + unit_at(g.row, u0 + i * g.lanes));
#pragma unroll
      for (int j = 0; j < kK; j++)
        if (to[j] >= 0) {
#pragma unroll
          for (int i = 0; i < kUnits; i++)
            if (u0 + i * g.lanes < g.row.n)
              *(Bits16u *)(out + to[j] * g.row.bytes + unit_at(g.row, u0 + i * g.lanes)) = v[i];
        }
    }
  } else {
    for (int u = lane; u < g.row.n; u += g.lanes) {
      const int64_t at = unit_at(g.row, u);
      const Bits16 v = load_unit(x + at, g.row.unit);
#pragma unroll
      for (int j = 0; j < kK; j++)
        if (to[j] >= 0) store_unit(out + to[j] * g.row.bytes + at, v, g.row.unit);
    }
  }
  for (int u = lane; u < g.scale.n; u += g.lanes) {
    const int64_t at = unit_at(g.scale, u);
    const Bits16 v = u == lane ? first : load_unit(scale + at, g.scale.unit);
#pragma unroll
    for (int j = 0; j < kK; j++)
      if (to[j] >= 0)
        store_unit((uint8_t *)a.out_scale + to[j] * g.scale.bytes + at, v, g.scale.unit);
  }
}

struct CombineArgs {
  taccl_combine_t a;
  int lanes;  // threads per token row
};

template <class T, int kK, bool kShort>
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs g) {
  constexpr int N = Vec<T>::kN;
  const taccl_combine_t &a = g.a;
  const int per = kThreads / g.lanes, lane = threadIdx.x & (g.lanes - 1), D = a.cols;
  const int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / g.lanes;
  if (t >= a.tokens) return;
  int64_t from[kK];
  float w[kK];
  choice_rows<kK>(a, t, g.lanes, from);
  choice_weights<kK>(a.weights, a.k, t, g.lanes, w);
  for (int u = lane; u * N < D; u += g.lanes) {
    const int c = kShort ? 0 : min(u * N, D - N);
    float s[N];
#pragma unroll
    for (int i = 0; i < N; i++) s[i] = 0;
    typename Vec<T>::V v[kK];
#pragma unroll
    for (int j = 0; j < kK; j++)
      if (from[j] >= 0) v[j] = load_vec<T, kShort>((const T *)a.buffer + from[j] * D + c, D - c);
#pragma unroll
    for (int j = 0; j < kK; j++)
      if (from[j] >= 0) {
#pragma unroll
        for (int i = 0; i < N; i++) s[i] += w[j] * (float)v[j][i];
      }
    typename Vec<T>::V o;
#pragma unroll
    for (int i = 0; i < N; i++) o[i] = (T)s[i];
    store_vec<T, kShort>((T *)a.out + t * a.out_stride + c, o, D - c);
  }
}

struct CombineBackwardArgs {
  taccl_combine_backward_t a;
  RowUnits row;
  int token_blocks, parts;
};

// kLanes threads per token: part of a wavefront, one, or a block
template <class T, int kK, int kLanes, bool kShort>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(CombineBackwardArgs g) {
  constexpr int N = Vec<T>::kN, kTokens = kThreads / kLanes, kWaves = (kLanes + 63) / 64;
  __shared__ float red[kThreads / 64][kK];
  const taccl_combine_backward_t &a = g.a;
  if ((int)blockIdx.x >= g.token_blocks) {
    const int b = blockIdx.x - g.token_blocks;
    zero_rows((uint8_t *)a.dbuffer, g.row, a.counts, a.capacity, b % a.num_experts,
              b / a.num_experts, g.parts);
    return;
  }
  const int lane = threadIdx.x % kLanes, D = a.cols;
  const int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes;
  if (kWaves == 1 && t >= a.tokens) return;  // else a block is one token
  int64_t at[kK];
  float w[kK], dot[kK];
  choice_rows<kK>(a, t, kLanes, at);
  choice_weights<kK>(a.weights, a.k, t, kLanes, w);
#pragma unroll
  for (int j = 0; j < kK; j++) dot[j] = 0;
  for (int u = lane; u * N < D; u += kLanes) {
    const int c = kShort ? 0 : min(u * N, D - N), twice = u * N - c;
    const auto d = load_vec<T, kShort>((const T *)a.dout + t * a.dout_stride + c, D - c);
    float e[N];  // for the dot products: without the columns of the unit before
#pragma unroll
    for (int i = 0; i < N; i++) e[i] = i < twice ? 0.0f : (float)d[i];
    typename Vec<T>::V v[kK];
#pragma unroll
    for (int j = 0; j < kK; j++)
      if (at[j] >= 0) v[j] = load_vec<T, kShort>((const T *)a.buffer + at[j] * D + c, D - c);
#pragma unroll
    for (int j = 0; j < kK; j++)
      if (at[j] >= 0) {
        typename Vec<T>::V o;
#pragma unroll
        for (int i = 0; i < N; i++) {
          o[i] = (T)(w[j] * (float)d[i]);
          dot[j] += e[i] * (float)v[j][i];
        }
        store_vec<T, kShort>((T *)a.dbuffer + at[j] * D + c, o, D - c);
      }
  }
#pragma unroll
  for (int j = 0; j < kK; j++) dot[j] = lanes_sum<kLanes < 64 ? kLanes : 64>(dot[j]);
  if (kWaves > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int j = 0; j < kK; j++) red[threadIdx.x >> 6][j] = dot[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kK; j++)
      for (int i = 1; i < kWaves; i++) dot[j] = i == 1 ? red[0][j] + red[1][j] : dot[j] + red[i][j];
  }
#pragma unroll
  for (int j = 0; j < kK; j++)
    if (lane == j && j < a.k) a.dweights[t * a.k + j] = dot[j];
}

// Threads per token row: enough for one unit each, at most `most`
int row_lanes(int64_t units, int most) {
  int lanes = 1;
  while (lanes < most && lanes < units) lanes *= 2;
  return lanes;
}

// Blocks per expert that zero rows: about 16 per CU in all, behind the tokens'
// blocks (ahead of them: 154 us instead of 147 for the rows named above)
int zero_parts(int64_t capacity, int E, int cus) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(capacity, (16 * (int64_t)cus + E - 1) / E));
}

#define BY_CHOICES(k, F) \
  ((k) <= 1 ? F(1) : (k) <= 2 ? F(2) : (k) <= 4 ? F(4) : (k) <= 8 ? F(8) : F(16))

template <class T>
const void *combine_fn(int k, int cols) {
  const bool brief = cols < Vec<T>::kN;  // a row shorter than a unit
#define F(K)                                            \
  (brief ? (const void *)combine_kernel<T, K, true>     \
         : (const void *)combine_kernel<T, K, false>)
  return BY_CHOICES(k, F);
#undef F
}
// lanes: threads per token (16, 32, 64 or kThreads)
template <class T>
const void *combine_backward_fn(int k, int cols, int lanes) {
#define G(K, L) (const void *)combine_backward_kernel<T, K, L, false>
#define F(K)                                                                         \
  (cols < Vec<T>::kN ? (const void *)combine_backward_kernel<T, K, 16, true>         \
   : lanes == 16     ? G(K, 16)                                                      \
   : lanes == 32     ? G(K, 32)                                                      \
   : lanes == 64     ? G(K, 64)                                                      \
                     : G(K, kThreads))
  return BY_CHOICES(k, F);
#undef F
#undef G
}

}  // namespace

hipError_t launch_dispatch(const taccl_dispatch_t &a, int cus, hipStream_t stream) {
  DispatchArgs g{};
  g.a = a;
  g.row = row_units((int64_t)a.cols * a.element_bytes, a.element_bytes);
  if (a.scale_cols) g.scale = row_units(4 * (int64_t)a.scale_cols, 4);
  g.lanes = row_lanes(g.row.n, 128);
  const int64_t per = kThreads / g.lanes;
  g.token_blocks = (int)((a.tokens + per - 1) / per);
  g.parts = zero_parts(a.capacity, a.num_experts, cus);
#define F(K) (const void *)dispatch_kernel<K>
  const void *fn = BY_CHOICES(a.k, F);
#undef F
  void *args[] = {&g};
  return hipLaunchKernel(fn, dim3((uint32_t)g.token_blocks + (uint32_t)a.num_experts * g.parts),
                         dim3(kThreads), args, 0, stream);
}

hipError_t launch_combine(const taccl_combine_t &a, hipStream_t stream) {
  CombineArgs g{a, 1};
  const int n = a.dtype == TACCL_F32 ? 4 : 8;
  g.lanes = row_lanes((a.cols + n - 1) / n, kThreads);
  const int64_t per = kThreads / g.lanes;
  const void *fn = a.dtype == TACCL_F32    ? combine_fn<float>(a.k, a.cols)
                   : a.dtype == TACCL_BF16 ? combine_fn<bf16_t>(a.k, a.cols)
                                           : combine_fn<f16_t>(a.k, a.cols);
  void *args[] = {&g};
  return hipLaunchKernel(fn, dim3((uint32_t)((a.tokens + per - 1) / per)), dim3(kThreads), args, 0,
                         stream);
}

hipError_t launch_combine_backward(const taccl_combine_backward_t &a, int cus,
                                   hipStream_t stream) {
  CombineBackwardArgs g{a, {}, 0, 1};
  const int size = a.dtype == TACCL_F32 ? 4 : 2;
  g.row = row_units((int64_t)a.cols * size, size);
  // a unit per lane up to a wavefront, a block past two units each (8192 x 6 rows of
  // 2048 bf16: 103 us with a wavefront, 95 so; 8192 x 4 of 1111 f32: 86 and 76)
  const int lanes = g.row.n > 128 ? kThreads : std::max(16, row_lanes(g.row.n, 64));
  const int64_t per = kThreads / lanes;
  g.token_blocks = (int)((a.tokens + per - 1) / per);
  g.parts = zero_parts(a.capacity, a.num_experts, cus);
  const void *fn = a.dtype == TACCL_F32    ? combine_backward_fn<float>(a.k, a.cols, lanes)
                   : a.dtype == TACCL_BF16 ? combine_backward_fn<bf16_t>(a.k, a.cols, lanes)
                                           : combine_backward_fn<f16_t>(a.k, a.cols, lanes);
  void *args[] = {&g};
  return hipLaunchKernel(fn, dim3((uint32_t)g.token_blocks + (uint32_t)a.num_experts * g.parts),
                         dim3(kThreads), args, 0, stream);
}

}  // namespace taccl
