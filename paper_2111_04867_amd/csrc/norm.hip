// Root-mean-square norm of rows after the residual's addition, with an 8-bit
// copy, and its gradient.
//
//   h = x + residual, r = 1 / sqrt(mean(h^2) + eps), y = w h r
//   dx = dtotal + r (a - u mean(a u)) with a = w dy, u = h r;  dw = sum_t dy u
//
// A row is held in registers between its two passes (statistics, outputs), so
// memory is read and written once: kTpr threads per row, kNv vectors of 16
// bytes each. Both kernels are bound by memory.
//
// Forward: one vector per thread as far as a block reaches. 8192 x 4096 bf16
// with residual and 8-bit copy (303 MB): 57 us a call (5.3 TB/s; a large copy
// 5.1), vector instructions busy 90% of it, most of them the divisions of the
// 8-bit copy. 512 threads took 58 us where 256 with two vectors took 63.5, 128
// with four 68.4 and a wavefront with eight 80.6 (with products by a reciprocal
// in the divisions' place): what counts is wavefronts in flight.
// Gradient: four vectors per thread, so that a block of two to eight rows needs
// few partial sums of dw, and 16-bit rows stay as they are stored (as_stored).
// 8192 x 2048 bf16: 29.7 us for both launches (134 MB; in a trace 27.0 us the
// first and 4.6 the second, on average), a block per row 36 us; 8192 x 4096: 55.9
// us with 128 threads per row, where 256 took 3 us more and a wavefront 16.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "elem.h"
#include "expert.h"

namespace taccl {

namespace {

constexpr float kF8Max = 448.0f;
constexpr float kAmaxMin = 0x1p-100f;

constexpr int block_threads(int tpr) { return tpr > 256 ? tpr : 256; }
// The gradient's blocks: eight rows at a time where a wavefront takes one, one
// block per CU (31.1 us for 8192 x 2048 bf16 with two blocks of four rows, 29.9
// so); wider rows two blocks of 256 threads (8192 x 4096: 55.1 us, 57.4 with one
// of 512).
constexpr int back_threads(int tpr) { return tpr <= 64 || tpr > 256 ? 512 : 256; }

// Sum or maximum of v over the kTpr threads of a row. `red`: a float per
// wavefront.
template <int kTpr, bool kMax>
__device__ __forceinline__ float row_reduce(float v, float *red) {
  constexpr int L = kTpr < 64 ? kTpr : 64;
  v = kMax ? lanes_max<L>(v) : lanes_sum<L>(v);
  if (kTpr <= 64) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  red += threadIdx.x / kTpr * (kTpr / 64);
  v = red[0];
#pragma unroll
  for (int i = 1; i < kTpr / 64; i++) v = kMax ? fmaxf(v, red[i]) : v + red[i];
  return v;
}

// Sums of v and m over the kTpr threads of a row. `red`: two floats per
// wavefront; rows in turn alternate between two of them, so one barrier per row
// is enough.
template <int kTpr>
__device__ __forceinline__ void row_sums(float &v, float &m, float *red) {
  constexpr int L = kTpr < 64 ? kTpr : 64;
  v = lanes_sum<L>(v);
  m = lanes_sum<L>(m);
  if (kTpr <= 64) return;
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[2 * w] = v;
    red[2 * w + 1] = m;
  }
  __syncthreads();
  red += 2 * (threadIdx.x / kTpr * (kTpr / 64));
  v = red[0];
  m = red[1];
#pragma unroll
  for (int i = 1; i < kTpr / 64; i++) {
    v += red[2 * i];
    m += red[2 * i + 1];
  }
}

// Maximum over groups of `lanes` (4, 8, 16, 32 or 64) consecutive lanes.
__device__ __forceinline__ float group_max(float v, int lanes) {
  v = fmaxf(v, dppf<kXor1>(v));
  v = fmaxf(v, dppf<kXor2>(v));
  if (lanes > 4) v = fmaxf(v, dppf<kHalfMirror>(v));
  if (lanes > 8) v = fmaxf(v, dppf<kMirror>(v));
  if (lanes > 16) v = fmaxf(v, __shfl_xor(v, 16));
  if (lanes > 32) v = fmaxf(v, __shfl_xor(v, 32));
  return v;
}

// N floats over `scale` in e4m3, stored at p; only elements first to end - 1 of
// them where those are not all. The quotient itself is rounded: a product with
// the scale's rounded reciprocal is another e4m3 number for 1 in 2e6 values of
// 32-bit rows and for 1 in 1e5 of 16-bit ones, which have more ties.
template <int N, bool kPart>
__device__ __forceinline__ void store_f8(uint8_t *p, const float *y, float scale, int first,
                                         int end) {
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; i++) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i] / scale, y[4 * i + 1] / scale, 0, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2] / scale, y[4 * i + 3] / scale, x, true);
    w[i] = (uint32_t)x;
  }
  typedef uint32_t V __attribute__((ext_vector_type(N / 4)));
  typedef V U __attribute__((aligned(1)));
  if (first == 0 && end >= N) {
    V v;
#pragma unroll
    for (int i = 0; i < N / 4; i++) v[i] = w[i];
    *(U *)p = v;
  } else if (kPart) {
#pragma unroll
    for (int i = 0; i < N; i++)
      if (i >= first && i < end) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// How a row ends: with a whole vector; with one that is moved back to end
// there, so that its first columns are another thread's too (they count once
// and are stored twice, alike: reading and writing a last vector in pieces,
// behind branches, took 7 us more for 8192 rows of 2004 columns); or before the
// first vector does.
enum RowEnd { kWhole, kMoved, kShort };

template <class T, int kTpr, int kNv, RowEnd kEnd>
__global__ __launch_bounds__(block_threads(kTpr)) void norm_kernel(taccl_norm_t a) {
  constexpr int N = Vec<T>::kN, kRows = block_threads(kTpr) / kTpr;
  __shared__ float red[2][block_threads(kTpr) / 64];
  const int lane = threadIdx.x % kTpr, D = a.cols;
  const int64_t at = (int64_t)blockIdx.x * kRows + threadIdx.x / kTpr;
  const bool live = at < a.rows;
  const int64_t row = live ? at : a.rows - 1;  // rows past the end: computed, not stored
  const T *x = (const T *)a.x + row * a.x_stride;
  const T *res = a.residual ? (const T *)a.residual + row * a.residual_stride : nullptr;
  // the columns of vector j: from `col`, `left` of them in the row (0: none),
  // the first `twice` of them the vector's before
  int col[kNv], left[kNv], twice[kNv];
  float h[kNv][N];
  typename Vec<T>::V wv[kNv];
#pragma unroll
  for (int j = 0; j < kNv; j++) {
    const int c = N * (lane + kTpr * j);
    col[j] = kEnd == kMoved ? min(c, D - N) : c;
    twice[j] = kEnd == kMoved ? c - col[j] : 0;
    left[j] = c < D ? D - col[j] : 0;
    const auto v = load_vec<T, kEnd == kShort>(x + col[j], left[j]);
#pragma unroll
    for (int i = 0; i < N; i++) h[j][i] = (float)v[i];
    if (res) {
      const auto r = load_vec<T, kEnd == kShort>(res + col[j], left[j]);
#pragma unroll
      for (int i = 0; i < N; i++) h[j][i] += (float)r[i];
    }
    wv[j] = load_vec<T, kEnd == kShort>((const T *)a.weight + col[j], left[j]);
  }
  float ss = 0;
#pragma unroll
  for (int j = 0; j < kNv; j++)
#pragma unroll
    for (int i = 0; i < N; i++) {
      const float once = kEnd == kMoved && i < twice[j] ? 0.0f : h[j][i];
      ss += once * once;
    }
  ss = row_reduce<kTpr, false>(ss, red[0]);
  const float r = 1.0f / sqrtf(ss / (float)D + a.eps);
  const int group = a.group && a.group < D ? a.group : 0;
  // one scale per row is by the values themselves: the maximum of h w, taken
  // with the sum and times r, rounds otherwise and can leave y's range
  float most = 0;
  if (a.q && !group) {
#pragma unroll
    for (int j = 0; j < kNv; j++)
#pragma unroll
      for (int i = 0; i < N; i++) most = fmaxf(most, fabsf(h[j][i] * r * (float)wv[j][i]));
    most = row_reduce<kTpr, true>(most, red[1]);
  }
#pragma unroll
  for (int j = 0; j < kNv; j++) {
    const int c = col[j], n = live ? left[j] : 0;
    if (a.total) {
      typename Vec<T>::V v;
#pragma unroll
      for (int i = 0; i < N; i++) v[i] = (T)h[j][i];
      store_vec<T, kEnd == kShort>((T *)a.total + row * a.total_stride + c, v, n);
    }
    float y[N];
    typename Vec<T>::V v;
#pragma unroll
    for (int i = 0; i < N; i++) {
      y[i] = h[j][i] * r * (float)wv[j][i];
      v[i] = (T)y[i];
    }
    if (a.out) store_vec<T, kEnd == kShort>((T *)a.out + row * a.out_stride + c, v, n);
    if (a.q) {
      const int c0 = N * (lane + kTpr * j);
      float m = most;
      int first = 0;
      if (group) {
        m = 0;
#pragma unroll
        for (int i = 0; i < N; i++)
          m = fmaxf(m, kEnd == kMoved && i < twice[j] ? 0.0f : fabsf(y[i]));
        m = group_max(m, group / N);
        // columns of the group before keep their own scale
        if (kEnd == kMoved && c0 % group == 0) first = twice[j];
      }
      const float scale = fminf(fmaxf(m, kAmaxMin), 3.4028234664e38f) / kF8Max;
      store_f8<N, kEnd != kWhole>(a.q + row * a.q_stride + c, y, scale, first, n);
      if (group ? n > 0 && c0 % group == 0 : live && c0 == 0)
        a.scale[row * a.scale_stride + (group ? c0 / group : 0)] = scale;
    }
  }
}

// Gradient: blocks take rows in turn; each thread sums its columns of dw
// over its rows, and a block's sums go to one row of `partial`. Columns past
// the last whole vector (kTail) go to the row's first lanes, one each: their
// vector in pieces, behind branches among the loads, took 4 us more for 3001
// rows of 1999 columns.
template <class T, int kTpr, int kNv, bool kTail>
__global__ __launch_bounds__(back_threads(kTpr)) void norm_backward_kernel(
    taccl_norm_backward_t a, float *partial) {
  constexpr int N = Vec<T>::kN, kRows = back_threads(kTpr) / kTpr;
  __shared__ float red[2][2 * (back_threads(kTpr) / 64)];
  constexpr int kCols = kTpr * kNv * N;
  __shared__ __align__(16) float sums[kRows > 1 ? kRows * kCols : 1];
  __shared__ float tail[kRows][N];
  const int lane = threadIdx.x % kTpr, sub = threadIdx.x / kTpr;
  const int D = a.cols, whole = kTail ? D / N * N : D;
  const bool more = kTail && lane < D - whole;  // has column whole + lane
  const T *w = (const T *)a.weight;
  typename Vec<T>::V wv[kNv];
  float acc[kNv][N], acc1 = 0;
  const float w1 = more ? (float)w[whole + lane] : 0.0f;
#pragma unroll
  for (int j = 0; j < kNv; j++) {
    const int c = N * (lane + kTpr * j);
    wv[j] = load_vec<T, false>(w + c, whole - c);
#pragma unroll
    for (int i = 0; i < N; i++) acc[j][i] = 0;
  }
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.rows;
       first += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const bool live = first + sub < a.rows;
    const int64_t row = live ? first + sub : a.rows - 1;
    const T *dy = (const T *)a.dout + row * a.dout_stride;
    const T *h = (const T *)a.h + row * a.h_stride;
    const T *dt = a.dtotal ? (const T *)a.dtotal + row * a.dtotal_stride : nullptr;
    T *dx = (T *)a.dx + row * a.dx_stride;
    typename Vec<T>::V dv[kNv], hv[kNv], tv[kNv];
    float ss = 0, dot = 0, d1 = 0, h1 = 0, t1 = 0;
#pragma unroll
    for (int j = 0; j < kNv; j++) {
      const int c = N * (lane + kTpr * j);
      dv[j] = load_vec<T, false>(dy + c, whole - c);
      hv[j] = load_vec<T, false>(h + c, whole - c);
    }
    if (dt) {
#pragma unroll
      for (int j = 0; j < kNv; j++) {
        const int c = N * (lane + kTpr * j);
        tv[j] = load_vec<T, false>(dt + c, whole - c);
      }
    }
    if (more) {
      d1 = (float)dy[whole + lane];
      h1 = (float)h[whole + lane];
      if (dt) t1 = (float)dt[whole + lane];
    }
#pragma unroll
    for (int j = 0; j < kNv; j++)
#pragma unroll
      for (int i = 0; i < N; i++) {
        const float x = (float)hv[j][i];
        ss += x * x;
        dot += x * ((float)dv[j][i] * (float)wv[j][i]);
      }
    if (kTail) {
      ss += h1 * h1;
      dot += h1 * (d1 * w1);
    }
#pragma unroll
    for (int j = 0; j < kNv; j++) {
      as_stored(dv[j]);
      as_stored(hv[j]);
      as_stored(wv[j]);
    }
    row_sums<kTpr>(ss, dot, red[turn]);
    const float r = 1.0f / sqrtf(ss / (float)D + a.eps);
    // h r^3 mean(a h) as (h r) (r mean(a h)): the cube leaves the range from rows
    // of 1e13 (or of 1e-13 without eps) on, these factors stay within it
    const float f = dot * r / (float)D;
#pragma unroll
    for (int j = 0; j < kNv; j++) {
      const int c = N * (lane + kTpr * j);
      typename Vec<T>::V o;
#pragma unroll
      for (int i = 0; i < N; i++) {
        const float x = (float)hv[j][i], d = (float)dv[j][i];
        const float u = x * r;
        float g = r * (d * (float)wv[j][i] - u * f);
        if (dt) g += (float)tv[j][i];
        o[i] = (T)g;
        if (live) acc[j][i] += d * u;
      }
      store_vec<T, false>(dx + c, o, live ? whole - c : 0);
    }
    if (more && live) {
      const float u1 = h1 * r;
      dx[whole + lane] = (T)(r * (d1 * w1 - u1 * f) + t1);
      acc1 += d1 * u1;
    }
  }
  float *out = partial + (int64_t)blockIdx.x * D;
  if (kRows == 1) {
#pragma unroll
    for (int j = 0; j < kNv; j++) {
      const int c = N * (lane + kTpr * j);
      if (c < whole) {
#pragma unroll
        for (int i = 0; i < N; i++) out[c + i] = acc[j][i];
      }
    }
    if (more) out[whole + lane] = acc1;
    return;
  }
  // the sums of the block's rows, in order
  float *own = sums + sub * kCols;
#pragma unroll
  for (int j = 0; j < kNv; j++)
#pragma unroll
    for (int i = 0; i < N; i++) own[N * (lane + kTpr * j) + i] = acc[j][i];
  if (more) tail[sub][lane] = acc1;
  __syncthreads();
  for (int c = threadIdx.x; c < D; c += blockDim.x) {
    float s = 0;
#pragma unroll
    for (int i = 0; i < kRows; i++) s += c < whole ? sums[i * kCols + c] : tail[i][c - whole];
    out[c] = s;
  }
}

// Columns of `partial` [n][cols] summed in a fixed order: 64 columns per
// block, 64 rows at a time, four of them on their way per thread.
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *partial, int n, int cols,
                                                           float *out) {
  __shared__ float part[64][64];
  const int c = blockIdx.x * 64 + 4 * (threadIdx.x & 15), slice = threadIdx.x >> 4;
  float s[4] = {0, 0, 0, 0};
  for (int i = slice; i < n; i += 256) {
    Vec<float>::V v[4];
#pragma unroll
    for (int j = 0; j < 4; j++)
      v[j] = load_vec<float, true>(partial + (int64_t)min(i + 64 * j, n - 1) * cols + c, cols - c);
#pragma unroll
    for (int j = 0; j < 4; j++)
      if (i + 64 * j < n) {
#pragma unroll
        for (int x = 0; x < 4; x++) s[x] += v[j][x];
      }
  }
#pragma unroll
  for (int x = 0; x < 4; x++) part[slice][4 * (threadIdx.x & 15) + x] = s[x];
  __syncthreads();
  const int col = threadIdx.x & 63, w = threadIdx.x >> 6;
  float t = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) t += part[4 * w + i][col];
  __syncthreads();
  part[w][col] = t;
  __syncthreads();
  if (w == 0 && blockIdx.x * 64 + col < cols) {
    for (int i = 1; i < 16; i++) t += part[i][col];
    out[blockIdx.x * 64 + col] = t;
  }
}

// The threads per row and vectors per thread that hold a row of `cols`
struct RowShape {
  int tpr, nv;
};
template <class T>
RowShape row_shape(int cols, bool backward) {
  const int v = (cols + Vec<T>::kN - 1) / Vec<T>::kN;
  if (v <= 16) return {16, 1};
  if (v <= 32) return {32, 1};
  if (v <= 64) return {64, 1};
  if (backward) {
    if (v <= 128) return {64, 2};
    if (v <= 256) return {64, 4};
    if (v <= 512) return {128, 4};
    if (v <= 1024) return {256, 4};
    if (v <= 2048) return {512, 4};
    return {512, 8};  // 32-bit rows only
  }
  if (v <= 128) return {128, 1};
  if (v <= 256) return {256, 1};
  if (v <= 512) return {512, 1};
  if (v <= 1024) return {1024, 1};
  if (v <= 2048) return {1024, 2};
  return {1024, 4};  // 32-bit rows only
}

template <class T>
const void *norm_fn(RowShape s, int cols) {
  if (cols < Vec<T>::kN) return (const void *)norm_kernel<T, 16, 1, kShort>;
  const bool whole = cols % Vec<T>::kN == 0;
#define PICK(TPR, NV)                                                            \
  if (s.tpr == TPR && s.nv == NV)                                                \
    return whole ? (const void *)norm_kernel<T, TPR, NV, kWhole>                 \
                 : (const void *)norm_kernel<T, TPR, NV, kMoved>;
  PICK(16, 1) PICK(32, 1) PICK(64, 1) PICK(128, 1) PICK(256, 1) PICK(512, 1) PICK(1024, 1) PICK(1024, 2)
  if constexpr (sizeof(T) == 4) {
    PICK(1024, 4)
  }
#undef PICK
  return nullptr;
}
template <class T, bool kTail>
const void *norm_backward_fn(RowShape s) {
#define PICK(TPR, NV) \
  if (s.tpr == TPR && s.nv == NV) return (const void *)norm_backward_kernel<T, TPR, NV, kTail>;
  PICK(16, 1) PICK(32, 1) PICK(64, 1) PICK(64, 2) PICK(64, 4) PICK(128, 4) PICK(256, 4) PICK(512, 4)
  if constexpr (sizeof(T) == 4) {
    PICK(512, 8)
  }
#undef PICK
  return nullptr;
}

template <class T>
const void *norm_pick_type(int cols, bool backward, RowShape &s) {
  s = row_shape<T>(cols, backward);
  if (!backward) return norm_fn<T>(s, cols);
  return cols % Vec<T>::kN ? norm_backward_fn<T, true>(s) : norm_backward_fn<T, false>(s);
}

const void *norm_pick(int dtype, int cols, bool backward, RowShape &s) {
  if (dtype == TACCL_F32) return norm_pick_type<float>(cols, backward, s);
  if (dtype == TACCL_BF16) return norm_pick_type<bf16_t>(cols, backward, s);
  return norm_pick_type<f16_t>(cols, backward, s);
}

}  // namespace

hipError_t launch_norm(const taccl_norm_t &a, hipStream_t stream) {
  RowShape s;
  const void *fn = norm_pick(a.dtype, a.cols, false, s);
  const int threads = block_threads(s.tpr), per = threads / s.tpr;
  void *args[] = {(void *)&a};
  return hipLaunchKernel(fn, dim3((uint32_t)((a.rows + per - 1) / per)), dim3(threads), args, 0,
                         stream);
}

hipError_t launch_norm_backward(const taccl_norm_backward_t &a, int cus, hipStream_t stream) {
  RowShape s;
  const void *fn = norm_pick(a.dtype, a.cols, true, s);
  const int threads = back_threads(s.tpr), per = threads / s.tpr;
  const int64_t most = std::min<int64_t>((int64_t)cus * (s.tpr <= 64 ? 1 : 2), kNormMaxBlocks);
  const int grid = (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + per - 1) / per, most));
  float *partial = grid == 1 ? a.dweight : (float *)a.workspace;
  void *args[] = {(void *)&a, &partial};
  hipError_t e = hipLaunchKernel(fn, dim3(grid), dim3(threads), args, 0, stream);
  if (e != hipSuccess || grid == 1) return e;
  const float *from = partial;
  int n = grid, cols = a.cols;
  float *out = a.dweight;
  void *sum_args[] = {&from, &n, &cols, &out};
  return hipLaunchKernel((const void *)column_sums_kernel, dim3((cols + 63) / 64), dim3(1024),
                         sum_args, 0, stream);
}

}  // namespace taccl
