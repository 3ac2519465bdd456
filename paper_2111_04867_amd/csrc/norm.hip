// Root-mean-square norm of rows after the residual's addition, with an 8-bit
// copy, and its gradient.
//
//   h = x + residual, r = 1 / sqrt(mean(h^2) + eps), y = w h r
//   dx = dtotal + r a - h r^3 mean(a h) with a = w dy;  dw = sum_t dy h r
//
// A row is held in registers between its two passes (statistics, outputs), so
// memory is read and written once: kTpr threads per row, kNv vectors of 16
// bytes each.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "elem.h"
#include "expert.h"

namespace taccl {

namespace {

constexpr float kF8Max = 448.0f;
constexpr float kAmaxMin = 0x1p-100f;

constexpr int block_threads(int tpr) { return tpr > 256 ? tpr : 256; }

// Sum of v, and maximum of m, over the kTpr threads of a row. `red`: two
// floats per wavefront; rows in turn alternate between two of them, so one
// barrier per row is enough.
template <int kTpr, bool kMax>
__device__ __forceinline__ void row_reduce(float &v, float &m, float *red) {
  constexpr int L = kTpr < 64 ? 16 : 64;
  v = lanes_sum<L>(v);
  if (kMax) m = lanes_max<L>(m);
  else m = lanes_sum<L>(m);
  if (kTpr <= 64) return;
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[2 * w] = v;
    red[2 * w + 1] = m;
  }
  __syncthreads();
  v = red[0];
  m = red[1];
#pragma unroll
  for (int i = 1; i < kTpr / 64; i++) {
    v += red[2 * i];
    m = kMax ? fmaxf(m, red[2 * i + 1]) : m + red[2 * i + 1];
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

// N floats to e4m3, stored at p (columns from `left` on are not)
template <int N, bool kTail>
__device__ __forceinline__ void store_f8(uint8_t *p, const float *y, float inv, int left) {
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; i++) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i] * inv, y[4 * i + 1] * inv, 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2] * inv, y[4 * i + 3] * inv, x, true);
  }
  typedef uint32_t V __attribute__((ext_vector_type(N / 4)));
  typedef V U __attribute__((aligned(1)));
  if (left >= N) {
    V v;
#pragma unroll
    for (int i = 0; i < N / 4; i++) v[i] = w[i];
    *(U *)p = v;
  } else if (kTail) {
#pragma unroll
    for (int i = 0; i < N; i++)
      if (i < left) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

template <class T, int kTpr, int kNv, bool kTail>
__global__ __launch_bounds__(block_threads(kTpr)) void norm_kernel(taccl_norm_t a) {
  constexpr int N = Vec<T>::kN, kRows = block_threads(kTpr) / kTpr;
  __shared__ float red[2 * (kTpr / 64 + 1)];
  const int lane = threadIdx.x % kTpr, D = a.cols;
  const int64_t at = (int64_t)blockIdx.x * kRows + threadIdx.x / kTpr;
  const bool live = at < a.rows;
  const int64_t row = live ? at : a.rows - 1;  // rows past the end: computed, not stored
  const T *x = (const T *)a.x + row * a.x_stride;
  const T *res = a.residual ? (const T *)a.residual + row * a.residual_stride : nullptr;
  float h[kNv][N];
  typename Vec<T>::V wv[kNv];
#pragma unroll
  for (int j = 0; j < kNv; j++) {
    const int c = N * (lane + kTpr * j);
    const auto v = load_vec<T, kTail>(x + c, D - c);
#pragma unroll
    for (int i = 0; i < N; i++) h[j][i] = (float)v[i];
    if (res) {
      const auto r = load_vec<T, kTail>(res + c, D - c);
#pragma unroll
      for (int i = 0; i < N; i++) h[j][i] += (float)r[i];
    }
    wv[j] = load_vec<T, kTail>((const T *)a.weight + c, D - c);
  }
  float ss = 0, most = 0;
#pragma unroll
  for (int j = 0; j < kNv; j++)
#pragma unroll
    for (int i = 0; i < N; i++) {
      ss += h[j][i] * h[j][i];
      most = fmaxf(most, fabsf(h[j][i] * (float)wv[j][i]));
    }
  row_reduce<kTpr, true>(ss, most, red);
  const float r = 1.0f / sqrtf(ss / (float)D + a.eps);
  const int group = a.group && a.group < D ? a.group : 0;
#pragma unroll
  for (int j = 0; j < kNv; j++) {
    const int c = N * (lane + kTpr * j), left = live ? D - c : 0;
    if (a.total) {
      typename Vec<T>::V v;
#pragma unroll
      for (int i = 0; i < N; i++) v[i] = (T)h[j][i];
      store_vec<T, kTail>((T *)a.total + row * a.total_stride + c, v, left);
    }
    float y[N];
    typename Vec<T>::V v;
#pragma unroll
    for (int i = 0; i < N; i++) {
      y[i] = h[j][i] * r * (float)wv[j][i];
      v[i] = (T)y[i];
    }
    if (a.out) store_vec<T, kTail>((T *)a.out + row * a.out_stride + c, v, left);
    if (a.q) {
      float m = most * r;
      if (group) {
        m = 0;
#pragma unroll
        for (int i = 0; i < N; i++) m = fmaxf(m, fabsf(y[i]));
        m = group_max(m, group / N);
      }
      m = fminf(fmaxf(m, kAmaxMin), 3.4028234664e38f);
      store_f8<N, kTail>(a.q + row * a.q_stride + c, y, kF8Max / m, left);
      if (group ? left > 0 && c % group == 0 : live && c == 0)
        a.scale[row * a.scale_stride + (group ? c / group : 0)] = m / kF8Max;
    }
  }
}

// Gradient: blocks take rows in turn; each thread sums its columns of dw
// over its rows, and a block's sums go to one row of `partial`.
template <class T, int kTpr, int kNv, bool kTail>
__global__ __launch_bounds__(block_threads(kTpr)) void norm_backward_kernel(
    taccl_norm_backward_t a, float *partial) {
  constexpr int N = Vec<T>::kN, kRows = block_threads(kTpr) / kTpr;
  __shared__ float red[2][2 * (kTpr / 64 + 1)];
  __shared__ float sums[kRows > 1 ? kTpr * kNv * N : 1];
  const int lane = threadIdx.x % kTpr, sub = threadIdx.x / kTpr, D = a.cols;
  typename Vec<T>::V wv[kNv];
  float acc[kNv][N];
#pragma unroll
  for (int j = 0; j < kNv; j++) {
    const int c = N * (lane + kTpr * j);
    wv[j] = load_vec<T, kTail>((const T *)a.weight + c, D - c);
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
    typename Vec<T>::V dv[kNv], hv[kNv];
    float ss = 0, dot = 0;
#pragma unroll
    for (int j = 0; j < kNv; j++) {
      const int c = N * (lane + kTpr * j);
      dv[j] = load_vec<T, kTail>(dy + c, D - c);
      hv[j] = load_vec<T, kTail>(h + c, D - c);
    }
#pragma unroll
    for (int j = 0; j < kNv; j++)
#pragma unroll
      for (int i = 0; i < N; i++) {
        const float x = (float)hv[j][i];
        ss += x * x;
        dot += x * ((float)dv[j][i] * (float)wv[j][i]);
      }
    row_reduce<kTpr, false>(ss, dot, red[turn]);
    const float r = 1.0f / sqrtf(ss / (float)D + a.eps);
    const float f = r * r * r * (dot / (float)D);
#pragma unroll
    for (int j = 0; j < kNv; j++) {
      const int c = N * (lane + kTpr * j), left = live ? D - c : 0;
      typename Vec<T>::V o, t;
      if (a.dtotal) t = load_vec<T, kTail>((const T *)a.dtotal + row * a.dtotal_stride + c, left);
#pragma unroll
      for (int i = 0; i < N; i++) {
        const float x = (float)hv[j][i], d = (float)dv[j][i];
        float g = r * (d * (float)wv[j][i]) - x * f;
        if (a.dtotal) g += (float)t[i];
        o[i] = (T)g;
        if (live) acc[j][i] += d * (x * r);
      }
      store_vec<T, kTail>((T *)a.dx + row * a.dx_stride + c, o, left);
    }
  }
  float *out = partial + (int64_t)blockIdx.x * D;
  if (kRows == 1) {
#pragma unroll
    for (int j = 0; j < kNv; j++)
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int c = N * (lane + kTpr * j) + i;
        if (c < D) out[c] = acc[j][i];
      }
    return;
  }
  for (int s = 0; s < kRows; s++) {  // the rows' sums in order
    if (sub == s) {
#pragma unroll
      for (int j = 0; j < kNv; j++)
#pragma unroll
        for (int i = 0; i < N; i++) {
          const int c = N * (lane + kTpr * j) + i;
          sums[c] = s ? sums[c] + acc[j][i] : acc[j][i];
        }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < D; c += blockDim.x) out[c] = sums[c];
}

// Columns of `partial` [n][cols] summed in a fixed order: 64 columns per
// block, 16 rows at a time.
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *partial, int n, int cols,
                                                           float *out) {
  __shared__ float part[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
  float s = 0;
  if (c < cols)
    for (int i = slice; i < n; i += 16) s += partial[(int64_t)i * cols + c];
  part[slice][threadIdx.x & 63] = s;
  __syncthreads();
  if (slice == 0 && c < cols) {
    for (int i = 1; i < 16; i++) s += part[i][threadIdx.x];
    out[c] = s;
  }
}

// The threads per row and vectors per thread that hold a row of `cols`
struct RowShape {
  int tpr, nv;
};
template <class T>
RowShape row_shape(int cols) {
  const int v = (cols + Vec<T>::kN - 1) / Vec<T>::kN;
  if (v <= 16) return {16, 1};
  if (v <= 64) return {64, 1};
  if (v <= 128) return {64, 2};
  if (v <= 256) return {256, 1};
  if (v <= 512) return {256, 2};
  if (v <= 1024) return {256, 4};
  if (v <= 2048) return {512, 4};
  return {512, 8};  // 32-bit rows only
}

#define NORM_SHAPES(F) F(16, 1) F(64, 1) F(64, 2) F(256, 1) F(256, 2) F(256, 4) F(512, 4)

template <class T, bool kTail>
const void *norm_fn(RowShape s, bool backward) {
#define PICK(TPR, NV)                                                    \
  if (s.tpr == TPR && s.nv == NV)                                        \
    return backward ? (const void *)norm_backward_kernel<T, TPR, NV, kTail> \
                    : (const void *)norm_kernel<T, TPR, NV, kTail>;
  NORM_SHAPES(PICK)
  if constexpr (sizeof(T) == 4) {
    PICK(512, 8)
  }
#undef PICK
  return nullptr;
}

template <class T>
const void *norm_pick_type(int cols, bool backward, RowShape &s) {
  s = row_shape<T>(cols);
  return cols % Vec<T>::kN ? norm_fn<T, true>(s, backward) : norm_fn<T, false>(s, backward);
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
  const int threads = block_threads(s.tpr), per = threads / s.tpr;
  const int grid = (int)std::max<int64_t>(
      1, std::min<int64_t>({(a.rows + per - 1) / per, (int64_t)cus * 2, kNormMaxBlocks}));
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
