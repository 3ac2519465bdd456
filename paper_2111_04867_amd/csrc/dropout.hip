// Dropout of rows with the residual's addition; its gradient is the same call
// on the gradient's rows, without a residual.
//
//   out = residual + (kept ? x / (1 - p) : 0)
//
// The random numbers are SplitMix64's outputs for a counter (workloads/candgen.c
// draws its candidates the same way), so no mask is stored: two columns share a
// 64-bit word, whose halves are compared with ceil(p 2^32). The generator's two
// 64-bit products per pair stay behind memory: 8192 x 4096 bf16 with a residual
// (201 MB) take 38 us, 5.3 TB/s, where a large copy reaches 5.0.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "elem.h"
#include "ffn.h"

namespace taccl {

namespace {

constexpr int kThreads = 256;
// a grid has fewer than 2^32 threads
constexpr int64_t kMaxBlocks = 1 << 23;

struct DropoutArgs {
  taccl_dropout_t a;
  uint32_t below;  // fields below it are dropped
  bool all;        // every value is
  float scale;
  int lanes;       // threads per row, a power of two up to kThreads
  int per_row;     // blocks per row (rows of more units than kThreads)
  int64_t first;   // the launch's first row
};

// The (at + 1)-th output of the SplitMix64 stream of `seed` (Steele, Lea and
// Flood, "Fast splittable pseudorandom number generators", OOPSLA 2014)
__device__ __forceinline__ uint64_t draw(uint64_t seed, uint64_t at) {
  uint64_t z = seed + (at + 1) * 0x9E3779B97F4A7C15ull;
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

template <class T, bool kTail>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs g) {
  constexpr int N = Vec<T>::kN;
  const taccl_dropout_t &a = g.a;
  const int lane = threadIdx.x & (g.lanes - 1), per = kThreads / g.lanes;
  const int64_t row = g.first + (int64_t)(blockIdx.x / g.per_row) * per + threadIdx.x / g.lanes;
  const int c = (int)(blockIdx.x % g.per_row * kThreads + lane) * N;
  if (row >= a.rows || c >= a.cols) return;
  const int left = a.cols - c;
  const auto x = load_vec<T, kTail>((const T *)a.x + row * a.x_stride + c, left);
  typename Vec<T>::V r, y;
  if (a.residual)
    r = load_vec<T, kTail>((const T *)a.residual + row * a.residual_stride + c, left);
  const uint64_t seed = (uint64_t)a.rng[0];
  const uint64_t at =
      (uint64_t)a.rng[1] + (uint64_t)row * ((uint32_t)(a.cols + 1) / 2) + c / 2;
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const uint64_t w = draw(seed, at + i / 2);
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const uint32_t field = (uint32_t)(w >> 32 * j);
      const float v = field >= g.below && !g.all ? (float)x[i + j] * g.scale : 0.0f;
      y[i + j] = (T)(a.residual ? v + (float)r[i + j] : v);
    }
  }
  store_vec<T, kTail>((T *)a.out + row * a.out_stride + c, y, left);
}

template <class T>
const void *dropout_fn(bool tail) {
  return tail ? (const void *)dropout_kernel<T, true> : (const void *)dropout_kernel<T, false>;
}

}  // namespace

hipError_t launch_dropout(const taccl_dropout_t &a, hipStream_t stream) {
  DropoutArgs g{a, 0, a.p >= 1, (float)(1 / (1 - a.p)), 1, 1, 0};
  const double below = std::ceil(a.p * 4294967296.0);
  g.all = below > 4294967295.0;
  g.below = g.all ? 0 : (uint32_t)below;
  const int n = a.dtype == TACCL_F32 ? 4 : 8, units = (a.cols + n - 1) / n;
  while (g.lanes < kThreads && g.lanes < units) g.lanes *= 2;
  g.per_row = (units + g.lanes - 1) / g.lanes;
  const int64_t per = kThreads / g.lanes;
  const bool tail = a.cols % n != 0;
  const void *fn = a.dtype == TACCL_F32    ? dropout_fn<float>(tail)
                   : a.dtype == TACCL_BF16 ? dropout_fn<bf16_t>(tail)
                                           : dropout_fn<f16_t>(tail);
  void *args[] = {&g};
  const int64_t most = kMaxBlocks / g.per_row * per;  // rows of a launch: 34 GB
  hipError_t e = hipSuccess;
  for (; g.first < a.rows && e == hipSuccess; g.first += most) {
    const int64_t n = std::min(most, a.rows - g.first);
    e = hipLaunchKernel(fn, dim3((uint32_t)((n + per - 1) / per * g.per_row)), dim3(kThreads), args,
                        0, stream);
  }
  return e;
}

}  // namespace taccl
