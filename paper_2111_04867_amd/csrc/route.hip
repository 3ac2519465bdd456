// Router: choice of k experts per token, the places of the choices, the
// experts' loads and the balance loss; and its gradient.
//
//   p = softmax(l); loss = coef E sum_e (counts_e / (n k)) (P_e / n)
//   dl = p (g - sum_e p_e g_e),  g_e = dloss coef E counts_e / (n^2 k)
//   chosen weights w_j = p_{e_j}: g_{e_j} += dw_j;
//   renormalised (w = softmax over the chosen logits):
//   dl_{e_j} += w_j (dw_j - sum_i w_i dw_i)
//
// A group of kL lanes holds one token's logits, kEpl consecutive experts per
// lane. The sums over tokens go through per-block partial results and a
// second launch, never through floating atomics, so their order is fixed.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "elem.h"
#include "expert.h"

namespace taccl {

namespace {

constexpr int kRouteThreads = 1024;
constexpr int kBackThreads = 256;

// per-block results: the experts' counts with the rows' count behind them,
// and the experts' probability sums
struct RoutePartial {
  uint32_t *counts;  // [blocks][E + 1]
  float *sums;       // [blocks][E]
  int per_block;     // tokens per block
  int blocks;
};

// One token's logits in a group of lanes: softmax statistics.
template <int kL, int kEpl>
struct TokenRow {
  float v[kEpl];  // minus infinity past the experts and in rows not taken

  template <class T>
  __device__ __forceinline__ void load(const T *row, int lane, int E, bool take) {
    constexpr int N = Vec<T>::kN < kEpl ? Vec<T>::kN : kEpl;
    const int first = lane * kEpl;
#pragma unroll
    for (int i = 0; i < kEpl; i++) v[i] = -__builtin_inff();
    if (!take) return;
    if (first + kEpl <= E) {
      typedef T W __attribute__((ext_vector_type(N)));
      typedef W U __attribute__((aligned(sizeof(T))));
#pragma unroll
      for (int i = 0; i < kEpl; i += N) {
        const W w = *(const U *)(row + first + i);
#pragma unroll
        for (int x = 0; x < N; x++) v[i + x] = (float)w[x];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEpl; i++)
        if (first + i < E) v[i] = (float)row[first + i];
    }
  }

  // the exponent's offset (0 in a row of minus infinities and NaNs), the
  // exponentials and 1 / their sum, 0 in a row without a number
  float base, inv;
  float p[kEpl];  // exp(v - base)
  __device__ __forceinline__ void softmax() {
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kEpl; i++) m = fmaxf(m, v[i]);
    m = lanes_max<kL>(m);
    base = m == -__builtin_inff() ? 0.0f : m;
    float s = 0;
#pragma unroll
    for (int i = 0; i < kEpl; i++) {
      p[i] = __expf(v[i] - base);
      s += p[i];
    }
    s = lanes_sum<kL>(s);
    inv = s == 0.0f ? 0.0f : 1.0f / s;
  }
};

// The balance loss and the totals from the experts' counts and sums in LDS
__device__ __forceinline__ void finish_loss(const taccl_route_t &a, const uint32_t *cnt,
                                            const float *sums, float *red) {
  const int E = a.num_experts;
  float s = 0;
  for (int e = threadIdx.x; e < E; e += blockDim.x) {
    a.counts[e] = (int32_t)cnt[e];
    a.prob_sums[e] = sums[e];
    s += (float)cnt[e] * sums[e];
  }
  s = lanes_sum<64>(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < (int)blockDim.x / 64; i++) s += red[i];
    const float n = (float)max(cnt[E], 1u);
    *a.loss = a.coef * (float)E * (s / (n * (float)a.k) / n);
    *a.rows = (int32_t)cnt[E];
  }
}

// First launch: per block of tokens. A tile is one token per group of lanes;
// the tile's choices of an expert are bits of one word per expert in LDS, so
// a choice's place is the count of the tiles before plus the bits below its
// own. A single block writes the final results.
template <class T, int kL, int kEpl>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(taccl_route_t a, RoutePartial part) {
  constexpr int kGroups = kRouteThreads / kL, kWaves = kRouteThreads / 64;
  constexpr int kCols = kL * kEpl;
  __shared__ uint64_t bits[kCols + 1];
  __shared__ uint32_t cnt[kCols + 1];
  __shared__ float sums[kWaves][kCols];
  __shared__ float red[kWaves];
  const int E = a.num_experts, k = a.k;
  const int lane = threadIdx.x % kL, group = threadIdx.x / kL;
  for (int e = threadIdx.x; e <= E; e += kRouteThreads) {
    bits[e] = 0;
    cnt[e] = 0;
  }
  float acc[kEpl];
#pragma unroll
  for (int i = 0; i < kEpl; i++) acc[i] = 0;
  const int64_t begin = (int64_t)blockIdx.x * part.per_block;
  const int64_t end = min(begin + part.per_block, a.tokens);
  __syncthreads();
  for (int64_t first = begin; first < end; first += kGroups) {
    const int64_t t = first + group;
    const bool inside = t < end;
    const bool take = inside && (!a.mask || a.mask[t]);
    TokenRow<kL, kEpl> x;
    x.load((const T *)a.logits + t * a.logits_stride, lane, E, take);
    x.softmax();
#pragma unroll
    for (int i = 0; i < kEpl; i++) acc[i] += x.p[i] * x.inv;
    // the k largest, one at a time; lane j keeps choice j
    int expert = -1;
    float weight = 0;
    for (int j = 0; j < k; j++) {
      float m = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < kEpl; i++) m = fmaxf(m, x.v[i]);
      m = lanes_max<kL>(m);
      uint32_t at = 0xFFFFFFFFu;
#pragma unroll
      for (int i = kEpl - 1; i >= 0; i--) at = x.v[i] == m ? (uint32_t)(lane * kEpl + i) : at;
      at = lanes_min<kL>(at);
      if (m == -__builtin_inff()) at = 0xFFFFFFFFu;
#pragma unroll
      for (int i = 0; i < kEpl; i++)
        x.v[i] = at == (uint32_t)(lane * kEpl + i) ? -__builtin_inff() : x.v[i];
      if (lane == j && at != 0xFFFFFFFFu) {
        expert = (int)at;
        weight = __expf(m - x.base);
      }
    }
    if (a.renorm) {
      const float s = lanes_sum<kL>(weight);
      weight = s == 0.0f ? 0.0f : weight / s;
    } else {
      weight *= x.inv;
    }
    if (lane < k && expert >= 0) atomicOr((unsigned long long *)&bits[expert], 1ull << group);
    if (lane == 0 && x.inv != 0.0f) atomicOr((unsigned long long *)&bits[E], 1ull << group);
    __syncthreads();
    if (inside && lane < k) {
      const int64_t o = t * k + lane;
      int slot = -1;
      if (expert >= 0) {
        const uint32_t place =
            cnt[expert] + (uint32_t)__popcll(bits[expert] & ((1ull << group) - 1));
        slot = part.blocks > 1 || !a.capacity || place < a.capacity ? (int)place : -1;
      }
      a.experts[o] = expert;
      a.weights[o] = weight;
      a.slots[o] = slot;
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kRouteThreads) {
      cnt[e] += (uint32_t)__popcll(bits[e]);
      bits[e] = 0;
    }
    __syncthreads();
  }
  // the block's probability sums: groups of a wavefront, then wavefronts
  if (kL == 16) {
#pragma unroll
    for (int i = 0; i < kEpl; i++) {
      acc[i] += __shfl_xor(acc[i], 16);
      acc[i] += __shfl_xor(acc[i], 32);
    }
  }
  if ((threadIdx.x & 63) < kL) {
#pragma unroll
    for (int i = 0; i < kEpl; i++) sums[threadIdx.x >> 6][lane * kEpl + i] = acc[i];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kRouteThreads) {
    float s = sums[0][e];
    for (int w = 1; w < kWaves; w++) s += sums[w][e];
    if (part.blocks > 1) part.sums[(int64_t)blockIdx.x * E + e] = s;
    else sums[0][e] = s;
  }
  if (part.blocks > 1) {
    for (int e = threadIdx.x; e <= E; e += kRouteThreads)
      part.counts[(int64_t)blockIdx.x * (E + 1) + e] = cnt[e];
    return;
  }
  __syncthreads();
  finish_loss(a, cnt, sums[0], red);
}

// Second launch: block b adds the counts of the blocks before b to the
// places of b's choices; the block behind them finishes the totals.
__global__ __launch_bounds__(kRouteThreads) void route_places_kernel(taccl_route_t a,
                                                                     RoutePartial part) {
  __shared__ uint32_t cnt[kMaxExperts + 1];
  __shared__ float sums[kMaxExperts];
  __shared__ float fsum[kRouteThreads];
  __shared__ float red[kRouteThreads / 64];
  const int E = a.num_experts, b = blockIdx.x;
  for (int e = threadIdx.x; e <= E; e += kRouteThreads) cnt[e] = 0;
  __syncthreads();
  // `slices` threads per expert
  int wide = 64;
  while (wide < E + 1 && wide < kRouteThreads) wide *= 2;
  const int slices = kRouteThreads / wide, slice = threadIdx.x / wide;
  for (int e = threadIdx.x % wide; e <= E; e += wide) {
    uint32_t n = 0;
    for (int i = slice; i < b; i += slices) n += part.counts[(int64_t)i * (E + 1) + e];
    if (n) atomicAdd(&cnt[e], n);
  }
  if (b < part.blocks) {
    __syncthreads();
    const int64_t begin = (int64_t)b * part.per_block;
    const int64_t end = min(begin + part.per_block, a.tokens);
    for (int64_t i = begin * a.k + threadIdx.x; i < end * a.k; i += kRouteThreads) {
      const int e = a.experts[i];
      if (e < 0) continue;
      const uint32_t place = (uint32_t)a.slots[i] + cnt[e];
      a.slots[i] = !a.capacity || place < a.capacity ? (int32_t)place : -1;
    }
    return;
  }
  for (int e0 = 0; e0 < E; e0 += wide) {
    const int e = e0 + threadIdx.x % wide;
    float s = 0;
    if (e < E)
      for (int i = slice; i < part.blocks; i += slices) s += part.sums[(int64_t)i * E + e];
    fsum[threadIdx.x] = s;
    __syncthreads();
    if (slice == 0 && e < E) {
      for (int i = 1; i < slices; i++) s += fsum[threadIdx.x + i * wide];
      sums[e] = s;
    }
    __syncthreads();
  }
  finish_loss(a, cnt, sums, red);
}

// Gradient: one token per group of lanes at a time. The chosen experts'
// terms go through a row of LDS per group (one wavefront reads and writes it,
// in order), zero outside them.
template <class T, int kL, int kEpl>
__global__ __launch_bounds__(kBackThreads) void route_backward_kernel(taccl_route_backward_t a) {
  constexpr int kGroups = kBackThreads / kL, kCols = kL * kEpl;
  __shared__ float chosen[kGroups][kCols];
  const int E = a.num_experts, k = a.k;
  const int lane = threadIdx.x % kL, group = threadIdx.x / kL;
  float *own = chosen[group] + lane * kEpl;
  const float n = (float)max(*a.rows, 1);
  const float scale = a.dloss ? *a.dloss * a.coef * (float)E / (n * n * (float)k) : 0.0f;
  float load[kEpl];
#pragma unroll
  for (int i = 0; i < kEpl; i++) {
    own[i] = 0;
    load[i] = lane * kEpl + i < E ? scale * (float)a.counts[lane * kEpl + i] : 0.0f;
  }
  for (int64_t first = (int64_t)blockIdx.x * kGroups; first < a.tokens;
       first += (int64_t)gridDim.x * kGroups) {
    const int64_t t = first + group;
    const bool inside = t < a.tokens;
    const bool take = inside && (!a.mask || a.mask[t]);
    const T *row = (const T *)a.logits + t * a.logits_stride;
    TokenRow<kL, kEpl> x;
    x.load(row, lane, E, take);
    int expert = -1;
    float dw = 0, weight = 0;
    if (a.dweights) {  // the same for every lane
      if (take && lane < k) {
        expert = a.experts[t * k + lane];
        if ((uint32_t)expert < (uint32_t)E) {
          dw = a.dweights[t * k + lane];
          weight = (float)row[expert];
        } else {
          expert = -1;
        }
      }
    }
    x.softmax();
    if (a.dweights) {
      weight = expert >= 0 ? __expf(weight - x.base) : 0.0f;
      float term = dw;
      if (a.renorm) {
        const float s = lanes_sum<kL>(weight);
        weight = s == 0.0f ? 0.0f : weight / s;
        term = weight * (dw - lanes_sum<kL>(weight * dw));
      }
      if (expert >= 0) chosen[group][expert] = term;
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");
    }
    float c[kEpl], dot = 0;
#pragma unroll
    for (int i = 0; i < kEpl; i++) {
      c[i] = a.dweights ? own[i] : 0.0f;
      x.p[i] *= x.inv;
      dot += x.p[i] * (a.renorm ? load[i] : load[i] + c[i]);
    }
    dot = lanes_sum<kL>(dot);
    if (a.dweights) {
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");
      if (expert >= 0) chosen[group][expert] = 0;
    }
    if (!inside) continue;
    T *out = (T *)a.dlogits + t * a.dlogits_stride + lane * kEpl;
    T g[kEpl];
#pragma unroll
    for (int i = 0; i < kEpl; i++)
      g[i] = (T)(x.inv == 0.0f ? 0.0f
                 : a.renorm    ? x.p[i] * (load[i] - dot) + c[i]
                               : x.p[i] * (load[i] + c[i] - dot));
    constexpr int N = Vec<T>::kN < kEpl ? Vec<T>::kN : kEpl;
    typedef T W __attribute__((ext_vector_type(N)));
    typedef W U __attribute__((aligned(sizeof(T))));
    if (lane * kEpl + kEpl <= E) {
#pragma unroll
      for (int i = 0; i < kEpl; i += N) {
        W w;
#pragma unroll
        for (int y = 0; y < N; y++) w[y] = g[i + y];
        *(U *)(out + i) = w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEpl; i++)
        if (lane * kEpl + i < E) out[i] = g[i];
    }
  }
}

// lanes per token and experts per lane: 16 lanes up to 256 experts
template <class T, bool kBack>
const void *route_fn(int E, int &lanes) {
  lanes = E <= 256 ? 16 : 64;
#define PICK(L, EPL) \
  (kBack ? (const void *)route_backward_kernel<T, L, EPL> : (const void *)route_kernel<T, L, EPL>)
  if (E <= 16) return PICK(16, 1);
  if (E <= 32) return PICK(16, 2);
  if (E <= 64) return PICK(16, 4);
  if (E <= 128) return PICK(16, 8);
  if (E <= 256) return PICK(16, 16);
  if (E <= 512) return PICK(64, 8);
  return PICK(64, 16);
#undef PICK
}

template <bool kBack>
const void *route_pick(int dtype, int E, int &lanes) {
  if (dtype == TACCL_F32) return route_fn<float, kBack>(E, lanes);
  if (dtype == TACCL_BF16) return route_fn<bf16_t, kBack>(E, lanes);
  return route_fn<f16_t, kBack>(E, lanes);
}

}  // namespace

hipError_t launch_route(const taccl_route_t &a, hipStream_t stream) {
  int lanes;
  const void *fn = route_pick<false>(a.dtype, a.num_experts, lanes);
  const int64_t tile = kRouteThreads / lanes;
  RoutePartial part;
  const int64_t tiles = (a.tokens + tile - 1) / tile;
  part.per_block =
      (int)(tile * std::max<int64_t>(1, (tiles + kRouteMaxBlocks - 1) / kRouteMaxBlocks));
  part.blocks = (int)std::max<int64_t>(1, (a.tokens + part.per_block - 1) / part.per_block);
  part.counts = (uint32_t *)a.workspace;
  part.sums = (float *)(part.counts + (int64_t)kRouteMaxBlocks * (a.num_experts + 1));
  void *args[] = {(void *)&a, &part};
  hipError_t e = hipLaunchKernel(fn, dim3(part.blocks), dim3(kRouteThreads), args, 0, stream);
  if (e != hipSuccess || part.blocks == 1) return e;
  return hipLaunchKernel((const void *)route_places_kernel, dim3(part.blocks + 1),
                         dim3(kRouteThreads), args, 0, stream);
}

hipError_t launch_route_backward(const taccl_route_backward_t &a, int cus, hipStream_t stream) {
  int lanes;
  const void *fn = route_pick<true>(a.dtype, a.num_experts, lanes);
  const int groups = kBackThreads / lanes;
  const int grid =
      (int)std::min<int64_t>((a.tokens + groups - 1) / groups, (int64_t)std::max(cus, 1) * 8);
  void *args[] = {(void *)&a};
  return hipLaunchKernel(fn, dim3(grid), dim3(kBackThreads), args, 0, stream);
}

}  // namespace taccl
