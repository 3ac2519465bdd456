// The expert layer of a few tokens: choice of the experts, their gated products
// and the weighted sum, in two launches.
//
//   out[t] = sum_j w[t][j] Wo_e (silu(Wg_e x[t]) * (Wu_e x[t])),  e = experts[t][j]
//
// The weights of the chosen experts are what has to be read, and they are read
// once: an expert's product takes 16 rows of its weights as one operand of a
// matrix instruction and all tokens as the other, straight from memory, with
// the shared axis split over the wavefronts of a block. Tokens that did not
// choose the expert come out as zeros.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "elem.h"
#include "expert.h"
#include "ffn.h"
#include "tile.h"

namespace taccl {

namespace {

constexpr int kTokens = kFfnTokens;
constexpr int kUpWaves = 8, kDownWaves = 16;

// The workspace: the chosen experts, then w a of every (expert, token) in
// chunks along the hidden axis: 4 floats, or 8 values as the sum of two 16-bit
// numbers (the weights are 16-bit then; a rounded to 16 bits would be off by as
// much as the result's own rounding, and the second product costs nothing that
// the weights' reading does not hide).
struct Chosen {
  int32_t n;
  int32_t experts[kMaxExperts];
};
constexpr int64_t kChosenBytes = (sizeof(Chosen) + 255) / 256 * 256;

int64_t hidden_wide(int64_t hidden) { return (hidden + 15) / 16 * 16; }

struct TokensArgs {
  taccl_ffn_tokens_t a;
  Chosen *chosen;
  uint8_t *act;
  int32_t wide;  // hidden, rounded up to 16
};

struct Choices {
  int16_t expert[kTokens][kMaxChoices];  // -1: none
  float weight[kTokens][kMaxChoices];
  uint32_t used[kMaxExperts / 32];  // of the local experts
  int16_t list[kMaxExperts];
  int32_t n;
};

__device__ __forceinline__ float load_logit(const void *p, int64_t i, int dtype) {
  return dtype == TACCL_F32    ? ((const float *)p)[i]
         : dtype == TACCL_BF16 ? (float)((const bf16_t *)p)[i]
                               : (float)((const f16_t *)p)[i];
}

// The choices of the router (route.hip) for token t by a row of 16 lanes: the
// largest logit k times, equal ones in the order of their index; minus infinity
// and NaN never, a NaN in the sum of the exponentials.
template <int kEpl>
__device__ __forceinline__ void choose(const taccl_ffn_tokens_t &a, int t, Choices &c) {
  const int lane = threadIdx.x & 15, E = a.num_experts;
  const bool take = t < a.tokens && (!a.mask || a.mask[t]);
  float v[kEpl];
#pragma unroll
  for (int i = 0; i < kEpl; i++) {
    const int e = i * 16 + lane;
    v[i] = take && e < E ? load_logit(a.logits, t * a.logits_stride + e, a.logits_dtype)
                         : -__builtin_inff();
  }
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < kEpl; i++) top = fmaxf(top, v[i]);
  top = lanes_max<16>(top);
  const float base = top == -__builtin_inff() ? 0.0f : top;
  float sum = 0;
#pragma unroll
  for (int i = 0; i < kEpl; i++)
    sum += __builtin_amdgcn_exp2f((v[i] - base) * 1.4426950408889634f);
  sum = lanes_sum<16>(sum);
  int own = -1;
  float p = 0;
  for (int j = 0; j < a.k; j++) {
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kEpl; i++) m = fmaxf(m, v[i]);
    m = lanes_max<16>(m);
    uint32_t at = 0xFFFFFFFFu;
#pragma unroll
    for (int i = kEpl - 1; i >= 0; i--) at = v[i] == m ? (uint32_t)(i * 16 + lane) : at;
    at = lanes_min<16>(at);
    if (m == -__builtin_inff()) at = 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < kEpl; i++) v[i] = at == (uint32_t)(i * 16 + lane) ? -__builtin_inff() : v[i];
    if (lane == j && at != 0xFFFFFFFFu) {
      own = (int)at;
      p = __builtin_amdgcn_exp2f((m - base) * 1.4426950408889634f);
    }
  }
  if (a.renorm) sum = lanes_sum<16>(p);
  if (t < a.tokens && lane < a.k) {
    c.expert[t][lane] = (int16_t)own;
    c.weight[t][lane] = own >= 0 ? p / sum : 0.0f;
    const int local = own - a.first_expert;
    if (own >= 0 && (uint32_t)local < (uint32_t)a.local_experts)
      atomicOr(&c.used[local >> 5], 1u << (local & 31));
  }
}

// All tokens' choices and the list of chosen local experts, in their order
__device__ __forceinline__ void choose_all(const taccl_ffn_tokens_t &a, Choices &c) {
  for (int i = threadIdx.x; i < kMaxExperts / 32; i += blockDim.x) c.used[i] = 0;
  __syncthreads();
  for (int t0 = 0; t0 < a.tokens; t0 += blockDim.x / 16) {
    const int t = t0 + threadIdx.x / 16;
    if (t0 + (int)(threadIdx.x / 64) * 4 >= a.tokens) break;  // by wavefronts
    if (a.num_experts <= 64) choose<4>(a, t, c);
    else if (a.num_experts <= 256) choose<16>(a, t, c);
    else choose<64>(a, t, c);
  }
  __syncthreads();
  if (threadIdx.x < 64) {  // a word's experts per lane of the first half
    uint32_t w = threadIdx.x < kMaxExperts / 32 ? c.used[threadIdx.x] : 0;
    const uint32_t upto = wave_scan_add(__popc(w));
    uint32_t at = upto - __popc(w);
    for (; w; w &= w - 1) c.list[at++] = (int16_t)(threadIdx.x * 32 + __builtin_ctz(w));
    if (threadIdx.x == 63) c.n = (int32_t)upto;
  }
  __syncthreads();
}

// Address of the chunk at hidden column f (a multiple of the chunk's) of a
// token: float chunks, or pairs of 16-bit ones
template <class T>
__device__ __forceinline__ uint8_t *act_at(const TokensArgs &g, int slot, int t, int f) {
  return g.act + ((int64_t)(slot * g.a.tokens + t) * g.wide + f) * 4;
}

// a of 16 hidden columns of an expert per turn: gate and up rows of its
// weights, by eight wavefronts that take steps of 128 bytes in turn.
template <class T, int NT, bool kTail>
__global__ __launch_bounds__(64 * kUpWaves) void tokens_up_kernel(TokensArgs g) {
  constexpr int N = Vec<T>::kN, U = NT == 1 ? 4 : 2;
  __shared__ Choices c;
  __shared__ F4 red[kUpWaves][2][NT][64];
  const taccl_ffn_tokens_t &a = g.a;
  const int D = a.cols, F = a.hidden, tiles = g.wide / 16;
  choose_all(a, c);
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < a.tokens * a.k; i += blockDim.x) {
      if (a.experts) a.experts[i] = c.expert[i / a.k][i % a.k];
      if (a.weights) a.weights[i] = c.weight[i / a.k][i % a.k];
    }
    for (int i = threadIdx.x; i < c.n; i += blockDim.x) g.chosen->experts[i] = c.list[i];
    if (threadIdx.x == 0) g.chosen->n = c.n;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int steps = (D + 8 * N - 1) / (8 * N);
  for (int item = blockIdx.x; item < c.n * tiles; item += gridDim.x) {
    const int slot = item / tiles, f0 = item % tiles * 16, e = c.list[slot];
    const T *gate = (const T *)a.w_in + ((int64_t)e * 2 * F + min(f0 + r, F - 1)) * D;
    const T *up = gate + (int64_t)F * D;
    const T *x[NT];
#pragma unroll
    for (int i = 0; i < NT; i++)
      x[i] = (const T *)a.x + min(16 * i + r, (int)a.tokens - 1) * a.x_stride;
    F4 ag[NT], au[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) ag[i] = au[i] = F4{0, 0, 0, 0};
    for (int s0 = wave; s0 < steps; s0 += U * kUpWaves) {
      Frag<T> fg[U][2], fu[U][2], fx[U][2][NT];
#pragma unroll
      for (int s = 0; s < U; s++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const int k = ((s0 + s * kUpWaves) * 8 + h * 4 + q) * N, left = D - k;
          fg[s][h].v = load_vec<T, kTail>(gate + k, left);
          fu[s][h].v = load_vec<T, kTail>(up + k, left);
#pragma unroll
          for (int i = 0; i < NT; i++) fx[s][h][i].v = load_vec<T, kTail>(x[i] + k, left);
        }
#pragma unroll
      for (int s = 0; s < U; s++)
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
          for (int i = 0; i < NT; i++) {
            ag[i] = multiply(fg[s][h], fx[s][h][i], ag[i]);
            au[i] = multiply(fu[s][h], fx[s][h][i], au[i]);
          }
    }
#pragma unroll
    for (int i = 0; i < NT; i++) {
      red[wave][0][i][lane] = ag[i];
      red[wave][1][i][lane] = au[i];
    }
    __syncthreads();
    // four hidden columns of a token per thread
    const int t = 16 * wave + r, f = f0 + 4 * q;
    if (wave < NT && t < a.tokens) {
      F4 sg = red[0][0][wave][lane], su = red[0][1][wave][lane];
#pragma unroll
      for (int w = 1; w < kUpWaves; w++) {
        sg += red[w][0][wave][lane];
        su += red[w][1][wave][lane];
      }
      float weight = 0;
      bool member = false;
      for (int j = 0; j < a.k; j++)
        if (c.expert[t][j] == e + a.first_expert) {
          member = true;
          weight = c.weight[t][j];
        }
      F4 y;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float s = sizeof(T) == 4
                            ? 1.0f / (1.0f + expf(-sg[i]))
                            : __builtin_amdgcn_rcpf(
                                  1.0f + __builtin_amdgcn_exp2f(sg[i] * -1.4426950408889634f));
        y[i] = member && f + i < F ? sg[i] * s * su[i] * weight : 0.0f;
      }
      if constexpr (sizeof(T) == 4) {
        *(F4 *)act_at<T>(g, slot, t, f) = y;
      } else {
        typedef T T4 __attribute__((ext_vector_type(4)));
        T4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; i++) {
          hi[i] = (T)y[i];
          const float rest = y[i] - (float)hi[i];
          lo[i] = (T)(rest - rest == 0 ? rest : 0.0f);  // not of an infinite number
        }
        uint8_t *p = act_at<T>(g, slot, t, f & ~7) + (f & 4) * 2;
        *(T4 *)p = hi;
        *(T4 *)(p + 16) = lo;
      }
    }
    __syncthreads();
  }
}

// 16 columns of the output: the chosen experts' rows of w_out one after the
// other as one long shared axis.
template <class T, int NT, bool kTail>
__global__ __launch_bounds__(64 * kDownWaves) void tokens_down_kernel(TokensArgs g) {
  constexpr int N = Vec<T>::kN, U = NT == 1 ? 2 : 1, kPlanes = sizeof(T) == 4 ? 1 : 2;
  __shared__ F4 red[kDownWaves][NT][64];
  const taccl_ffn_tokens_t &a = g.a;
  const int D = a.cols, F = a.hidden;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int d0 = blockIdx.x * 16, steps = (F + 8 * N - 1) / (8 * N), n = g.chosen->n;
  F4 acc[NT];
#pragma unroll
  for (int i = 0; i < NT; i++) acc[i] = F4{0, 0, 0, 0};
  for (int s0 = wave; s0 < n * steps; s0 += U * kDownWaves) {
    Frag<T> fw[U][2], fa[U][2][NT][kPlanes];
#pragma unroll
    for (int s = 0; s < U; s++) {
      const int step = s0 + s * kDownWaves, slot = min(step / steps, n - 1);
      const int e = g.chosen->experts[slot];
      const T *w = (const T *)a.w_out + ((int64_t)e * D + min(d0 + r, D - 1)) * F;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int k = (step % steps * 8 + h * 4 + q) * N;
        const int left = step < n * steps ? F - k : 0;
        fw[s][h].v = load_vec<T, kTail>(w + k, left);
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
          for (int p = 0; p < kPlanes; p++) {
            const uint8_t *at = act_at<T>(g, slot, min(16 * i + r, (int)a.tokens - 1), k) + 16 * p;
            fa[s][h][i][p].v = load_vec<T, false>((const T *)at, left > 0 ? N : 0);
          }
      }
    }
#pragma unroll
    for (int s = 0; s < U; s++)
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
          for (int p = 0; p < kPlanes; p++) acc[i] = multiply(fw[s][h], fa[s][h][i][p], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < NT; i++) red[wave][i][lane] = acc[i];
  __syncthreads();
  const int t = 16 * wave + r, d = d0 + 4 * q;
  if (wave < NT && t < a.tokens) {
    F4 y = red[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kDownWaves; w++) y += red[w][wave][lane];
    T *out = (T *)a.out + t * a.out_stride + d;
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (d + i < D) out[i] = (T)y[i];
  }
}

template <class T, bool kTail>
const void *tokens_fn(int tokens, bool up) {
#define F(NT)                                            \
  (up ? (const void *)tokens_up_kernel<T, NT, kTail>     \
      : (const void *)tokens_down_kernel<T, NT, kTail>)
  return tokens <= 16 ? F(1) : tokens <= 32 ? F(2) : F(4);
#undef F
}
const void *tokens_fn(int dtype, int tokens, bool tail, bool up) {
#define F(T) (tail ? tokens_fn<T, true>(tokens, up) : tokens_fn<T, false>(tokens, up))
  return dtype == TACCL_F32 ? F(float) : dtype == TACCL_BF16 ? F(bf16_t) : F(f16_t);
#undef F
}

}  // namespace

int64_t ffn_tokens_space(int64_t tokens, int64_t experts, int64_t k, int64_t hidden) {
  return kChosenBytes + std::min(experts, tokens * k) * tokens * hidden_wide(hidden) * 4;
}

hipError_t launch_ffn_tokens(const taccl_ffn_tokens_t &a, int cus, hipStream_t stream) {
  TokensArgs g{a, (Chosen *)a.workspace, (uint8_t *)a.workspace + kChosenBytes,
               (int32_t)hidden_wide(a.hidden)};
  const int n = a.dtype == TACCL_F32 ? 4 : 8;
  void *args[] = {&g};
  const int64_t items =
      std::min<int64_t>(a.local_experts, a.tokens * a.k) * (g.wide / 16);
  hipError_t e = hipLaunchKernel(tokens_fn(a.dtype, (int)a.tokens, a.cols % n != 0, true),
                                 dim3((uint32_t)std::min<int64_t>(items, 2 * cus)),
                                 dim3(64 * kUpWaves), args, 0, stream);
  if (e != hipSuccess) return e;
  return hipLaunchKernel(tokens_fn(a.dtype, (int)a.tokens, a.hidden % n != 0, false),
                         dim3((uint32_t)(a.cols + 15) / 16), dim3(64 * kDownWaves), args, 0,
                         stream);
}

}  // namespace taccl
