// Router: choice of k experts per token, the places of the choices, the
// experts' loads and the balance loss; and its gradient.
//
//   p = softmax(l); loss = coef E sum_e (counts_e / (n k)) (P_e / n)
//   dl = p (g - sum_e p_e g_e),  g_e = dloss coef E counts_e / (n^2 k)
//   chosen weights w_j = p_{e_j}: g_{e_j} += dw_j;
//   renormalised (w = softmax over the chosen logits):
//   dl_{e_j} += w_j (dw_j - sum_i w_i dw_i)
//
// A group of kL lanes holds one token's logits, kEpl experts per lane. The sums
// over tokens go through per-block partial results and a second launch, never
// through floating atomics, so their order is fixed; a small batch takes one
// block and one launch.
//
// What bounds it (averages of a trace): 32768 tokens, 256 experts, 8 choices, f32
// (33.5 MB, 7 us of memory) take 16.0 us in the first launch, half of them vector
// instructions (980 per wavefront, that is for eight tokens), and 5.9 us in the
// second, which is mostly launch and round trips to memory; 64 experts and 4
// choices 8.3 and 5.3 us. Taking the k maxima one after the other took 1.5 times
// the threshold's time. The gradient (69 MB, 14 us of memory) takes 21.5 us: the
// chosen logits are read where the choices, read before them, say.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "elem.h"
#include "expert.h"

namespace taccl {

namespace {

constexpr int kRouteThreads = 1024;
constexpr int kBackThreads = 256;
// up to kSmallTile tokens a block of 256 threads, up to kOneBlock one of 1024
// (two launches: 11.6 instead of 9 us), up to kSmallBlocks blocks of 256 again,
// so that the tokens are spread over the CUs (6000 tokens, 64 experts: 11.0 us a
// call for both launches, about one more with 1024)
constexpr int kSmallTile = 16, kOneBlock = 128, kSmallBlocks = 8192;

// Per-block results: the experts' counts and probability sums in rows padded
// to whole 16-byte vectors, and the tokens that count.
struct RoutePartial {
  float *sums;       // [blocks][wide]
  uint32_t *rows;    // [blocks]
  uint16_t *counts;  // [blocks][wide]
  unsigned long long *loss;  // the finishing blocks' shares of the loss
  int wide;
  int per_block;  // tokens per block
  int blocks;
};

// One token's logits in a group of kL lanes. The experts are dealt out in
// vectors of kN, one to each lane in turn, so that a group reads one piece of
// memory at a time; element i of a lane is expert index(lane, i), which grows
// with i.
template <class T, int kL, int kEpl>
struct TokenRow {
  static constexpr int kN = Vec<T>::kN < kEpl ? Vec<T>::kN : kEpl;
  static constexpr int kSlots = kEpl / kN;
  typedef T W __attribute__((ext_vector_type(kN)));
  typedef W U __attribute__((aligned(sizeof(T))));
  static __device__ __forceinline__ int index(int lane, int i) {
    return lane * kN + i / kN * (kL * kN) + i % kN;
  }

  // the logits as they are stored: minus infinity past the experts and in rows
  // not taken
  struct Raw {
    W w[kSlots];
    __device__ __forceinline__ void load(const T *row, int lane, int E, bool take) {
      if (E == kL * kEpl && take) {
#pragma unroll
        for (int s = 0; s < kSlots; s++) w[s] = *(const U *)(row + index(lane, s * kN));
        return;
      }
#pragma unroll
      for (int s = 0; s < kSlots; s++)
#pragma unroll
        for (int x = 0; x < kN; x++) w[s][x] = (T)-__builtin_inff();
      if (!take) return;
      asm volatile("" : "+v"(lane));  // its comparisons are not made ahead for the other path
#pragma unroll
      for (int s = 0; s < kSlots; s++) {
        const int e = index(lane, s * kN);
        if (e + kN <= E) {
          w[s] = *(const U *)(row + e);
        } else {
#pragma unroll
          for (int x = 0; x < kN; x++)
            if (e + x < E) w[s][x] = row[e + x];
        }
      }
    }
  };

  float v[kEpl];
  __device__ __forceinline__ void take(const Raw &r) {
#pragma unroll
    for (int i = 0; i < kEpl; i++) v[i] = (float)r.w[i / kN][i % kN];
  }

  // Softmax: the lane's maximum and the exponent's offset (0 in a row of minus
  // infinities and NaNs); the exponentials and 1 / their sum, 0 in a row
  // without a number. The offset is taken off before the product with log2(e):
  // as fma(logit, log2e, -(offset log2e)) the rounding of the second product
  // would be a factor of the whole row that overflows from offsets of 1e9 on.
  float top, base, inv;
  float p[kEpl];  // exp(v - base)
  __device__ __forceinline__ float power(float logit) const {
    return __builtin_amdgcn_exp2f((logit - base) * 1.4426950408889634f);
  }
  __device__ __forceinline__ void maxima() {
    top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kEpl; i++) top = fmaxf(top, v[i]);
    const float m = lanes_max<kL>(top);
    base = m == -__builtin_inff() ? 0.0f : m;
  }
  __device__ __forceinline__ void exponentials() {
    float s = 0;
#pragma unroll
    for (int i = 0; i < kEpl; i++) {
      p[i] = power(v[i]);
      s += p[i];
    }
    s = lanes_sum<kL>(s);
    inv = s == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(s);  // within one unit in the last place
  }
};

// floats as integers in the same order (both zeros alike, no NaN); kNone is
// below minus infinity's
constexpr int kNone = -0x7FFFFFFF;
__device__ __forceinline__ int order_key(float v) {
  const int x = __builtin_bit_cast(int, v + 0.0f);
  return x ^ ((x >> 31) & 0x7FFFFFFF);
}

#define IN_ROW(F) \
  F(1) F(2) F(3) F(4) F(5) F(6) F(7) F(8) F(9) F(10) F(11) F(12) F(13) F(14) F(15)

// Rank (0 = largest) of a lane's candidate in its row of 16 lanes, equal
// logits in the order of their expert; `n` candidates in the row, in lanes 0 to
// n - 1 of it. A 16-bit logit and the expert make one key; 32-bit ones are
// equal so seldom that the experts are compared only then.
template <class T>
__device__ __forceinline__ int row_rank(bool there, float logit, int expert, uint32_t n) {
  int key;
  if constexpr (sizeof(T) == 2) {
    const int x = __builtin_bit_cast(int16_t, (T)(logit + 0.0f));
    key = (int)((uint32_t)(x ^ ((x >> 15) & 0x7FFF)) << 16 | (0xFFFFu - (uint32_t)expert));
  } else {
    key = order_key(logit);
  }
  if (!there) key = kNone;
  uint32_t rank = 0;
#define BEATEN(R) rank += dppi<0x120 + R>(key) > key ? 1u : 0u;
  IN_ROW(BEATEN)
#undef BEATEN
  if (sizeof(T) == 2) return (int)rank;
  uint32_t taken = there ? 1u << rank : 0u;
  taken |= (uint32_t)dppi<kRor8>((int)taken);
  taken |= (uint32_t)dppi<kRor4>((int)taken);
  taken |= (uint32_t)dppi<kRor2>((int)taken);
  taken |= (uint32_t)dppi<kRor1>((int)taken);
  if (!__any(taken != (1u << n) - 1)) return (int)rank;
#define EQUAL(R)                                        \
  {                                                     \
    const int k = dppi<0x120 + R>(key);                 \
    const int x = dppi<0x120 + R>(expert);              \
    rank += k == key && x < expert ? 1u : 0u;           \
  }
  IN_ROW(EQUAL)
#undef EQUAL
  return (int)rank;
}

// The row's keys in descending order (bitonic merges over mirrored halves)
__device__ __forceinline__ int row_sorted(int v, int lane) {
  auto step = [&](int o, int bit) {
    const int hi = max(v, o), lo = min(v, o);
    v = lane & bit ? lo : hi;
  };
  constexpr int kMirror4 = 0x1B;  // quad_perm [3, 2, 1, 0]
  step(dppi<kXor1>(v), 1);
  step(dppi<kMirror4>(v), 2);
  step(dppi<kXor1>(v), 1);
  step(dppi<kHalfMirror>(v), 4);
  step(dppi<kXor2>(v), 2);
  step(dppi<kXor1>(v), 1);
  step(dppi<kMirror>(v), 8);
  step(dppi<kMirror4>(dppi<kHalfMirror>(v)), 4);
  step(dppi<kXor2>(v), 2);
  step(dppi<kXor1>(v), 1);
  return v;
}

// A lane's choice: rank among the token's choices, expert (-1: none) and logit
struct Choice {
  int rank, expert;
  float logit;
};

// One at a time: the row's maximum k times. Changes x.v.
template <class T, int kL, int kEpl>
__device__ __forceinline__ Choice choose_each(TokenRow<T, kL, kEpl> &x, int k, int lane) {
  Choice c{lane, -1, 0.0f};
  asm volatile("" : "+v"(lane));  // nothing of this is worked out ahead, where it is seldom used
  for (int j = 0; j < k; j++) {
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kEpl; i++) m = fmaxf(m, x.v[i]);
    m = lanes_max<kL>(m);
    uint32_t at = 0xFFFFFFFFu;
#pragma unroll
    for (int i = kEpl - 1; i >= 0; i--) at = x.v[i] == m ? (uint32_t)x.index(lane, i) : at;
    at = lanes_min<kL>(at);
    if (m == -__builtin_inff()) at = 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < kEpl; i++)
      x.v[i] = at == (uint32_t)x.index(lane, i) ? -__builtin_inff() : x.v[i];
    if (lane == j && at != 0xFFFFFFFFu) {
      c.expert = (int)at;
      c.logit = m;
    }
  }
  return c;
}

// By a threshold: the k-th largest of the lanes' maxima bounds the k-th
// largest logit from below, so the choices are among the logits that reach it.
// Where at most 16 do (for k = 8 about 10 of 256 random ones, 0.7% of the rows
// have more), lanes 0 to 15 of the group take one each, and their ranks are
// the choice. list_ranked() finds the candidates and reads their logits from
// the group's row in LDS (a lane's element is no register index; read from
// memory, they would have to wait for the next tile's logits, which are on
// their way), to be used behind the exponentials by rank_listed(). False: some
// row of the wavefront has more.
template <class T, int kL, int kEpl>
__device__ __forceinline__ bool list_ranked(const TokenRow<T, kL, kEpl> &x, int k, int lane,
                                            float *stage, uint16_t *list, Choice &c,
                                            uint32_t &n) {
  typedef TokenRow<T, kL, kEpl> Row;
  // at least the lowest number: minus infinities are never chosen
  float bound = -__FLT_MAX__;
  if (kL == 16) {
    const int sorted = row_sorted(order_key(x.top), lane);  // by every lane of the row
    int b = lane == k - 1 ? sorted : kNone;
    b = max(b, dppi<kRor8>(b));
    b = max(b, dppi<kRor4>(b));
    b = max(b, dppi<kRor2>(b));
    b = max(b, dppi<kRor1>(b));
    bound = fmaxf(bound, __builtin_bit_cast(float, b ^ ((b >> 31) & 0x7FFFFFFF)));
  } else {
    float m = x.top, most = m;
    for (int j = 0; j < k; j++) {  // the lanes' maxima, one lane after the other
      most = lanes_max<kL>(m);
      const uint64_t same = __ballot(m == most) >> ((threadIdx.x & 63) - lane);
      if (same && lane == __ffsll((unsigned long long)same) - 1) m = -__builtin_inff();
    }
    bound = fmaxf(most, bound);
  }
  uint32_t hit = 0;
#pragma unroll
  for (int i = 0; i < kEpl; i++) hit |= x.v[i] >= bound ? 1u << i : 0u;
#pragma unroll
  for (int i = 0; i < kEpl; i++) stage[Row::index(lane, i)] = x.v[i];
  const uint32_t mine = __popc(hit);
  uint32_t upto = row_scan_add(mine), all;
  if (kL > 16) upto += dpp<kBcast15, 0xa>(upto);
  if (kL > 32) upto += dpp<kBcast31, 0xc>(upto);
  if (kL == 16) all = dpp<0x15F>(upto);  // the group's last lane
  else all = (uint32_t)__shfl((int)upto, (threadIdx.x & 63) - lane + kL - 1);
  if (__any(all > 16)) return false;
  uint32_t at = upto - mine;
  const uint32_t first = (uint32_t)lane * Row::kN;  // Row::index(lane, 0)
  do {  // a lane without a further one writes past the list
    const uint32_t i = (uint32_t)__builtin_ctz(hit | 1u << 31);
    list[hit ? at : 16] = (uint16_t)(first + i + i / Row::kN * (kL * Row::kN - Row::kN));
    hit &= hit - 1;
    at++;
  } while (__any(hit));
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");  // one wavefront's LDS accesses are in order
  n = all;
  c = Choice{lane, -1, 0.0f};
  if ((uint32_t)lane < all) {
    c.expert = list[lane];
    c.logit = stage[c.expert];
  }
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
  return true;
}
template <class T>
__device__ __forceinline__ void rank_listed(Choice &c, uint32_t n, int lane) {
  const int rank = row_rank<T>(c.expert >= 0, c.logit, c.expert, lane < 16 ? n : 0);
  if (c.expert >= 0) c.rank = rank;
}

// Sums of two registers across the wavefront's halves (rows: across its odd
// and even rows of 16 lanes), a's in the lower half (even rows) and b's in the
// upper one. The swap puts half of each register into the other, so one
// addition does both.
__device__ __forceinline__ float swapped_sum(float a, float b, bool rows) {
  const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
  const auto r = rows ? __builtin_amdgcn_permlane16_swap(x, y, false, false)
                      : __builtin_amdgcn_permlane32_swap(x, y, false, false);
  const uint32_t first = r[0], second = r[1];
  return __uint_as_float(first) + __uint_as_float(second);
}
// Sums over the four rows, one of four values to each: the totals of v[0],
// v[2], v[1], v[3] in rows 0 to 3
__device__ __forceinline__ float rows_sum(const float *v) {
  return swapped_sum(swapped_sum(v[0], v[1], false), swapped_sum(v[2], v[3], false), true);
}

// The balance loss and the totals from the experts' counts and sums in LDS
__device__ __forceinline__ void finish_loss(const taccl_route_t &a, const uint32_t *cnt,
                                            const float *sums, uint32_t rows, float *red) {
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
    const float n = (float)max(rows, 1u);
    *a.loss = a.coef * (float)E * (s / (n * (float)a.k) / n);
    *a.rows = (int32_t)rows;
  }
}

// First launch: per block of tokens. The block's wavefronts take tokens on
// their own, up to kStep of the block, and leave every choice as a bit of the
// expert's words in LDS (one bit per token). A choice's place in the block is
// then the count of the steps before plus the bits below its own. A single
// block writes the final results.
constexpr int kStep = 256, kWords = kStep / 64;

template <class T, int kL, int kEpl, bool kRanked>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(taccl_route_t a, RoutePartial part) {
  constexpr int kWaves = kRouteThreads / 64, kCols = kL * kEpl;
  __shared__ uint64_t bits[kCols + 1][kWords];
  __shared__ uint32_t cnt[kCols + 1];
  // a tile's logits, and behind the last tile the wavefronts' sums
  __shared__ __align__(16) float stage[kRanked ? kRouteThreads / kL : kWaves][kCols];
  float (*sums)[kCols] = stage;
  __shared__ float red[kWaves];
  __shared__ uint16_t list[kRanked ? kRouteThreads / kL : 1][16 + 1];
  // the step's choices and weights: written to memory when it is done, since a
  // store between the tiles would have the next tile's logits wait for it
  __shared__ int16_t picked[kStep * kMaxChoices];
  __shared__ float weighed[kStep * kMaxChoices];
  const int E = a.num_experts, k = a.k;
  const int lane = threadIdx.x % kL, group = threadIdx.x / kL, groups = blockDim.x / kL;
  for (int e = threadIdx.x; e <= E; e += blockDim.x) {
#pragma unroll
    for (int w = 0; w < kWords; w++) bits[e][w] = 0;
    cnt[e] = 0;
  }
  float acc[kEpl];
#pragma unroll
  for (int i = 0; i < kEpl; i++) acc[i] = 0;
  const int64_t begin = (int64_t)blockIdx.x * part.per_block;
  const int64_t end = min(begin + part.per_block, a.tokens);
  if (blockIdx.x == 0 && threadIdx.x == 0) *part.loss = 0;  // for the second launch
  // a tile's logits are on their way while the one before is worked on
  typedef TokenRow<T, kL, kEpl> Row;
  typename Row::Raw next;
  auto fetch = [&](int64_t t) {
    next.load((const T *)a.logits + t * a.logits_stride, lane, E,
              t < end && (!a.mask || a.mask[t]));
  };
  fetch(begin + group);
  __syncthreads();
  for (int64_t first = begin; first < end; first += kStep) {
    const int n = (int)min((int64_t)kStep, end - first);  // tokens of the step
    for (int tile = 0; tile < n; tile += groups) {
      const int at = tile + group;
      const int64_t t = first + at;
      const bool inside = at < n;
      Row x;
      x.take(next);
      // the wait for this tile's loads comes before the next tile's are issued
#pragma unroll
      for (int i = 0; i < kEpl; i++) asm volatile("" : "+v"(x.v[i]));
      fetch(t + groups);
      x.maxima();
      Choice c;
      uint32_t n_listed = 0;
      const bool listed =
          kRanked && list_ranked(x, k, lane, stage[group], list[group], c, n_listed);
      x.exponentials();
#pragma unroll
      for (int i = 0; i < kEpl; i++) acc[i] += x.p[i] * x.inv;
      if (listed) rank_listed<T>(c, n_listed, lane);
      else c = choose_each(x, k, lane);
      const int expert = c.rank < k ? c.expert : -1;
      float weight = expert >= 0 ? x.power(c.logit) : 0.0f;
      if (a.renorm) {
        // summed with the j-th choice's in lane j, however the choices were found:
        // that is up to the wavefront's other tokens, on which a row's bits do not
        // depend
        float w = weight;
        if (listed) {
          const int to = (int)(threadIdx.x & 63) - lane + c.rank;
          w = __int_as_float(__builtin_amdgcn_ds_permute(4 * to, __float_as_int(weight)));
        }
        const float s = lanes_sum<kL>(w);
        weight *= s == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(s);
      } else {
        weight = expert >= 0 ? weight * x.inv : 0.0f;  // inv may be NaN
      }
      const unsigned long long bit = 1ull << (at & 63);
      if (expert >= 0) atomicOr((unsigned long long *)&bits[expert][at >> 6], bit);
      if (lane == 0 && x.inv != 0.0f) atomicOr((unsigned long long *)&bits[E][at >> 6], bit);
      if (inside && c.rank < k) {
        picked[at * k + c.rank] = (int16_t)expert;
        weighed[at * k + c.rank] = weight;
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * k; i += blockDim.x) {
      const int e = picked[i], at = i / k;
      int slot = -1;
      if (e >= 0) {
        const int word = at >> 6;
        uint32_t place = cnt[e] + (uint32_t)__popcll(bits[e][word] & ((1ull << (at & 63)) - 1));
        for (int w = 0; w < word; w++) place += (uint32_t)__popcll(bits[e][w]);
        slot = part.blocks > 1 || !a.capacity || place < a.capacity ? (int)place : -1;
      }
      a.experts[first * k + i] = e;
      a.weights[first * k + i] = weighed[i];
      a.slots[first * k + i] = slot;
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += blockDim.x) {
#pragma unroll
      for (int w = 0; w < kWords; w++) {
        cnt[e] += (uint32_t)__popcll(bits[e][w]);
        bits[e][w] = 0;
      }
    }
    __syncthreads();
  }
  // the block's probability sums: rows of a wavefront, then wavefronts
  float *mine = sums[threadIdx.x >> 6];
  if (kL == 64) {
#pragma unroll
    for (int i = 0; i < kEpl; i++) mine[Row::index(lane, i)] = acc[i];
  } else if (kL == 32) {
    const int upper = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < kEpl; i += 2)
      mine[Row::index(lane, i) + upper] = swapped_sum(acc[i], acc[i + 1], false);
  } else {
    const int r = (threadIdx.x & 63) >> 4, turn = (r >> 1) | (r & 1) << 1;  // rows_sum's order
#pragma unroll
    for (int i = 0; i < kEpl; i += 4) {
      float v[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4 && i + j < kEpl; j++) v[j] = acc[i + j];
      const float s = rows_sum(v);
      if (i + turn < kEpl) mine[Row::index(lane, i) + turn] = s;
    }
  }
  __syncthreads();
  const int waves = blockDim.x >> 6;
  for (int e = threadIdx.x; e < kCols; e += blockDim.x) {
    float s = sums[0][e];
    for (int w = 1; w < waves; w++) s += sums[w][e];
    if (part.blocks == 1) {
      sums[0][e] = s;
    } else if (e < part.wide) {
      part.sums[(int64_t)blockIdx.x * part.wide + e] = s;
      part.counts[(int64_t)blockIdx.x * part.wide + e] = e < E ? (uint16_t)cnt[e] : 0;
    }
  }
  if (part.blocks > 1) {
    if (threadIdx.x == 0) part.rows[blockIdx.x] = cnt[E];
    return;
  }
  __syncthreads();
  finish_loss(a, cnt, sums[0], cnt[E], red);
}

// Column sums of n rows of `wide` values by all threads: a thread takes a
// vector of columns of every so many rows. add() reads them, kLoads rows at a
// time; finish() sums the threads' parts into `out` in LDS. `lds`:
// kRouteThreads vectors.
template <class V, int kN, class S, int kLoads>
struct ColumnSums {
  typedef V Vk __attribute__((ext_vector_type(kN)));
  typedef S Sk __attribute__((ext_vector_type(kN)));
  int wide, parts, slices;
  Sk s;

  // of the `w` columns at `from`, in rows `stride` values apart
  __device__ __forceinline__ void add(const V *from, int n, int w, int stride) {
    wide = w;
    parts = w / kN;  // vectors per row, at most 256
    slices = min(kRouteThreads / parts, 32);  // finish() reads them in turn
    const int slice = threadIdx.x / parts;
#pragma unroll
    for (int c = 0; c < kN; c++) s[c] = 0;
    if (slice >= slices) return;
    const Vk *p = (const Vk *)from + threadIdx.x % parts;
    for (int i = slice; i < n; i += kLoads * slices) {
      Vk x[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; j++)
        x[j] = p[(int64_t)min(i + j * slices, n - 1) * (stride / kN)];
#pragma unroll
      for (int j = 0; j < kLoads; j++)
        if (i + j * slices < n) s += __builtin_convertvector(x[j], Sk);
    }
  }
  __device__ __forceinline__ void finish(S *lds, S *out) {
    if ((int)threadIdx.x < parts * slices) ((Sk *)lds)[threadIdx.x] = s;
    __syncthreads();
    for (int e = threadIdx.x; e < wide; e += kRouteThreads) {
      S t = 0;
      for (int i = 0; i < slices; i++) t += lds[i * wide + e];
      out[e] = t;
    }
    __syncthreads();
  }
};

// Second launch: block b adds the counts of the blocks before b to the
// places of b's choices. The blocks behind them total kFinishCols experts
// each (one block for all 256 of them takes 3 us for what its CU has to read,
// 8 instead of 5.9 us in all). Their shares of the loss, in [0, E], meet in one
// 64-bit word: 48 bits of them as whole numbers of 2^-37, whose sum does not
// depend on the order, 8 bits that count shares that are NaN and 8 that count
// blocks, so that whoever adds the last one holds the loss. Each block loads
// what it needs at once: a round trip to memory is the larger part of its time.
constexpr int kFinishCols = 32;

__global__ __launch_bounds__(kRouteThreads) void route_places_kernel(taccl_route_t a,
                                                                     RoutePartial part) {
  __shared__ __align__(16) uint32_t lds[8 * kRouteThreads];
  __shared__ uint32_t cnt[kMaxExperts];
  const int b = blockIdx.x, wide = part.wide;
  ColumnSums<uint16_t, 8, uint32_t, 8> counts;
  if (b >= part.blocks) {
    __shared__ float sums[kFinishCols];
    const int first = (b - part.blocks) * kFinishCols, cols = min(kFinishCols, wide - first);
    ColumnSums<float, 4, float, 8> probs;
    uint32_t n = threadIdx.x < part.blocks ? part.rows[threadIdx.x] : 0;
    counts.add(part.counts + first, part.blocks, cols, wide);
    probs.add(part.sums + first, part.blocks, cols, wide);
    counts.finish(lds, cnt);
    probs.finish((float *)lds, sums);
    n = wave_scan_add(n);
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    n = 0;
    for (int w = 0; w < kRouteThreads / 64; w++) n += lds[w];
    const int c = threadIdx.x, e = first + c;
    float s = 0;
    if (c < cols && e < a.num_experts) {
      a.counts[e] = (int32_t)cnt[c];
      a.prob_sums[e] = sums[c];
      s = (float)cnt[c] * sums[c];
    }
    s = lanes_sum<64>(s);
    if (threadIdx.x) return;
    const float rows = (float)max(n, 1u);
    s = s / (rows * (float)a.k) / rows * (float)a.num_experts;
    const unsigned long long mine =
        s != s ? 1ull << 8 | 1 : (unsigned long long)((double)s * 0x1p37) << 16 | 1;
    const unsigned long long all = atomicAdd(part.loss, mine) + mine;
    if ((int)(all & 0xFF) != (int)gridDim.x - part.blocks) return;
    *a.loss = all & 0xFF00 ? __builtin_nanf("") : a.coef * (float)((double)(all >> 16) * 0x1p-37);
    *a.rows = (int32_t)n;
    return;
  }
  const int64_t begin = (int64_t)b * part.per_block * a.k;
  const int64_t end = min(begin + (int64_t)part.per_block * a.k, a.tokens * a.k);
  int64_t i = begin + threadIdx.x;
  int e = i < end ? a.experts[i] : -1;
  int local = i < end ? a.slots[i] : 0;
  counts.add(part.counts, b, wide, wide);
  counts.finish(lds, cnt);
  while (i < end) {
    if (e >= 0) {
      const uint32_t place = (uint32_t)local + cnt[e];
      a.slots[i] = !a.capacity || place < a.capacity ? (int32_t)place : -1;
    }
    i += kRouteThreads;
    if (i < end) {
      e = a.experts[i];
      local = a.slots[i];
    }
  }
}

// Gradient: one token per group of lanes at a time. The chosen experts'
// terms go through a row of LDS per group (one wavefront reads and writes it,
// in order), zero outside them.
template <class T, int kL, int kEpl>
__global__ __launch_bounds__(kBackThreads) void route_backward_kernel(taccl_route_backward_t a) {
  typedef TokenRow<T, kL, kEpl> Row;
  constexpr int kGroups = kBackThreads / kL, kCols = kL * kEpl, kN = Row::kN;
  __shared__ __align__(16) float chosen[kGroups][kCols];
  const int E = a.num_experts, k = a.k;
  const int lane = threadIdx.x % kL, group = threadIdx.x / kL;
  float *own = chosen[group];
  const float n = (float)max(*a.rows, 1);
  const float scale = a.dloss ? *a.dloss * a.coef * (float)E / (n * n * (float)k) : 0.0f;
  float load[kEpl];
#pragma unroll
  for (int i = 0; i < kEpl; i++) {
    const int e = Row::index(lane, i);
    own[e] = 0;
    load[i] = e < E ? scale * (float)a.counts[e] : 0.0f;
  }
  for (int64_t first = (int64_t)blockIdx.x * kGroups; first < a.tokens;
       first += (int64_t)gridDim.x * kGroups) {
    const int64_t t = first + group;
    const bool inside = t < a.tokens;
    const bool take = inside && (!a.mask || a.mask[t]);
    const T *row = (const T *)a.logits + t * a.logits_stride;
    int expert = -1;
    float dw = 0, weight = 0;
    if (a.dweights && take && lane < k) {
      expert = a.experts[t * k + lane];
      dw = a.dweights[t * k + lane];
    }
    typename Row::Raw raw;
    raw.load(row, lane, E, take);
    Row x;
    x.take(raw);
    if ((uint32_t)expert < (uint32_t)E) weight = (float)row[expert];
    else expert = -1;
    x.maxima();
    x.exponentials();
    if (a.dweights) {
      weight = expert >= 0 ? x.power(weight) : 0.0f;
      float term = dw;
      if (a.renorm) {
        const float s = lanes_sum<kL>(weight);
        weight *= s == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(s);
        term = weight * (dw - lanes_sum<kL>(weight * dw));
      }
      if (expert >= 0) own[expert] = term;
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");
    }
    float c[kEpl], dot = 0;
#pragma unroll
    for (int i = 0; i < kEpl; i++) {
      c[i] = a.dweights ? own[Row::index(lane, i)] : 0.0f;
      x.p[i] *= x.inv;
      dot += x.p[i] * (a.renorm ? load[i] : load[i] + c[i]);
    }
    dot = lanes_sum<kL>(dot);
    if (a.dweights) {
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");
      if (expert >= 0) own[expert] = 0;
    }
    if (!inside) continue;
    T *out = (T *)a.dlogits + t * a.dlogits_stride;
#pragma unroll
    for (int s = 0; s < Row::kSlots; s++) {
      typename Row::W w;
#pragma unroll
      for (int y = 0; y < kN; y++) {
        const int i = s * kN + y;
        w[y] = (T)(x.inv == 0.0f ? 0.0f
                   : a.renorm    ? x.p[i] * (load[i] - dot) + c[i]
                                 : x.p[i] * (load[i] + c[i] - dot));
      }
      const int e = Row::index(lane, s * kN);
      if (e + kN <= E) {
        *(typename Row::U *)(out + e) = w;
      } else {
#pragma unroll
        for (int y = 0; y < kN; y++)
          if (e + y < E) out[e + y] = w[y];
      }
    }
  }
}

// lanes per token and experts per lane: 16 lanes up to 256 experts, 16 experts
// from there on (32768 tokens, 300 experts: first launch 25 us, 37 in 64 lanes of 8)
#define BY_EXPERTS(E, F)                                                                   \
  ((E) <= 16 ? F(16, 1) : (E) <= 32 ? F(16, 2) : (E) <= 64 ? F(16, 4) : (E) <= 128 ? F(16, 8) \
   : (E) <= 256 ? F(16, 16) : (E) <= 512 ? F(32, 16) : F(64, 16))
int token_lanes(int E) { return E <= 256 ? 16 : E <= 512 ? 32 : 64; }

template <class T>
const void *route_fn(int E, int k) {
  const bool ranked = k <= 8 || E <= 16;
#define F(L, EPL)                                               \
  (ranked ? (const void *)route_kernel<T, L, EPL, true>         \
          : (const void *)route_kernel<T, L, EPL, false>)
  return BY_EXPERTS(E, F);
#undef F
}
template <class T>
const void *route_backward_fn(int E) {
#define F(L, EPL) (const void *)route_backward_kernel<T, L, EPL>
  return BY_EXPERTS(E, F);
#undef F
}

}  // namespace

hipError_t launch_route(const taccl_route_t &a, hipStream_t stream) {
  const int E = a.num_experts;
  const void *fn = a.dtype == TACCL_F32    ? route_fn<float>(E, a.k)
                   : a.dtype == TACCL_BF16 ? route_fn<bf16_t>(E, a.k)
                                           : route_fn<f16_t>(E, a.k);
  // small blocks spread few tokens over the CUs
  const int threads = a.tokens <= kSmallTile || (a.tokens > kOneBlock && a.tokens <= kSmallBlocks)
                          ? 256
                          : kRouteThreads;
  const int64_t tile = threads / token_lanes(E);
  const int64_t tiles = (a.tokens + tile - 1) / tile;
  RoutePartial part;
  part.wide = (E + 7) / 8 * 8;
  part.per_block =
      (int)(tile * std::max<int64_t>(1, (tiles + kRouteMaxBlocks - 1) / kRouteMaxBlocks));
  if (a.tokens <= kOneBlock) part.per_block = kOneBlock;
  part.blocks = (int)std::max<int64_t>(1, (a.tokens + part.per_block - 1) / part.per_block);
  part.sums = (float *)a.workspace;
  part.rows = (uint32_t *)(part.sums + (int64_t)kRouteMaxBlocks * part.wide);
  part.counts = (uint16_t *)(part.rows + kRouteMaxBlocks);
  part.loss = (unsigned long long *)(part.counts + (int64_t)kRouteMaxBlocks * part.wide);
  void *args[] = {(void *)&a, &part};
  hipError_t e = hipLaunchKernel(fn, dim3(part.blocks), dim3(threads), args, 0, stream);
  if (e != hipSuccess || part.blocks == 1) return e;
  const int finish = (part.wide + kFinishCols - 1) / kFinishCols;
  return hipLaunchKernel((const void *)route_places_kernel, dim3(part.blocks + finish),
                         dim3(kRouteThreads), args, 0, stream);
}

hipError_t launch_route_backward(const taccl_route_backward_t &a, int cus, hipStream_t stream) {
  const int E = a.num_experts;
  const void *fn = a.dtype == TACCL_F32    ? route_backward_fn<float>(E)
                   : a.dtype == TACCL_BF16 ? route_backward_fn<bf16_t>(E)
                                           : route_backward_fn<f16_t>(E);
  const int groups = kBackThreads / token_lanes(E);
  const int grid =
      (int)std::min<int64_t>((a.tokens + groups - 1) / groups, (int64_t)std::max(cus, 1) * 8);
  void *args[] = {(void *)&a};
  return hipLaunchKernel(fn, dim3(grid), dim3(kBackThreads), args, 0, stream);
}

}  // namespace taccl
