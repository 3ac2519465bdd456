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
constexpr int kWaves = 4, kThreads = 64 * kWaves;
// blocks that a CU holds
constexpr int kPerCu = 4;
template <class T>
constexpr int kDownPerCu = sizeof(T) == 4 ? 4 : 3;
constexpr int kMaxParts = 16;

// An entry is up to 16 tokens that chose the same expert: the columns of one
// matrix operand.
constexpr int kMaxEntries = kTokens * kMaxChoices;

// The workspace: the entries, then w a of every one of their tokens: a row of
// floats, or two of 16-bit numbers whose sum it is (the weights are 16-bit then;
// a rounded to 16 bits would be off by as much as the result's own rounding, and
// the second product costs nothing that the weights' reading does not hide).
struct Chosen {
  int32_t n;
  uint32_t tokens[kMaxEntries][2];  // bits
  int16_t experts[kMaxEntries];
  int16_t rows[kMaxEntries];  // the first token's row
  int32_t done[kSplitTiles];  // parts of a tile of columns that are there
};
constexpr int64_t kChosenBytes = (sizeof(Chosen) + 255) / 256 * 256;

int64_t hidden_wide(int64_t hidden) { return (hidden + 15) / 16 * 16; }

struct TokensArgs {
  taccl_ffn_tokens_t a;
  Chosen *chosen;
  uint8_t *act;
  F4 *partial;   // [parts][tiles][tokens][4]
  int32_t wide;  // hidden, rounded up to 16
  int32_t parts;
  int32_t most;  // entries, at most
};

struct Choices {
  int16_t expert[kTokens][kMaxChoices];  // -1: none
  float weight[kTokens][kMaxChoices];
  uint32_t tokens[kMaxExperts][2];  // of the local experts
  // the entries: expert, with the number of tokens before in 16s above its 10
  // bits, and row
  int16_t list[kMaxEntries], rows[kMaxEntries];
  int32_t n;
};

// The choices of the router (route.hip) for token t by kL lanes: the largest
// logit k times, equal ones in the order of their index; minus infinity and NaN
// never, a NaN in the sum of the exponentials.
template <class T, int kL, int kEpl>
__device__ __forceinline__ void choose(const taccl_ffn_tokens_t &a, int t, Choices &c) {
  const int lane = threadIdx.x & (kL - 1), E = a.num_experts;
  const bool take = t < a.tokens && (!a.mask || a.mask[t]);
  const T *row = (const T *)a.logits + t * a.logits_stride;
  float v[kEpl];
#pragma unroll
  for (int i = 0; i < kEpl; i++) {
    const int e = i * kL + lane;
    v[i] = take && e < E ? (float)row[e] : -__builtin_inff();
  }
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < kEpl; i++) top = fmaxf(top, v[i]);
  top = lanes_max<kL>(top);
  const float base = top == -__builtin_inff() ? 0.0f : top;
  float sum = 0;
#pragma unroll
  for (int i = 0; i < kEpl; i++)
    sum += __builtin_amdgcn_exp2f((v[i] - base) * 1.4426950408889634f);
  sum = lanes_sum<kL>(sum);
  int own = -1;
  float p = 0;
  for (int j = 0; j < a.k; j++) {
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kEpl; i++) m = fmaxf(m, v[i]);
    m = lanes_max<kL>(m);
    uint32_t at = 0xFFFFFFFFu;
#pragma unroll
    for (int i = kEpl - 1; i >= 0; i--) at = v[i] == m ? (uint32_t)(i * kL + lane) : at;
    at = lanes_min<kL>(at);
    if (m == -__builtin_inff()) at = 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < kEpl; i++)
      v[i] = at == (uint32_t)(i * kL + lane) ? -__builtin_inff() : v[i];
    if (lane == j && at != 0xFFFFFFFFu) {
      own = (int)at;
      p = __builtin_amdgcn_exp2f((m - base) * 1.4426950408889634f);
    }
  }
  if (a.renorm) sum = lanes_sum<kL>(p);
  if (t < a.tokens && lane < a.k) {
    c.expert[t][lane] = (int16_t)own;
    c.weight[t][lane] = own >= 0 ? p / sum : 0.0f;
    const int local = own - a.first_expert;
    if (own >= 0 && (uint32_t)local < (uint32_t)a.local_experts)
      atomicOr(&c.tokens[local][t >> 5], 1u << (t & 31));
  }
}
// a row of 16 lanes per token, past 256 experts a wavefront
template <class T>
__device__ __forceinline__ void choose_each(const taccl_ffn_tokens_t &a, Choices &c) {
  const int wave = threadIdx.x >> 6, row = threadIdx.x >> 4 & 3;
  const int per = a.num_experts <= 256 ? 4 : 1;  // tokens of a wavefront
  for (int t0 = wave * per; t0 < a.tokens; t0 += kWaves * per) {
    if (a.num_experts <= 64) choose<T, 16, 4>(a, t0 + row, c);
    else if (a.num_experts <= 256) choose<T, 16, 16>(a, t0 + row, c);
    else choose<T, 64, 16>(a, t0, c);
  }
}

// All tokens' choices and the entries, in the experts' order
__device__ __forceinline__ void choose_all(const taccl_ffn_tokens_t &a, Choices &c) {
  for (int i = threadIdx.x; i < a.local_experts; i += kThreads) c.tokens[i][0] = c.tokens[i][1] = 0;
  __syncthreads();
  if (a.logits_dtype == TACCL_F32) choose_each<float>(a, c);
  else if (a.logits_dtype == TACCL_BF16) choose_each<bf16_t>(a, c);
  else choose_each<f16_t>(a, c);
  __syncthreads();
  if (threadIdx.x < 64) {
    uint32_t at = 0, row = 0;
    for (int e0 = 0; e0 < a.local_experts; e0 += 64) {
      const int e = e0 + threadIdx.x;
      const uint32_t n =
          e < a.local_experts ? __popc(c.tokens[e][0]) + __popc(c.tokens[e][1]) : 0;
      // entries in the upper half of a word, rows in the lower
      const uint32_t own = (n + 15) / 16 << 16 | n, upto = wave_scan_add(own);
      uint32_t i = at + ((upto - own) >> 16), r = row + ((upto - own) & 0xFFFF);
      for (uint32_t g = 0; g * 16 < n; g++, i++, r += 16) {
        c.list[i] = (int16_t)(e | g << 10);
        c.rows[i] = (int16_t)r;
      }
      const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
      at += all >> 16;
      row += all & 0xFFFF;
    }
    if (threadIdx.x == 0) c.n = (int32_t)at;
  }
  __syncthreads();
}

// The n-th of the tokens, -1 without one
__device__ __forceinline__ int token_of(const uint32_t *tokens, int n) {
  const int low = __popc(tokens[0]);
  uint32_t m = n < low ? tokens[0] : tokens[1];
  int at = n < low ? 0 : 32;
  n -= n < low ? 0 : low;
  if (n >= __popc(m)) return -1;
#pragma unroll
  for (int w = 16; w; w /= 2) {
    const int c = __popc(m & ((1u << w) - 1));
    at += n >= c ? w : 0;
    m = n >= c ? m >> w : m;
    n -= n >= c ? c : 0;
  }
  return at;
}

// LDS writes of the block are done; loads from memory may be on their way
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One operand's pieces of a step of 128 bytes (two products' worth) of a row of
// K. The last step is moved back to end with the row, and what it has in common
// with the one before is cleared by finish_step(); a row shorter than a step is
// read in parts (kShort).
template <class T>
constexpr int kTokenStep = 8 * Vec<T>::kN;
template <class T, bool kShort>
__device__ __forceinline__ void load_step(Frag<T> *f, const T *p, int step, int K) {
  constexpr int N = Vec<T>::kN;
  const int q = threadIdx.x >> 4 & 3;
  const int k0 = kShort ? 0 : min(step * kTokenStep<T>, K - kTokenStep<T>);
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const int k = k0 + (h * 4 + q) * N;
    if (kShort) f[h].v = load_vec<T, true>(p + k, K - k);
    else f[h].v = *(const typename Vec<T>::U *)(p + k);
  }
}
template <class T, bool kShort>
__device__ __forceinline__ void finish_step(Frag<T> *f, int step, int K) {
  constexpr int N = Vec<T>::kN;
  const int again = (step + 1) * kTokenStep<T> - K;  // elements in common
  if (kShort || again <= 0) return;
  const int q = threadIdx.x >> 4 & 3;
#pragma unroll
  for (int h = 0; h < 2; h++) {
    Chunk v = __builtin_bit_cast(Chunk, f[h].v);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int n = again - (h * 4 + q) * N - i * (N / 4);  // of this word's elements
      v[i] &= n <= 0 ? ~0u : N == 8 && n == 1 ? 0xFFFF0000u : 0u;
    }
    f[h].v = __builtin_bit_cast(typename Vec<T>::V, v);
  }
}

// w a of 8 hidden columns of an entry per turn: 8 gate and 8 up rows of its
// expert's weights make one operand, its tokens the other; kSplit wavefronts
// take steps of 128 bytes in turn. The next steps are on their way while those
// before are multiplied, across turns too.
template <class T, int kSplit, bool kShort>
__global__ __launch_bounds__(kThreads, kPerCu) void tokens_up_kernel(TokensArgs g) {
  constexpr int U = 2;
  __shared__ Choices c;
  __shared__ F4 red[2][kWaves][64];
  const taccl_ffn_tokens_t &a = g.a;
  const int D = a.cols, F = a.hidden, tiles = g.wide / 8;
  choose_all(a, c);
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < a.tokens * a.k; i += kThreads) {
      if (a.experts) a.experts[i] = c.expert[i / a.k][i % a.k];
      if (a.weights) a.weights[i] = c.weight[i / a.k][i % a.k];
    }
    for (int i = threadIdx.x; i < c.n; i += kThreads) {
      const int e = c.list[i] & (kMaxExperts - 1), from = (c.list[i] >> 10) * 16;
      uint32_t some[2] = {c.tokens[e][0], c.tokens[e][1]};
      // without the tokens before and behind
      const int t0 = token_of(some, from), t1 = token_of(some, from + 16);
      uint64_t m = (uint64_t)some[1] << 32 | some[0];
      m &= ~0ull << t0;
      if (t1 >= 0) m &= (1ull << t1) - 1;
      g.chosen->tokens[i][0] = (uint32_t)m;
      g.chosen->tokens[i][1] = (uint32_t)(m >> 32);
      g.chosen->experts[i] = (int16_t)e;
      g.chosen->rows[i] = c.rows[i];
    }
    for (int i = threadIdx.x; i < kSplitTiles; i += kThreads) g.chosen->done[i] = 0;
    if (threadIdx.x == 0) g.chosen->n = c.n;
  }
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int steps = (D + kTokenStep<T> - 1) / kTokenStep<T>;
  const int batches = (steps + U * kSplit - 1) / (U * kSplit);

  struct Batch {
    Frag<T> w[U][2], x[U][2];
  };
  constexpr int kGroups = kWaves / kSplit;  // of wavefronts, each with turns of its own
  const int share = wave % kSplit, group = wave / kSplit;
  const int start = blockIdx.x * kGroups + group, stride = gridDim.x * kGroups;
  // the next batch to load: its turn, place in it and operands
  int next = start, part = 0;
  const T *w = nullptr, *x = nullptr;
  auto load = [&](Batch &b) {
    if (next >= c.n * tiles) return;
    if (part == 0) {
      const int entry = c.list[next / tiles], f = min(next % tiles * 8 + (r & 7), F - 1);
      const int e = entry & (kMaxExperts - 1), t = token_of(c.tokens[e], (entry >> 10) * 16 + r);
      w = (const T *)a.w_in + ((int64_t)e * 2 * F + (r < 8 ? f : F + f)) * D;
      // columns without a token take the first one's row; they are not stored
      x = (const T *)a.x + __shfl(t, t < 0 ? 0 : lane) * a.x_stride;
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int s = (part * U + u) * kSplit + share;
      if (s < steps) {
        load_step<T, kShort>(b.w[u], w, s, D);
        load_step<T, kShort>(b.x[u], x, s, D);
      }
    }
    if (++part == batches) {
      part = 0;
      next += stride;
    }
  };
  F4 acc = {0, 0, 0, 0};
  int item = start, done = 0;
  uint32_t turns = 0;
  auto multiply_batch = [&](Batch &b) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int s = (done * U + u) * kSplit + share;
      if (s < steps) {
        finish_step<T, kShort>(b.w[u], s, D);
        finish_step<T, kShort>(b.x[u], s, D);
#pragma unroll
        for (int h = 0; h < 2; h++) acc = multiply(b.w[u][h], b.x[u][h], acc);
      }
    }
    if (++done < batches) return;
    done = 0;
    const uint32_t turn = turns & 1;
    const int f = item % tiles * 8 + 4 * q, slot = item / tiles;
    item += stride;
    F4 other = acc;  // the up rows' results
    if (kSplit == 1) {
#pragma unroll
      for (int i = 0; i < 4; i++) other[i] = __shfl_xor(acc[i], 32);
    } else {
      red[turn][wave][lane] = acc;
      lds_barrier();
    }
    // the turns' sums go to the wavefronts in turn: lanes 0 to 31 take four
    // hidden columns of a token, whose gate rows they and whose up rows lanes 32
    // to 63 held
    const int e = c.list[slot] & (kMaxExperts - 1);
    const int t = q < 2 && share == (int)(turns & (kSplit - 1))
                      ? token_of(c.tokens[e], (c.list[slot] >> 10) * 16 + r) : -1;
    if (t >= 0) {
      F4 sg = acc, su = other;
      if (kSplit > 1) {
        sg = red[turn][0][lane];
        su = red[turn][0][lane + 32];
#pragma unroll
        for (int v = 1; v < kSplit; v++) {
          sg += red[turn][v][lane];
          su += red[turn][v][lane + 32];
        }
      }
      float weight = 0;
      for (int j = 0; j < a.k; j++)
        if (c.expert[t][j] == e + a.first_expert) weight = c.weight[t][j];
      F4 y;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        // 16 bits: off by up to (|g| + 12) 2^-24 of itself, 0 for an infinite exponential
        const float s = sizeof(T) == 4
                            ? 1.0f / (1.0f + expf(-sg[i]))
                            : __builtin_amdgcn_rcpf(
                                  1.0f + __builtin_amdgcn_exp2f(sg[i] * -1.4426950408889634f));
        y[i] = f + i < F ? sg[i] * s * su[i] * weight : 0.0f;
      }
      T *row = (T *)(g.act + (int64_t)(c.rows[slot] + r) * g.wide * 4) + f;
      if constexpr (sizeof(T) == 4) {
        *(F4 *)row = y;
      } else {
        typedef T T4 __attribute__((ext_vector_type(4)));
        T4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; i++) {
          hi[i] = (T)y[i];
          const float rest = y[i] - (float)hi[i];
          lo[i] = (T)(rest - rest == 0 ? rest : 0.0f);  // not of an infinite number
        }
        *(T4 *)row = hi;
        *(T4 *)(row + g.wide) = lo;
      }
    }
    acc = F4{0, 0, 0, 0};
    turns++;  // the other half's readers are behind this turn's barrier
  };
  Batch even, odd;
  load(even);
  const int end = c.n * tiles;
  while (item < end) {
    load(odd);
    multiply_batch(even);
    if (item >= end) break;
    load(even);
    multiply_batch(odd);
  }
}

// 16 columns of the output, or a part of their sum: the entries' rows of w_out
// one after the other are one long shared axis, dealt out to parts where the
// columns alone make too few blocks. The last part to arrive adds them up, in
// their order. Up to 16 tokens a column of the operand is a token; more are
// added up per wavefront in LDS, entry by entry (kFold 0). Up to 8 (4) tokens
// leave half (three quarters) of the operand's columns empty: they take the
// tokens at the next step (three steps), and the other operand's rows are 8 (4)
// columns of the output at both (four) steps. The results off this diagonal are
// dropped, and there are two (four) times the tiles, which saves the parts: the
// join takes about 3 us (4 tokens, 2 of 16 experts of 512 x 256 f32: 6.1 us with
// four parts, 5.0 folded).
template <class T, int kFold, bool kShort>
__global__ __launch_bounds__(kThreads, kDownPerCu<T>) void tokens_down_kernel(TokensArgs g) {
  constexpr int U = 2, kPlanes = sizeof(T) == 4 ? 1 : 2;
  constexpr bool kMany = kFold == 0;
  constexpr int kSteps = kMany ? 1 : kFold;     // of an operand
  constexpr int kRows = 16 / kSteps;            // columns of the output
  constexpr int kTok = kMany ? kTokens : kRows;  // tokens
  __shared__ F4 sums[kWaves * kSteps][kTok][kRows / 4];
  __shared__ uint32_t tokens[kMaxEntries][2];
  __shared__ int16_t experts[kMaxEntries], rows[kMaxEntries];
  __shared__ int last;
  const taccl_ffn_tokens_t &a = g.a;
  const int D = a.cols, F = a.hidden, n = g.chosen->n;
  // those past the n-th are not used: n is on its way too
  for (int i = threadIdx.x; i < g.most; i += kThreads) {
    tokens[i][0] = g.chosen->tokens[i][0];
    tokens[i][1] = g.chosen->tokens[i][1];
    rows[i] = g.chosen->rows[i];
    experts[i] = g.chosen->experts[i];
  }
  if (kMany)
    for (int i = threadIdx.x; i < kWaves * kTok * (kRows / 4); i += kThreads)
      (&sums[0][0][0])[i] = F4{0, 0, 0, 0};
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int tile = blockIdx.x / g.parts, part = blockIdx.x % g.parts, d0 = tile * kRows;
  const int steps = (F + kTokenStep<T> - 1) / kTokenStep<T>;

  struct Batch {
    Frag<T> w[U][2], x[U][kPlanes][2];
    int slot[U], step[U];
    bool there[U];
  };
  // rows and columns r, r + kRows, ... of the operands are at steps one later each
  const int own = r % kRows, later = r / kRows;
  const T *first = (const T *)a.w_out + (int64_t)min(d0 + own, D - 1) * F;
  // of the part's steps every kWaves-th, or every kWaves-th few
  const int64_t all = (int64_t)n * steps, begin = all * part / g.parts;
  const int64_t end = all * (part + 1) / g.parts, from = begin + wave * kSteps;
  const int count =
      from < end ? (int)((end - from + kWaves * kSteps - 1) / (kWaves * kSteps)) : 0;
  const int rest = (int)min(end - from - later, (int64_t)1 << 30);  // steps from the lane's first on
  int slot = 0, s = 0;
  if (count) {
    slot = (int)((from + later) / steps);
    s = (int)((from + later) % steps);
  }
  int loaded = 0, done = 0;
  auto load = [&](Batch &b) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (loaded + u >= count) continue;
      b.slot[u] = slot;
      b.step[u] = s;
      const bool in = kSteps == 1 || (loaded + u) * (kWaves * kSteps) < rest;
      if (kSteps > 1) {
        b.w[u][0].v = b.w[u][1].v = typename Vec<T>::V{};
      }
      // the token's row, or zeros
      int row = 0;
      bool &there = b.there[u];
      there = false;
      if (in) {
        load_step<T, kShort>(b.w[u], first + (int64_t)experts[slot] * D * F, s, F);
        const uint32_t low = tokens[slot][0], high = tokens[slot][1];
        if (kMany) {
          there = r < __popc(low) + __popc(high);
          row = rows[slot] + r;
        } else {
          there = low >> own & 1;
          row = rows[slot] + __popc(low & ((1u << own) - 1));
        }
      }
#pragma unroll
      for (int p = 0; p < kPlanes; p++) {
        b.x[u][p][0].v = b.x[u][p][1].v = typename Vec<T>::V{};
        if (there)
          load_step<T, kShort>(b.x[u][p],
                               (const T *)(g.act + (int64_t)row * g.wide * 4) + p * g.wide, s, F);
      }
      s += kWaves * kSteps;
      while (s >= steps) {
        s -= steps;
        slot++;
      }
    }
    loaded += U;
  };
  F4 acc = {0, 0, 0, 0};
  int now = count ? slot : 0;  // the entry that acc belongs to
  auto flush = [&]() {
    const int t = token_of(tokens[now], r);
    if (t >= 0) sums[wave][t][q] += acc;
    acc = F4{0, 0, 0, 0};
  };
  auto multiply_batch = [&](Batch &b) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (done + u >= count) continue;
      if (kMany && b.slot[u] != now) {
        flush();
        now = b.slot[u];
      }
      finish_step<T, kShort>(b.w[u], b.step[u], F);
      F4 sum = acc;
#pragma unroll
      for (int p = 0; p < kPlanes; p++) {
        finish_step<T, kShort>(b.x[u][p], b.step[u], F);
#pragma unroll
        for (int h = 0; h < 2; h++) sum = multiply(b.w[u][h], b.x[u][p][h], sum);
      }
      // zero times an infinite or NaN weight of an expert that the token did not choose
#pragma unroll
      for (int i = 0; i < 4; i++) acc[i] = kMany || b.there[u] ? sum[i] : acc[i];
    }
    done += U;
  };
  Batch even, odd;
  load(even);
  while (done < count) {
    load(odd);
    multiply_batch(even);
    load(even);
    multiply_batch(odd);
  }
  if (kMany) {
    if (count) flush();
  } else if (q * 4 / kRows == later) {
    sums[wave * kSteps + later][own][q % (kRows / 4)] = acc;
  }
  __syncthreads();

  // thread (t, c): four columns of a token
  const int t = threadIdx.x / (kRows / 4), c = threadIdx.x % (kRows / 4);
  const bool mine = t < a.tokens;
  F4 y = {0, 0, 0, 0};
  if (mine) {
    y = sums[0][t][c];
#pragma unroll
    for (int v = 1; v < kWaves * kSteps; v++) y += sums[v][t][c];
  }
  if (g.parts > 1) {
    const int64_t stride = (int64_t)(gridDim.x / g.parts) * a.tokens * (kRows / 4);
    float *partial = (float *)(g.partial + ((int64_t)tile * a.tokens + t) * (kRows / 4) + c);
    if (mine) put(partial + part * stride * 4, y);
    if (!last_of(&g.chosen->done[tile], g.parts, &last)) return;
    if (mine) {
      y = get(partial);
      for (int p = 1; p < g.parts; p++) y += get(partial + p * stride * 4);
    }
  }
  if (mine) {
    const int d = d0 + 4 * c;
    T *out = (T *)a.out + t * a.out_stride + d;
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (d + i < D) out[i] = (T)y[i];
  }
}

template <class T, int kSplit>
const void *up_fn(int cols) {
  return cols < kTokenStep<T> ? (const void *)tokens_up_kernel<T, kSplit, true>
                              : (const void *)tokens_up_kernel<T, kSplit, false>;
}
template <class T>
const void *up_fn(int cols, bool split) {
  return split ? up_fn<T, kWaves>(cols) : up_fn<T, 1>(cols);
}

template <class T, int kFold>
const void *down_fn(int hidden) {
  return hidden < kTokenStep<T> ? (const void *)tokens_down_kernel<T, kFold, true>
                                : (const void *)tokens_down_kernel<T, kFold, false>;
}
template <class T>
const void *down_fn(int hidden, int fold) {
  return fold == 0   ? down_fn<T, 0>(hidden)
         : fold == 1 ? down_fn<T, 1>(hidden)
         : fold == 2 ? down_fn<T, 2>(hidden)
                     : down_fn<T, 4>(hidden);
}

int64_t act_bytes(int64_t tokens, int64_t k, int64_t hidden) {
  return tokens * k * hidden_wide(hidden) * 4;
}

}  // namespace

int64_t ffn_tokens_space(int64_t tokens, int64_t k, int64_t cols, int64_t hidden) {
  return kChosenBytes + act_bytes(tokens, k, hidden) +
         kMaxParts * ((cols + 15) / 16) * tokens * 64;
}

hipError_t launch_ffn_tokens(const taccl_ffn_tokens_t &a, int cus, hipStream_t stream) {
  uint8_t *ws = (uint8_t *)a.workspace;
  TokensArgs g{a, (Chosen *)ws, ws + kChosenBytes, nullptr, (int32_t)hidden_wide(a.hidden), 1, 0};
  g.partial = (F4 *)(g.act + act_bytes(a.tokens, a.k, a.hidden));
  void *args[] = {&g};
#define BY_TYPE(F, ...)                              \
  (a.dtype == TACCL_F32    ? F<float>(__VA_ARGS__)   \
   : a.dtype == TACCL_BF16 ? F<bf16_t>(__VA_ARGS__)  \
                           : F<f16_t>(__VA_ARGS__))
  // entries, at most
  const int64_t choices = a.tokens * a.k;
  const int64_t most = std::min<int64_t>(choices, a.local_experts + choices / 16);
  // Where every wavefront has turns of its own, a row of few steps stays with one,
  // without a join per turn (us a call, shared and not: 20 tokens, 8 of 68 experts
  // of 64 x 3392 f32 134 and 93; 16, 8 of 64 of 512 x 2048 bf16 92 and 81; 64, 8 of
  // 64 of 1024 x 1024 120 and 116; but one token, 4 of 64 of 256 x 1024 10.9 and 11.6).
  const int n = a.dtype == TACCL_F32 ? 4 : 8;
  const int64_t turns = most * (g.wide / 8), row_steps = (a.cols + 8 * n - 1) / (8 * n);
  const bool split = row_steps > 16 || turns < kWaves * kPerCu * cus;
  const int64_t blocks =
      std::min<int64_t>(split ? turns : (turns + kWaves - 1) / kWaves, kPerCu * cus);
  g.most = (int32_t)most;
  hipError_t e = hipLaunchKernel(BY_TYPE(up_fn, a.cols, split), dim3((uint32_t)blocks), dim3(kThreads),
                                 args, 0, stream);
  if (e != hipSuccess) return e;
  // the smallest tiles that the chip holds at once, then parts of at least eight
  // operands' steps per wavefront, if that many entries are there
  const int64_t held = (a.dtype == TACCL_F32 ? kDownPerCu<float> : kDownPerCu<bf16_t>) * cus;
  int fold = a.tokens > 16 ? 0 : a.tokens > 8 ? 1 : a.tokens > 4 ? 2 : 4;
  auto tiles_of = [&](int64_t f) { return (a.cols * std::max<int64_t>(f, 1) + 15) / 16; };
  while (fold > 1 && tiles_of(fold) > held) fold /= 2;
  const int64_t tiles = tiles_of(fold), steps = most * ((a.hidden + 8 * n - 1) / (8 * n));
  g.parts = (int)std::max<int64_t>(
      1, std::min<int64_t>({held / tiles, steps / (8 * kWaves * std::max(fold, 1)), kMaxParts}));
  return hipLaunchKernel(BY_TYPE(down_fn, a.hidden, fold), dim3((uint32_t)(tiles * g.parts)),
                         dim3(kThreads), args, 0, stream);
#undef BY_TYPE
}

}  // namespace taccl
