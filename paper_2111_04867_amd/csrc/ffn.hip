// Experts' gated feed-forward on the rows that an Alltoall brings, and its
// gradient.
//
//   g = x Wg^T, u = x Wu^T, a = silu(g) u, y = a Wo^T
//   da = dy Wo, dg = da u s (1 + g (1 - s)), du = da g s, s = 1 / (1 + exp(-g))
//   dx = dg Wg + du Wu, dWo = dy^T a, dWg = dg^T x, dWu = du^T x
//
// An expert's rows of all sources count as one matrix: a first small launch
// numbers the rows below the counts, lists the tiles of rows that exist, and
// zeroes the rows of the output past the counts. The products follow, two
// forward and four backward, on the matrix units (tile.h).
//
// Sums are 32-bit floats, one after the other along a block's part of the shared
// axis. Between the products a, dg and du are rounded to the arrays' type, as they
// are operands of matrix instructions of that type: for 16 bits that makes the
// error of a result 0.0023 of its size (bf16) instead of 0.0017, 0.00029 (f16)
// instead of 0.00021. Held as two 16-bit numbers they would double the operand's
// bytes and its product's instructions, which bound these products.
//
// What bounds them: loads of tiles from L2, and what a tile does before its first
// and behind its last step. 64 experts, 980 rows of 4096 bf16 each, hidden 1536: 1466
// and 816 us forward (1070 and 960 TFLOP/s over the rows, 63 and 56% of the
// matrix units' time; loading the tiles alone takes as long). The gradient of
// 490 rows of 2048, hidden 1024: 246 us dg and du, 318 dx, 367 and 197 dw_in and
// dw_out, which store 0.8 GB behind eight steps a tile.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "expert.h"
#include "ffn.h"
#include "tile.h"

namespace taccl {

namespace {

struct FfnTile {
  int32_t expert, row;
};

constexpr int kPlanThreads = 256;

int64_t rounded(int64_t n) { return (n + 255) / 256 * 256; }

// rows of a tile: each size has its own list, 2^(5 + i) rows in list i
constexpr int kLists = 4;
constexpr int64_t list_rows(int i) { return 32 << i; }
constexpr int list_of(int rows) { return rows == 256 ? 3 : rows == 128 ? 2 : rows == 64 ? 1 : 0; }

}  // namespace

FfnSpace ffn_space(int64_t sources, int64_t experts, int64_t capacity, int64_t hidden, int dtype,
                   bool backward) {
  const int64_t slots = sources * capacity, rows = experts * slots;
  const int64_t size = dtype == TACCL_F32 ? 4 : 2;
  FfnSpace s{};
  s.num_tiles = rounded(4 * experts);
  int64_t at = s.num_tiles + 256;
  for (int i = 0; i < kLists; i++) {
    s.tiles[i] = at;
    at += rounded(8 * experts * ((slots + list_rows(i) - 1) / list_rows(i)));
  }
  s.map = at;
  s.act = s.map + (sources > 1 ? rounded(4 * rows) : 0);
  s.dpre = s.act + rounded(rows * hidden * size);
  s.done = s.dpre + (backward ? rounded(2 * rows * hidden * size) : 0);
  s.partial = s.done + 4 * 4 * kSplitTiles;
  // parts are worth it where a product has few tiles, small ones, and weights'
  // gradients over many rows, or few in its last turn
  s.least = s.partial + rounded(std::min<int64_t>(64 << 20, (3 << 18) + 64 * rows));
  s.bytes = s.partial + rounded(std::min<int64_t>(64 << 20, (3 << 19) + 8192 * rows));
  return s;
}

namespace {

struct PlanArgs {
  const int32_t *counts;  // [S][E]
  int64_t capacity;
  int32_t sources, experts;
  int32_t map_parts, zero_parts;  // blocks per expert, per source and expert
  int32_t *rows, *num_tiles, *map;  // map: or null
  FfnTile *tiles[kLists];
  int32_t lists;  // bits: those that a product reads
  int32_t *done;  // zeroed
  uint8_t *zero;  // rows past the counts are zeroed; or null
  int64_t row_bytes;
};

__device__ __forceinline__ int32_t rows_of(const PlanArgs &g, int64_t i) {
  return (int32_t)min((int64_t)max(g.counts[i], 0), g.capacity);
}

// Inclusive sum over the block's threads of v; `all` becomes the total
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *red, uint32_t &all) {
  const uint32_t own = wave_scan_add(v), w = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) red[w] = own;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (uint32_t i = 0; i < kPlanThreads / 64; i++) {
    before += i < w ? red[i] : 0;
    all += red[i];
  }
  return own + before;
}

// Block 0 counts and lists; then come the blocks that number an expert's rows
// and those that zero a source's rows of an expert.
__global__ __launch_bounds__(kPlanThreads) void ffn_plan_kernel(PlanArgs g) {
  __shared__ uint32_t red[kPlanThreads / 64];
  __shared__ int32_t rows[kMaxExperts];
  __shared__ uint32_t from[kMaxExperts + 1];  // an expert's first tile, a source's first row
  const int E = g.experts, S = g.sources;
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < 4 * kSplitTiles; i += kPlanThreads) g.done[i] = 0;
    for (int e = threadIdx.x; e < E; e += kPlanThreads) rows[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < S * E; i += kPlanThreads) atomicAdd(&rows[i % E], rows_of(g, i));
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kPlanThreads) g.rows[e] = rows[e];
    for (int l = 0; l < kLists; l++) {
      if (!(g.lists >> l & 1)) continue;
      const uint32_t tile = (uint32_t)list_rows(l);
      uint32_t total = 0;
      for (int e0 = 0; e0 < E; e0 += kPlanThreads) {
        const int e = e0 + threadIdx.x;
        const uint32_t mine = e < E ? ((uint32_t)rows[e] + tile - 1) / tile : 0;
        uint32_t all;
        const uint32_t upto = total + block_scan(mine, red, all);
        if (e < E) from[e + 1] = upto;
        total += all;
      }
      if (threadIdx.x == 0) {
        from[0] = 0;
        g.num_tiles[l] = (int32_t)total;
      }
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < total; i += kPlanThreads) {
        int e = 0;  // the last expert whose first tile is not behind i, among those with tiles
        for (int n = E; n > 1; n = (n + 1) / 2)
          if (e + n / 2 < E && from[e + n / 2] <= i) e += n / 2;
        g.tiles[l][i] = FfnTile{e, (int32_t)((i - from[e]) * tile)};
      }
      __syncthreads();
    }
    return;
  }
  int b = blockIdx.x - 1;
  if (b < E * g.map_parts) {
    const int e = b % E, part = b / E;
    int32_t *map = g.map + e * S * g.capacity;
    uint32_t first = 0;
    for (int s0 = 0; s0 < S; s0 += kPlanThreads) {
      const int s = s0 + threadIdx.x;
      const uint32_t n = s < S ? (uint32_t)rows_of(g, (int64_t)s * E + e) : 0;
      uint32_t all;
      const uint32_t upto = block_scan(n, red, all);
      if (threadIdx.x == 0) from[0] = 0;
      from[threadIdx.x + 1] = upto;
      __syncthreads();
      // the rows of these sources, a row per thread and turn
      for (uint32_t i = part * kPlanThreads + threadIdx.x; i < all;
           i += g.map_parts * kPlanThreads) {
        int at = 0;
#pragma unroll
        for (int n = kPlanThreads / 2; n; n /= 2)
          if (from[at + n] <= i) at += n;
        map[first + i] = (int32_t)(((int64_t)(s0 + at) * E + e) * g.capacity + (i - from[at]));
      }
      first += all;
      __syncthreads();
    }
    return;
  }
  b -= E * g.map_parts;
  const int i = b % (S * E), part = b / (S * E);
  const int64_t n = rows_of(g, i);
  zero_piece<kPlanThreads>(g.zero + (i * g.capacity + n) * g.row_bytes,
                           (g.capacity - n) * g.row_bytes, part, g.zero_parts);
}

// The products. kUp: a from x and w_in (and the stored g, u); kDown: y from a
// and w_out; kGrad: dg, du (and a again) from dy, w_out and the stored g, u;
// kDx: dx from dg, du and w_in; kDwOut, kDwIn: the weights' gradients.
enum Kind { kUp, kDown, kGrad, kDx, kDwOut, kDwIn };

struct ProductArgs {
  const void *a, *b;
  void *out, *more;  // kUp: a, pre (or null); kGrad: dpre, a
  const void *pre;   // kGrad
  const int32_t *rows, *num_tiles, *map;
  const FfnTile *tiles;
  int64_t slots;  // sources * capacity
  int32_t cols, hidden, experts;
  int32_t row_tiles, col_tiles;  // kDw*: tiles of an expert; else row_tiles is unused
  int32_t parts;   // blocks that share a tile's steps
  // The chip holds `round` blocks (0: not looked at). Where the last tiles are
  // fewer, up to `last_parts` blocks share one of them, `room` parts in all.
  uint32_t round, last_parts, room;
  int32_t *done;   // [tiles]
  float *partial;  // [tiles][parts][tile]
};

template <class T>
__device__ __forceinline__ float sigmoid(float g) {
  if constexpr (sizeof(T) == 4) return 1.0f / (1.0f + expf(-g));
  // off by up to (|g| + 12) 2^-24 of itself: the exponent's product is rounded, which
  // the exponential multiplies by |g|, then the exponential and the reciprocal are
  // within two units each. Where the exponential is finite, |g| < 89, that is 6e-6,
  // an eightieth of a 16-bit result's own rounding; 0 where it is infinite.
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
}

// A tile of BM rows by BN columns, by WM x WN wavefronts; LDS holds SA steps of
// the rows and SB of the columns.
template <int M, int N, int kM, int kN, int kA, int kB>
struct Shape {
  static constexpr int BM = M, BN = N, WM = kM, WN = kN, SA = kA, SB = kB;
  static constexpr int kThreads = 64 * WM * WN, kLds = (SA * BM + SB * BN) * kStepBytes;
};

template <class T, int kKind, bool kMapped, bool kFast, class Z>
__device__ __forceinline__ void product(const ProductArgs &g, uint32_t b, char *lds) {
  constexpr bool kWeights = kKind == kDwOut || kKind == kDwIn;
  constexpr bool kAcrossA = kWeights, kAcrossB = kKind != kUp && kKind != kDown;
  constexpr int BM = Z::BM, BN = Z::BN, WM = Z::WM, WN = Z::WN;
  constexpr int SA = Z::SA, SB = Z::SB;
  constexpr int kThreads = Z::kThreads, MI = BM / WM / 16, NI = BN / WN / 16;
  constexpr int kTileA = BM * kStepBytes, kTileB = BN * kStepBytes;
  char *const lds_b = lds + SA * kTileA;
  const int D = g.cols, F = g.hidden;

  // Blocks go to the XCDs in turn; 32 consecutive ones of an XCD take a piece
  // of 8 tiles of columns by 4 of rows, whose operands its L2 holds. The pieces'
  // rows of tiles start at different steps: rows a power of two apart have one
  // step in few of the L2's channels (1480 us to 1463 for the up projection).
  const uint32_t per_xcd = b >> 3;
  const uint32_t place_of = ((per_xcd >> 5) * 8 + (b & 7)) * 32 + (per_xcd & 31);
  const uint32_t entries = kWeights ? (uint32_t)(g.experts * g.row_tiles) : (uint32_t)*g.num_tiles;
  uint32_t parts = (uint32_t)g.parts, alone = 0;  // tiles that are not shared
  if (g.round) {
    const uint32_t all = entries * (uint32_t)g.col_tiles, last = all % g.round;
    if (last && place_of >= all - last) {
      parts = max(1u, min(g.last_parts, g.room / last));
      alone = all - last;
    }
  }
  const uint32_t id = alone + (place_of - alone) / parts, part = (place_of - alone) % parts;
  const uint32_t group = id / (entries * 8), width = min(8u, (uint32_t)g.col_tiles - group * 8);
  if (entries == 0 || group * 8 >= (uint32_t)g.col_tiles) return;
  const uint32_t in = id - group * entries * 8, entry = in / width;
  if (entry >= entries) return;
  const int tn = (int)(group * 8 + in % width);
  FfnTile t;
  if (kWeights) t = FfnTile{(int)(entry / g.row_tiles), (int)(entry % g.row_tiles) * BM};
  else t = g.tiles[entry];
  const int e = t.expert, n = g.rows[e];
  const int64_t first = e * g.slots;
  const int32_t *map = g.map ? g.map + first : nullptr;

  // operands: the buffer's rows by their numbers, compact rows, weights
  Operand<T> oa, ob;
  constexpr bool kBufferA = kKind == kUp || kKind == kGrad || kKind == kDwOut;
  const int lda = kKind == kDown ? F : kKind == kDx || kKind == kDwIn ? 2 * F : D;
  oa.p = (const T *)g.a + (kBufferA && map ? 0 : first * lda);
  oa.end = (const T *)g.a + (int64_t)g.experts * g.slots * lda;
  oa.ld = lda;
  oa.map = kBufferA ? map : nullptr;
  const int ldb = kKind == kUp || kKind == kDx || kKind == kDwIn ? D : F;
  if (kWeights) ob.p = (const T *)g.b + (kKind == kDwIn && map ? 0 : first * ldb);
  else ob.p = (const T *)g.b + (int64_t)e * D * F * (kKind == kUp || kKind == kDx ? 2 : 1);
  ob.end = (const T *)g.b + (kWeights ? g.slots * ldb
                             : (int64_t)D * F * (kKind == kUp || kKind == kDx ? 2 : 1)) * g.experts;
  ob.ld = ldb;
  ob.map = kKind == kDwIn ? map : nullptr;
  const int K = kWeights ? n : kKind == kDown ? F : kKind == kDx ? 2 * F : D;
  // columns of the product; the up projection's tile has gate and up columns,
  // half each, of as many hidden ones
  constexpr int kCols = kKind == kUp ? BN / 2 : BN;
  const int N = kKind == kUp || kKind == kGrad || kKind == kDwOut ? F : D;
  const int M = kKind == kDwOut ? D : kKind == kDwIn ? 2 * F : n;
  const int n0 = tn * kCols;

  Loader<T, kAcrossA, kMapped && kKind == kDwOut, kFast, BM, kThreads> la;
  Loader<T, kAcrossB, kMapped && kKind == kDwIn, kFast, BN, kThreads> lb;
  if constexpr (kAcrossA) la.across(oa, K, t.row, M);
  else la.along(oa, K, [&](int r) { return min(t.row + r, M - 1); });
  if constexpr (kAcrossB) {
    lb.across(ob, K, n0, N);
  } else if constexpr (kKind == kUp) {
    // a wavefront's columns: its gate ones, then its up ones
    lb.along(ob, K, [&](int r) {
      const int w = r / (16 * NI), q = r % (16 * NI);
      return (q < 8 * NI ? 0 : F) + min(n0 + w * 8 * NI + q % (8 * NI), F - 1);
    });
  } else {
    lb.along(ob, K, [&](int r) { return min(n0 + r, N - 1); });
  }

  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wm = wave / WN * (16 * MI), wn = wave % WN * (16 * NI);
  F4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; i++)
#pragma unroll
    for (int j = 0; j < NI; j++) acc[i][j] = F4{0, 0, 0, 0};

  constexpr int kStep = kStepBytes / (int)sizeof(T);
  // This part's steps: from the `first_step`-th on, at most 2^16 of up to 16 parts.
  // Fixed here in scalar registers: the loop is laid out worse where the compiler
  // carries on with the number of parts that the tile list decides (gradient of 8 x
  // 600 rows of 2048 f32, hidden 1024: 1237 us a call, so 1203).
  const int all_steps = (K + kStep - 1) / kStep;
  int first_step = (int)((uint32_t)all_steps * part / parts);
  asm volatile("" : "+s"(first_step));
  int steps = (int)((uint32_t)all_steps * (part + 1) / parts) - first_step;
  asm volatile("" : "+s"(steps));
  constexpr int kLoads = la.kLoads + lb.kLoads;
  const int turn = kFast ? (int)((uint64_t)steps * (id >> 3 & 31) / 32) : 0;
  auto place = [&](int s) {  // in the shared axis, of step s; past the end its end
    if (s >= steps) return all_steps * kStep;
    return (first_step + (s + turn >= steps ? s + turn - steps : s + turn)) * kStep;
  };
  // A step's products, row of parts by row, whose operands are read two rows
  // ahead; `ahead(q)` is called before row q. The order is kept as it stands:
  // by itself the compiler reads an operand right where it is needed.
  auto multiply_step = [&](const char *from_a, const char *from_b, auto ahead) {
    constexpr int kHalves = 2, kDepth = MI < 2 ? 1 : 2;
    Frag<T> fa[kHalves][MI], fb[kHalves][NI];
    auto read_a = [&](int q) {
      fa[q / MI][q % MI] = read_frag<T, kAcrossA, BM>(from_a, wm + 16 * (q % MI), q / MI);
    };
    auto read_b = [&](int h, int j) {
      fb[h][j] = read_frag<T, kAcrossB, BN>(from_b, wn + 16 * j, h);
    };
#pragma unroll
    for (int j = 0; j < NI; j++) read_b(0, j);
#pragma unroll
    for (int q = 0; q < kDepth; q++) read_a(q);
#pragma unroll
    for (int q = 0; q < kHalves * MI; q++) {
      if (q + kDepth < kHalves * MI) read_a(q + kDepth);
      if (q / MI + 1 < kHalves && q % MI >= MI - kDepth) {
#pragma unroll
        for (int j = 0; j < NI / kDepth; j++)
          read_b(q / MI + 1, (q % MI - (MI - kDepth)) * (NI / kDepth) + j);
      }
      ahead(q);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < NI; j++)
        acc[q % MI][j] = multiply(fb[q / MI][j], fa[q / MI][q % MI], acc[q % MI][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if constexpr (kFast) {
    // Every step loads, past the end zeros that nothing uses, so that a step's
    // loads are there when no more than those of SA - 2 and SB - 2 steps are on
    // their way.
    static_assert(SA >= SB && SB >= 2);
    auto load_a = [&](int i, int s, char *to) { la.load(i, place(s), to); };
    auto load_b = [&](int i, int s, char *to) { lb.load(i, place(s), to); };
    // Rows looked up are waited for with all loads on their way, which are none
    // behind the barrier of two steps.
    static_assert(!kMapped || (SA == 2 && SB == 2));
    auto look_up = [&](int s) {
      la.look_up(place(s));
      lb.look_up(place(s));
    };
    look_up(0);
#pragma unroll
    for (int s = 0; s < SA - 1; s++) {
      if (s < SB - 1)
#pragma unroll
        for (int i = 0; i < lb.kLoads; i++) load_b(i, s, lds_b + s * kTileB);
#pragma unroll
      for (int i = 0; i < la.kLoads; i++) load_a(i, s, lds + s * kTileA);
    }
    look_up(1);
    int now_a = 0, now_b = 0;
    for (int s = 0; s < steps; s++) {
      tile_barrier<la.kLoads *(SA - 2) + lb.kLoads *(SB - 2)>();
      char *next_a = lds + (now_a == 0 ? SA - 1 : now_a - 1) * kTileA;
      char *next_b = lds_b + (now_b == 0 ? SB - 1 : now_b - 1) * kTileB;
      multiply_step(lds + now_a * kTileA, lds_b + now_b * kTileB, [&](int q) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
          if (i < q * kLoads / MI || i >= (q + 1) * kLoads / MI) continue;
          if (i < lb.kLoads) load_b(i, s + SB - 1, next_b);
          else load_a(i - lb.kLoads, s + SA - 1, next_a);
        }
        if (q == MI) look_up(s + 2);
      });
      now_a = now_a == SA - 1 ? 0 : now_a + 1;
      now_b = now_b == SB - 1 ? 0 : now_b + 1;
    }
  } else {
    // Chunks wait in registers, those of two steps on their way. Steps with parts
    // of chunks come last, one at a time: their loads have branches, behind
    // which the compiler waits for everything on its way (in one loop with the
    // others the gradient of 32 x 640 rows of 2047 f16, hidden 1023, took 1399 us,
    // 983 so).
    Chunk held[2][kLoads];
    auto fetch = [&](Chunk(&h)[kLoads], int s, const auto &a, const auto &b) {
#pragma unroll
      for (int i = 0; i < kLoads; i++)
        h[i] = i < a.kLoads ? a.fetch_whole(i, place(s)) : b.fetch_whole(i - a.kLoads, place(s));
    };
    auto keep = [&](const Chunk(&h)[kLoads], int odd) {
#pragma unroll
      for (int i = 0; i < kLoads; i++) {
        char *to = i < la.kLoads ? lds + odd * kTileA : lds_b + odd * kTileB;
        *(Chunk *)(to + ((i < la.kLoads ? i : i - la.kLoads) * kThreads + threadIdx.x) * 16) = h[i];
      }
    };
    const int whole = min(min(la.whole_steps(), lb.whole_steps()) - first_step, steps);
    auto look_up = [&](int s) {
      la.look_up(place(s));
      lb.look_up(place(s));
    };
    if (whole > 0) {
      look_up(0);
      fetch(held[0], 0, la, lb);
      look_up(min(1, whole - 1));
      fetch(held[1], min(1, whole - 1), la, lb);
      look_up(min(2, whole - 1));
      keep(held[0], 0);
      auto step = [&](int s, Chunk(&old)[kLoads], Chunk(&later)[kLoads]) {
        tile_barrier<63>();  // of LDS alone
        const auto a = la;  // with the rows of this step
        const auto b = lb;
        look_up(min(s + 3, whole - 1));
        fetch(old, min(s + 2, whole - 1), a, b);
        multiply_step(lds + (s & 1) * kTileA, lds_b + (s & 1) * kTileB, [](int) {});
        keep(later, ~s & 1);
      };
      int s = 0;
      for (; s + 1 < whole; s += 2) {
        step(s, held[0], held[1]);
        step(s + 1, held[1], held[0]);
      }
      if (s < whole) step(s, held[0], held[1]);
    }
    for (int s = max(whole, 0); s < steps; s++) {
      tile_barrier<63>();
      look_up(s);
#pragma unroll
      for (int i = 0; i < kLoads; i++)
        held[0][i] = i < la.kLoads ? la.fetch(i, place(s)) : lb.fetch(i - la.kLoads, place(s));
      keep(held[0], 0);
      tile_barrier<63>();
      multiply_step(lds, lds_b, [](int) {});
    }
  }

  // Lane l has columns l / 16 * 4 + 0..3 of row l % 16 of every 16 x 16 part.
  // Each wavefront passes 16 rows at a time through LDS of its own, so that a
  // row's results leave in whole chunks next to each other (stored as they are,
  // 8 bytes here and there, the four products of the gradient of 64 x 490 rows
  // took 1583 us instead of 1440).
  tile_barrier<0>();
  if (parts > 1) {
    const uint32_t tile = id - alone;
    constexpr int kAll = MI * NI, kOnce = kAll < 16 ? kAll : 16;
    float *sums = g.partial + (int64_t)tile * parts * (BM * BN) + wave * (kAll * 256) + lane * 4;
    put_ready();
#pragma unroll
    for (int i = 0; i < kAll; i++) put_chunk(sums + part * (BM * BN) + i * 256, acc[i / NI][i % NI]);
    if (!last_of(g.done + tile, (int)parts, (int32_t *)lds)) return;
    // in their order, whichever was last
    for (int p = 0; p < (int)parts; p++)
#pragma unroll
      for (int i0 = 0; i0 < kAll; i0 += kOnce) {
        F4 v[kOnce];
        get_chunks(v, sums + p * (BM * BN) + i0 * 256);
#pragma unroll
        for (int i = 0; i < kOnce; i++) {
          F4 &sum = acc[(i0 + i) / NI][(i0 + i) % NI];
          sum = p ? sum + v[i] : v[i];
        }
      }
    __syncthreads();
  }
  constexpr int kN = Vec<T>::kN, kPitch = 16 * NI * 4 + 16;
  constexpr int kPer = (kKind == kUp ? 8 : 16) * NI / kN;  // chunks of a row
  char *own = lds + wave * (16 * kPitch);
#pragma unroll
  for (int i = 0; i < MI; i++) {
#pragma unroll
    for (int j = 0; j < NI; j++)
      *(F4 *)(own + (lane & 15) * kPitch + (16 * j + (lane >> 4) * 4) * 4) = acc[i][j];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int it = 0; it < (16 * kPer + 63) / 64; it++) {
      const int id = it * 64 + lane, r = id / kPer, c = id % kPer * kN;
      const int m = t.row + wm + 16 * i + r;
      if (r >= 16 || m >= M) continue;
      const char *from = own + r * kPitch + c * 4;
      const int64_t compact = first + m, row = kWeights ? 0 : map ? map[m] : compact;
      if constexpr (kKind == kUp) {
        const int f = n0 + wn / 2 + c, left = F - f;
        typename Vec<T>::V a, gate, up;
#pragma unroll
        for (int x = 0; x < kN; x++) {
          const float vg = *(const float *)(from + 4 * x);
          const float vu = *(const float *)(from + 32 * NI + 4 * x);
          gate[x] = (T)vg;
          up[x] = (T)vu;
          a[x] = (T)(vg * sigmoid<T>(vg) * vu);
        }
        store_vec<T, !kFast>((T *)g.out + compact * F + f, a, left);
        if (g.more) {
          T *pre = (T *)g.more + row * 2 * F + f;
          store_vec<T, !kFast>(pre, gate, left);
          store_vec<T, !kFast>(pre + F, up, left);
        }
      } else if constexpr (kKind == kGrad) {
        const int f = n0 + wn + c, left = F - f;
        const T *pre = (const T *)g.pre + row * 2 * F + f;
        const auto gate = load_vec<T, !kFast>(pre, left), up = load_vec<T, !kFast>(pre + F, left);
        typename Vec<T>::V a, dg, du;
#pragma unroll
        for (int x = 0; x < kN; x++) {
          const float vg = (float)gate[x], vu = (float)up[x], sg = sigmoid<T>(vg), act = vg * sg;
          const float da = *(const float *)(from + 4 * x);
          a[x] = (T)(act * vu);
          du[x] = (T)(da * act);
          dg[x] = (T)(da * vu * (sg * (1.0f + vg * (1.0f - sg))));
        }
        T *dpre = (T *)g.out + compact * 2 * F + f;
        store_vec<T, !kFast>(dpre, dg, left);
        store_vec<T, !kFast>(dpre + F, du, left);
        store_vec<T, !kFast>((T *)g.more + compact * F + f, a, left);
      } else {
        const int64_t to = kKind == kDwOut  ? (int64_t)e * D + m
                           : kKind == kDwIn ? (int64_t)e * 2 * F + m
                                            : row;
        typename Vec<T>::V v;
#pragma unroll
        for (int x = 0; x < kN; x++) v[x] = (T)*(const float *)(from + 4 * x);
        store_vec<T, !kFast>((T *)g.out + to * N + n0 + wn + c, v, N - (n0 + wn + c));
      }
    }
    // the next rows' writes stay behind these reads
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// LDS up to its 160 KB: as many bytes on their way as it holds (256 x 128: 2020 us
// with two steps, 1701 with three for the up projection above)
using Tiny = Shape<32, 64, 2, 2, 4, 4>;
using Small = Shape<64, 64, 2, 2, 2, 2>;
using Medium = Shape<128, 128, 2, 2, 2, 2>;
using Wide = Shape<128, 256, 2, 4, 3, 3>;
using Large = Shape<256, 256, 2, 4, 3, 2>;
using MappedWide = Shape<128, 256, 2, 4, 2, 2>;
using MappedLarge = Shape<256, 256, 2, 4, 2, 2>;
enum Size { kTiny, kSmall, kMedium, kWide, kLarge };

template <class T, int kKind, bool kMapped, bool kFast, class Z>
__global__ __launch_bounds__(Z::kThreads, Z::BM == 64 ? 4 : 2) void ffn_product_kernel(ProductArgs g) {
  extern __shared__ __align__(16) char lds[];
  product<T, kKind, kMapped, kFast, Z>(g, blockIdx.x, lds);
}

// The three products of the gradient that need dg and du (and a), in one launch:
// blocks up to dx's, those of w_in's gradient, and the rest.
struct LastArgs {
  ProductArgs dx, in, out;
  uint32_t dx_blocks, in_blocks;
};
template <class T, bool kMapped, bool kFast, class Z>
__global__ __launch_bounds__(Z::kThreads, Z::BM == 64 ? 4 : 2) void ffn_last_kernel(LastArgs g) {
  extern __shared__ __align__(16) char lds[];
  uint32_t b = blockIdx.x;
  if (b < g.dx_blocks) return product<T, kDx, false, kFast, Z>(g.dx, b, lds);
  b -= g.dx_blocks;
  if (b < g.in_blocks) return product<T, kDwIn, kMapped, kFast, Z>(g.in, b, lds);
  product<T, kDwOut, kMapped, kFast, Z>(g.out, b - g.in_blocks, lds);
}

// What a launch needs to know of a kernel
struct Kernel {
  const void *fn;
  int rows, cols, threads, lds;
  int held() const { return cols == 256 ? 1 : rows == 64 ? 4 : 2; }  // blocks of a CU
};
template <class Z>
Kernel shaped(const void *fn) {
  return {fn, Z::BM, Z::BN, Z::kThreads, Z::kLds};
}
template <class T, int kKind, bool kMapped, bool kFast>
Kernel kernel_of(Size size) {
#define F(Z) shaped<Z>((const void *)ffn_product_kernel<T, kKind, kMapped, kFast, Z>)
  if constexpr (kKind == kDwOut || kKind == kDwIn) {  // smaller ones: ffn_last_kernel
    if constexpr (kFast && sizeof(T) == 2) {
      if constexpr (kMapped) return size == kWide ? F(MappedWide) : F(MappedLarge);
      else return size == kWide ? F(Wide) : F(Large);
    }
  } else {
    if constexpr (kFast && sizeof(T) == 2) {
      if (size == kWide) return F(Wide);
      if (size == kLarge) return F(Large);
    }
    return size == kTiny ? F(Tiny) : size == kSmall ? F(Small) : F(Medium);
  }
#undef F
}
template <class T, int kKind>
Kernel kernel_of(bool mapped, bool fast, Size size) {
  if constexpr (kKind == kDwOut || kKind == kDwIn)  // the others' rows are fixed before the steps
    return mapped ? kernel_of<T, kKind, true, true>(size) : kernel_of<T, kKind, false, true>(size);
  else
    return fast ? kernel_of<T, kKind, false, true>(size) : kernel_of<T, kKind, false, false>(size);
}
template <int kKind>
Kernel kernel_of(int dtype, bool mapped, bool fast, Size size) {
  if constexpr (kKind != kDwOut && kKind != kDwIn)
    if (dtype == TACCL_F32) return kernel_of<float, kKind>(mapped, fast, size);
  return dtype == TACCL_BF16 ? kernel_of<bf16_t, kKind>(mapped, fast, size)
                             : kernel_of<f16_t, kKind>(mapped, fast, size);
}
template <class T, bool kMapped, bool kFast>
Kernel last_kernel(Size size) {
#define F(Z) shaped<Z>((const void *)ffn_last_kernel<T, kMapped, kFast, Z>)
  return size == kSmall ? F(Small) : F(Medium);
#undef F
}
template <class T>
Kernel last_kernel(bool mapped, bool fast, Size size) {
  return mapped ? (fast ? last_kernel<T, true, true>(size) : last_kernel<T, true, false>(size))
                : (fast ? last_kernel<T, false, true>(size) : last_kernel<T, false, false>(size));
}

template <class... P>
bool aligned16(P... p) {
  return (((uintptr_t)p % 16 == 0) && ...);
}

// Time of a step of 128 bytes by tile size: a CU holds `held` blocks, which take
// `full` microseconds a step each, and `alone` if there is only one. Measured: f16
// and bf16 with all CUs busy, on the up projection of 64 x 980 rows of 4096, hidden
// 1536 (1434, 1571, 1773 and 2784 us from Large to Small), single blocks on 4 x 196
// rows; in 32 bits the matrix instructions' time.
struct Pace {
  Size size;
  int rows, cols, held;
  double full, alone;
};
constexpr Pace kPaces16[] = {{kLarge, 256, 256, 1, 1.75, 1.75},
                             {kWide, 128, 256, 1, 1.15, 1.1},
                             {kMedium, 128, 128, 2, 1.3, 0.8},
                             {kSmall, 64, 64, 4, 0.95, 0.5},
                             {kTiny, 32, 64, 2, 0.45, 0.45}};
constexpr Pace kPaces32[] = {{kMedium, 128, 128, 2, 3.4, 1.8},
                             {kSmall, 64, 64, 4, 1.8, 0.6},
                             {kTiny, 32, 64, 2, 0.6, 0.4}};

// What the launches of a call share
struct Products {
  ProductArgs base{};
  const FfnTile *tiles[kLists];
  int32_t *done;
  float *partial;
  int64_t partial_bytes;
  bool fast;
  int dtype, cus;
  int64_t slots;
  hipStream_t stream;

  int64_t count(int64_t m, int64_t n, int rows, int cols) const {
    return base.experts * ((m + rows - 1) / rows) * ((n + cols - 1) / cols);
  }
  // Size of the tiles of a product of m rows and n columns per expert: the one
  // whose steps take the least time
  Size size_of(int64_t m, int64_t n) const {
    Size best = kMedium;
    double least = 1e300;
    auto consider = [&](const Pace &c) {
      if (!fast && c.size >= kWide) return;
      const double turns = (double)count(m, n, c.rows, c.cols) / (c.held * cus);
      const double t = std::max(c.alone, turns * c.full);
      if (t < least) {
        least = t;
        best = c.size;
      }
    };
    if (dtype == TACCL_F32)
      for (const Pace &c : kPaces32) consider(c);
    else
      for (const Pace &c : kPaces16) consider(c);
    return best;
  }

  // the list that a product's kernel reads, as a bit
  template <int kKind>
  int list(int64_t m, int64_t n) const {
    const Kernel k = kernel_of<kKind>(dtype, base.map != nullptr, fast, size_of(m, n));
    return 1 << list_of(k.rows);
  }
  // arguments of product `number` of a call with this kernel's tiles, over a
  // shared axis of K, and its blocks; `used` bytes of the partial sums are taken
  ProductArgs args(const Kernel &k, int number, const void *a, const void *b, void *out, int64_t m,
                   int64_t n, int64_t K, uint32_t &blocks, int64_t &used) const {
    ProductArgs g = base;
    g.a = a;
    g.b = b;
    g.out = out;
    g.tiles = tiles[list_of(k.rows)];
    g.num_tiles += list_of(k.rows);
    g.col_tiles = (int)((n + k.cols - 1) / k.cols);
    g.row_tiles = (int)((m + k.rows - 1) / k.rows);
    // Few tiles share their steps among parts, as many as CUs hold at two blocks
    // each (one of the largest tiles), of at least eight steps (2 x 340 rows of 4587
    // f32, hidden 32: 64 us a call without, 27 with). More sums than 4096
    // bytes a row cost more than they save (gradient of 4 x 1000 rows of 2048 bf16,
    // hidden 1024: 138 us, with 8192 142).
    const int64_t count = (int64_t)g.experts * g.row_tiles * g.col_tiles;
    const int64_t step = dtype == TACCL_F32 ? 32 : 64, size = (int64_t)k.rows * k.cols * 4;
    const int64_t sums = std::min(partial_bytes, (3 << 18) + 4096 * base.experts * slots);
    int64_t parts = 1;
    if (count <= kSplitTiles)
      parts = std::max<int64_t>(
          1, std::min({std::min(2, k.held()) * (int64_t)cus / count, K / (8 * step), (int64_t)16,
                       (sums - used) / (count * size)}));
    g.parts = (int)parts;
    g.done = done + number * kSplitTiles;
    g.partial = partial + used / 4;
    if (parts > 1) used += count * parts * size;
    // ids come in pieces of 32 by 8 XCDs
    blocks = out ? (uint32_t)((count * parts + 255) / 256 * 256) : 0;
    return g;
  }
  // a product of m rows and n columns per expert, alone in a launch
  template <int kKind>
  hipError_t run(int number, const void *a, const void *b, void *out, int64_t m, int64_t n,
                 int64_t K, void *more = nullptr, const void *pre = nullptr) const {
    const Kernel k = kernel_of<kKind>(dtype, base.map != nullptr, fast, size_of(m, n));
    uint32_t blocks;
    int64_t used = 0;
    ProductArgs g = args(k, number, a, b, out, m, n, K, blocks, used);
    // The tiles of rows that exist may leave most of the chip without one in their
    // last turn, which only the device knows: up to four blocks share such a tile,
    // of at least eight steps each, one block per CU in all (us a call without and
    // so: 8 x 600 rows of 2048 f32, hidden 1024 654 and 556, 570 with two blocks per
    // CU; 8 x 200 of 4096 bf16, hidden 1536, room for 1024 165 and 144; gradient of
    // 6 x 700 of 2048 bf16, hidden 1408 277 and 253). Adding up the parts takes as
    // long as about eight steps: axes of less than 24 are not shared (gradient of 4
    // x 1000 of 2048 bf16, hidden 1024 132, shared 138). Through registers parts have
    // sixteen (20 x 500 rows of 2047 f16, hidden 1023 247, with eight 263).
    const int64_t steps = K / (dtype == TACCL_F32 ? 32 : 64), round = (int64_t)cus * k.held();
    const int64_t last_parts =
        steps < 24 ? 1 : std::min<int64_t>(steps / (fast ? 8 : 16), 4);
    if (g.parts == 1 && last_parts > 1 && round <= kSplitTiles && round % 256 == 0) {
      g.round = (uint32_t)round;
      g.last_parts = (uint32_t)last_parts;
      g.room = (uint32_t)std::min<int64_t>(cus, partial_bytes / ((int64_t)k.rows * k.cols * 4));
      blocks = (uint32_t)((blocks + round - 1) / round * round);
    }
    g.more = more;
    g.pre = pre;
    void *p[] = {&g};
    if (!out) return hipSuccess;
    return hipLaunchKernel(k.fn, dim3(blocks), dim3(k.threads), p, k.lds, stream);
  }
};

template <class A>
Products products(const A &a, const FfnSpace &sp, bool fast, int cus, hipStream_t stream) {
  uint8_t *ws = (uint8_t *)a.workspace;
  Products p;
  p.dtype = a.dtype;
  p.fast = fast;
  p.cus = cus;
  p.slots = a.sources * a.capacity;
  p.stream = stream;
  ProductArgs &g = p.base;
  g.rows = (const int32_t *)(ws + sp.rows);
  g.num_tiles = (const int32_t *)(ws + sp.num_tiles);
  g.map = a.sources > 1 ? (const int32_t *)(ws + sp.map) : nullptr;
  g.slots = p.slots;
  g.cols = a.cols;
  g.hidden = a.hidden;
  g.experts = a.num_experts;
  for (int i = 0; i < kLists; i++) p.tiles[i] = (const FfnTile *)(ws + sp.tiles[i]);
  p.done = (int32_t *)(ws + sp.done);
  p.partial = (float *)(ws + sp.partial);
  p.partial_bytes = std::min(a.workspace_bytes, sp.bytes) - sp.partial;
  return p;
}

// The first launch, for products with tiles of the lists `lists`
template <class A>
hipError_t launch_plan(const A &a, const Products &p, int lists, void *zero) {
  PlanArgs q{};
  q.counts = a.counts;
  q.capacity = a.capacity;
  q.sources = a.sources;
  q.experts = a.num_experts;
  q.rows = (int32_t *)p.base.rows;
  q.num_tiles = (int32_t *)p.base.num_tiles;
  q.map = (int32_t *)p.base.map;
  for (int i = 0; i < kLists; i++) q.tiles[i] = (FfnTile *)p.tiles[i];
  q.lists = lists;
  q.done = p.done;
  q.zero = (uint8_t *)zero;
  q.row_bytes = a.cols * (a.dtype == TACCL_F32 ? 4 : 2);
  // four blocks per CU, in whole ones per piece
  auto parts = [&](int64_t pieces, int64_t most) {
    return (int)std::max<int64_t>(1, std::min(most, (4 * p.cus + pieces - 1) / pieces));
  };
  const int64_t pieces = (int64_t)q.sources * q.experts;
  if (q.map) q.map_parts = parts(q.experts, (p.slots + kPlanThreads - 1) / kPlanThreads);
  if (zero) q.zero_parts = parts(pieces, q.capacity);
  const int64_t blocks = 1 + (int64_t)q.experts * q.map_parts + pieces * q.zero_parts;
  void *args[] = {&q};
  return hipLaunchKernel((const void *)ffn_plan_kernel, dim3((uint32_t)blocks), dim3(kPlanThreads),
                         args, 0, p.stream);
}

// whole, aligned chunks everywhere
bool whole_chunks(int dtype, int cols, int hidden) {
  const int n = dtype == TACCL_F32 ? 4 : 8;
  return cols % n == 0 && hidden % n == 0;
}

}  // namespace

hipError_t launch_ffn(const taccl_ffn_t &a, int cus, hipStream_t stream) {
  const FfnSpace sp =
      ffn_space(a.sources, a.num_experts, a.capacity, a.hidden, a.dtype, false);
  const bool fast = whole_chunks(a.dtype, a.cols, a.hidden) &&
                    aligned16(a.buffer, a.w_in, a.w_out, a.out, a.pre);
  const Products p = products(a, sp, fast, cus, stream);
  void *act = (uint8_t *)a.workspace + sp.act;
  const int64_t D = a.cols, F = a.hidden;
  hipError_t e = launch_plan(a, p, p.list<kUp>(p.slots, 2 * F) | p.list<kDown>(p.slots, D), a.out);
  if (e == hipSuccess) e = p.run<kUp>(0, a.buffer, a.w_in, act, p.slots, 2 * F, D, a.pre);
  if (e == hipSuccess) e = p.run<kDown>(1, act, a.w_out, a.out, p.slots, D, F);
  return e;
}

hipError_t launch_ffn_backward(const taccl_ffn_backward_t &a, int cus, hipStream_t stream) {
  const FfnSpace sp = ffn_space(a.sources, a.num_experts, a.capacity, a.hidden, a.dtype, true);
  const bool fast =
      whole_chunks(a.dtype, a.cols, a.hidden) &&
      aligned16(a.dout, a.buffer, a.w_in, a.w_out, a.pre, a.dbuffer, a.dw_in, a.dw_out);
  const Products p = products(a, sp, fast, cus, stream);
  void *act = (uint8_t *)a.workspace + sp.act, *dpre = (uint8_t *)a.workspace + sp.dpre;
  const int64_t D = a.cols, F = a.hidden;
  const bool mapped = p.base.map != nullptr;
  // Large products one by one, small ones together: alone they leave CUs empty.
  const bool each = fast && a.dtype != TACCL_F32 &&
                    std::min({p.size_of(p.slots, D), p.size_of(2 * F, D), p.size_of(D, F)}) >= kWide;
  // the longest tile alone, or all of them at full CUs
  auto time = [&](Size of) {
    const Pace *c = a.dtype == TACCL_F32 ? kPaces32 : kPaces16;
    while (c->size != of) c++;
    const double step = a.dtype == TACCL_F32 ? 32 : 64, by_f = 2 * F / step, by_rows = p.slots / step;
    const double all = p.count(p.slots, D, c->rows, c->cols) * by_f +
                       (p.count(2 * F, D, c->rows, c->cols) + p.count(D, F, c->rows, c->cols)) *
                           by_rows;
    return std::max(c->alone * std::max(by_f, by_rows), all * c->full / (c->held * cus));
  };
  const Size size = time(kMedium) < time(kSmall) ? kMedium : kSmall;
  const Kernel k = a.dtype == TACCL_F32    ? last_kernel<float>(mapped, fast, size)
                   : a.dtype == TACCL_BF16 ? last_kernel<bf16_t>(mapped, fast, size)
                                           : last_kernel<f16_t>(mapped, fast, size);
  hipError_t e = launch_plan(a, p,
                             p.list<kGrad>(p.slots, F) |
                                 (each ? p.list<kDx>(p.slots, D) : 1 << list_of(k.rows)),
                             a.dbuffer);
  if (e == hipSuccess) e = p.run<kGrad>(0, a.dout, a.w_out, dpre, p.slots, F, D, act, a.pre);
  if (e != hipSuccess) return e;
  if (each) {
    e = p.run<kDx>(1, dpre, a.w_in, a.dbuffer, p.slots, D, 2 * F);
    if (e == hipSuccess) e = p.run<kDwIn>(2, dpre, a.buffer, a.dw_in, 2 * F, D, p.slots);
    if (e == hipSuccess) e = p.run<kDwOut>(3, a.dout, act, a.dw_out, D, F, p.slots);
    return e;
  }
  LastArgs g{};
  uint32_t out_blocks;
  int64_t used = 0;
  g.out = p.args(k, 3, a.dout, act, a.dw_out, D, F, p.slots, out_blocks, used);
  g.in = p.args(k, 2, dpre, a.buffer, a.dw_in, 2 * F, D, p.slots, g.in_blocks, used);
  g.dx = p.args(k, 1, dpre, a.w_in, a.dbuffer, p.slots, D, 2 * F, g.dx_blocks, used);
  void *args[] = {&g};
  return hipLaunchKernel(k.fn, dim3(g.dx_blocks + g.in_blocks + out_blocks), dim3(k.threads), args,
                         k.lds, stream);
}

}  // namespace taccl
