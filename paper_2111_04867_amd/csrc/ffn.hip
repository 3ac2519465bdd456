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
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ffn.h"
#include "tile.h"

namespace taccl {

namespace {

struct FfnTile {
  int32_t expert, row;
};

constexpr int kPlanThreads = 256;

int64_t rounded(int64_t n) { return (n + 255) / 256 * 256; }

constexpr int kMinTile = 64;  // rows of the smallest tile, for the list's length

}  // namespace

FfnSpace ffn_space(int64_t sources, int64_t experts, int64_t capacity, int64_t hidden, int dtype,
                   bool backward) {
  const int64_t slots = sources * capacity, rows = experts * slots;
  const int64_t size = dtype == TACCL_F32 ? 4 : 2;
  FfnSpace s{};
  s.num_tiles = rounded(4 * experts);
  s.tiles = s.num_tiles + 256;
  s.map = s.tiles + rounded(8 * experts * ((slots + kMinTile - 1) / kMinTile));
  s.act = s.map + (sources > 1 ? rounded(4 * rows) : 0);
  s.dpre = s.act + rounded(rows * hidden * size);
  s.bytes = s.dpre + (backward ? rounded(2 * rows * hidden * size) : 0);
  return s;
}

namespace {

struct PlanArgs {
  const int32_t *counts;  // [S][E]
  int64_t capacity;
  int32_t sources, experts, tile, parts;
  int32_t *rows, *num_tiles, *map;  // map: or null
  FfnTile *tiles;
  uint8_t *zero;  // rows past the counts are zeroed; or null
  int64_t row_bytes;
};

__device__ __forceinline__ int64_t rows_of(const PlanArgs &g, int s, int e) {
  return min((int64_t)max(g.counts[(int64_t)s * g.experts + e], 0), g.capacity);
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

// Block 0 counts and lists, the others number and zero the rows of an expert.
__global__ __launch_bounds__(kPlanThreads) void ffn_plan_kernel(PlanArgs g) {
  __shared__ uint32_t red[kPlanThreads / 64];
  if (blockIdx.x == 0) {
    uint32_t first = 0;
    for (int e0 = 0; e0 < g.experts; e0 += kPlanThreads) {
      const int e = e0 + threadIdx.x;
      int64_t n = 0;
      if (e < g.experts) {
        for (int s = 0; s < g.sources; s++) n += rows_of(g, s, e);
        g.rows[e] = (int32_t)n;
      }
      const uint32_t mine = (uint32_t)((n + g.tile - 1) / g.tile);
      uint32_t all;
      const uint32_t at = first + block_scan(mine, red, all) - mine;
      for (uint32_t i = 0; i < mine; i++)
        g.tiles[at + i] = FfnTile{e, (int32_t)(i * (uint32_t)g.tile)};
      first += all;
    }
    if (threadIdx.x == 0) *g.num_tiles = (int32_t)first;
    return;
  }
  const int b = blockIdx.x - 1, e = b % g.experts, part = b / g.experts;
  const int64_t slots = g.sources * g.capacity;
  if (g.map) {
    int32_t *map = g.map + e * slots;
    uint32_t first = 0;
    for (int s0 = 0; s0 < g.sources; s0 += kPlanThreads) {
      const int s = s0 + threadIdx.x;
      const uint32_t n = s < g.sources ? (uint32_t)rows_of(g, s, e) : 0;
      uint32_t all;
      const uint32_t at = first + block_scan(n, red, all) - n;
      // each source's rows by the whole block, one source after the other
      __shared__ uint32_t from[kPlanThreads], len[kPlanThreads];
      from[threadIdx.x] = at;
      len[threadIdx.x] = n;
      __syncthreads();
      for (int i = 0; i < min(kPlanThreads, g.sources - s0); i++) {
        const int64_t row = ((int64_t)(s0 + i) * g.experts + e) * g.capacity;
        for (uint32_t j = part * kPlanThreads + threadIdx.x; j < len[i];
             j += g.parts * kPlanThreads)
          map[from[i] + j] = (int32_t)(row + j);
      }
      first += all;
    }
  }
  if (g.zero) {
    for (int s = 0; s < g.sources; s++) {
      const int64_t n = rows_of(g, s, e), row = ((int64_t)s * g.experts + e) * g.capacity + n;
      zero_piece<kPlanThreads>(g.zero + row * g.row_bytes, (g.capacity - n) * g.row_bytes, part,
                               g.parts);
    }
  }
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
};

template <class T>
__device__ __forceinline__ float sigmoid(float g) {
  if constexpr (sizeof(T) == 4) return 1.0f / (1.0f + expf(-g));
  // within a few units in the last place of 32 bits for the g of a size that
  // 16 bits show; 0 for an infinite exponential
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
}

// Four results of a row; `left` columns of it exist
template <class T, bool kFast>
__device__ __forceinline__ void store_four(T *p, F4 v, int left) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  if (kFast) {
    if (left > 0) *(T4 *)p = T4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < left) p[i] = (T)v[i];
  }
}
template <class T, bool kFast>
__device__ __forceinline__ F4 load_four(const T *p, int left) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  F4 v = {0, 0, 0, 0};
  if (kFast) {
    if (left > 0) {
      const T4 t = *(const T4 *)p;
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] = (float)t[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < left) v[i] = (float)p[i];
  }
  return v;
}

// A tile of BM rows by BN columns; WM x WN wavefronts.
template <class T, int kKind, bool kFast, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void ffn_product_kernel(ProductArgs g) {
  constexpr bool kWeights = kKind == kDwOut || kKind == kDwIn;
  constexpr bool kAcrossA = kWeights, kAcrossB = kKind != kUp && kKind != kDown;
  constexpr int kThreads = 64 * WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
  constexpr int kBuffer = (BM + BN) * kStepBytes;
  extern __shared__ __align__(16) char lds[];
  const int D = g.cols, F = g.hidden;

  // Blocks go to the XCDs in turn; 32 consecutive ones of an XCD take a piece
  // of 8 tiles of columns by 4 of rows, whose operands its L2 holds.
  const uint32_t b = blockIdx.x, per_xcd = b >> 3;
  const uint32_t id = ((per_xcd >> 5) * 8 + (b & 7)) * 32 + (per_xcd & 31);
  const uint32_t entries = kWeights ? (uint32_t)(g.experts * g.row_tiles) : (uint32_t)*g.num_tiles;
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
  oa.ld = lda;
  oa.map = kBufferA ? map : nullptr;
  const int ldb = kKind == kUp || kKind == kDx || kKind == kDwIn ? D : F;
  if (kWeights) ob.p = (const T *)g.b + (kKind == kDwIn && map ? 0 : first * ldb);
  else ob.p = (const T *)g.b + (int64_t)e * D * F * (kKind == kUp || kKind == kDx ? 2 : 1);
  ob.ld = ldb;
  ob.map = kKind == kDwIn ? map : nullptr;
  const int K = kWeights ? n : kKind == kDown ? F : kKind == kDx ? 2 * F : D;
  // columns of the product; the up projection's tile has gate and up columns,
  // half each, of as many hidden ones
  constexpr int kCols = kKind == kUp ? BN / 2 : BN;
  const int N = kKind == kUp || kKind == kGrad || kKind == kDwOut ? F : D;
  const int M = kKind == kDwOut ? D : kKind == kDwIn ? 2 * F : n;
  const int n0 = tn * kCols;

  Loader<T, kAcrossA, kFast, BM, kThreads> la;
  Loader<T, kAcrossB, kFast, BN, kThreads> lb;
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

  const int steps = (K + kStepK<T> - 1) / kStepK<T>;
  if (steps > 0) {
    la.load(0, lds);
    lb.load(0, lds + BM * kStepBytes);
    la.store(lds);
    lb.store(lds + BM * kStepBytes);
  }
  for (int s = 0; s < steps; s++) {
    char *now = lds + (s & 1) * kBuffer, *next = lds + (~s & 1) * kBuffer;
    tile_barrier();
    if (s + 1 < steps) {
      la.load((s + 1) * kStepK<T>, next);
      lb.load((s + 1) * kStepK<T>, next + BM * kStepBytes);
    }
#pragma unroll
    for (int h = 0; h < 2; h++) {
      Frag<T> fa[MI], fb[NI];
#pragma unroll
      for (int i = 0; i < MI; i++) fa[i] = read_frag<T, kAcrossA, BM>(now, wm + 16 * i, h);
#pragma unroll
      for (int j = 0; j < NI; j++)
        fb[j] = read_frag<T, kAcrossB, BN>(now + BM * kStepBytes, wn + 16 * j, h);
#pragma unroll
      for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NI; j++) acc[i][j] = multiply(fb[j], fa[i], acc[i][j]);
    }
    if (s + 1 < steps) {
      la.store(next);
      lb.store(next + BM * kStepBytes);
    }
  }

  // Lane l has columns l / 16 * 4 + 0..3 of row l % 16 of every 16 x 16 part.
#pragma unroll
  for (int i = 0; i < MI; i++) {
    const int m = t.row + wm + 16 * i + (lane & 15);
    if (m >= M) continue;
    const int64_t compact = first + m, row = kWeights ? 0 : map ? map[m] : compact;
    const int c0 = lane >> 4 << 2;
    if constexpr (kKind == kUp) {
#pragma unroll
      for (int j = 0; j < NI / 2; j++) {
        const int f = n0 + wn / 2 + 16 * j + c0, left = F - f;
        const F4 gate = acc[i][j], up = acc[i][j + NI / 2];
        F4 a;
#pragma unroll
        for (int x = 0; x < 4; x++) a[x] = gate[x] * sigmoid<T>(gate[x]) * up[x];
        store_four<T, kFast>((T *)g.out + compact * F + f, a, left);
        if (g.more) {
          T *pre = (T *)g.more + row * 2 * F + f;
          store_four<T, kFast>(pre, gate, left);
          store_four<T, kFast>(pre + F, up, left);
        }
      }
    } else if constexpr (kKind == kGrad) {
#pragma unroll
      for (int j = 0; j < NI; j++) {
        const int f = n0 + wn + 16 * j + c0, left = F - f;
        const T *pre = (const T *)g.pre + row * 2 * F + f;
        const F4 gate = load_four<T, kFast>(pre, left), up = load_four<T, kFast>(pre + F, left);
        F4 a, dg, du;
#pragma unroll
        for (int x = 0; x < 4; x++) {
          const float sg = sigmoid<T>(gate[x]), da = acc[i][j][x], act = gate[x] * sg;
          a[x] = act * up[x];
          du[x] = da * act;
          dg[x] = da * up[x] * (sg * (1.0f + gate[x] * (1.0f - sg)));
        }
        T *dpre = (T *)g.out + compact * 2 * F + f;
        store_four<T, kFast>(dpre, dg, left);
        store_four<T, kFast>(dpre + F, du, left);
        store_four<T, kFast>((T *)g.more + compact * F + f, a, left);
      }
    } else {
      const int64_t to = kKind == kDwOut ? (int64_t)e * D + m : kKind == kDwIn ? (int64_t)e * 2 * F + m : row;
#pragma unroll
      for (int j = 0; j < NI; j++) {
        const int c = n0 + wn + 16 * j + c0;
        store_four<T, kFast>((T *)g.out + to * N + c, acc[i][j], N - c);
      }
    }
  }
}

// a tile's shape
struct Shape {
  int rows, cols, threads;
};
constexpr Shape kLarge{256, 256, 512}, kSmall{128, 128, 256};

template <class T, int kKind, bool kFast>
const void *product_fn(bool large) {
  if constexpr (kFast && sizeof(T) == 2)
    if (large) return (const void *)ffn_product_kernel<T, kKind, kFast, 256, 256, 2, 4>;
  return (const void *)ffn_product_kernel<T, kKind, kFast, 128, 128, 2, 2>;
}
template <int kKind>
const void *product_of(int dtype, bool fast, bool large) {
#define F(T) (fast ? product_fn<T, kKind, true>(large) : product_fn<T, kKind, false>(large))
  return dtype == TACCL_F32 ? F(float) : dtype == TACCL_BF16 ? F(bf16_t) : F(f16_t);
#undef F
}

template <class... P>
bool aligned16(P... p) {
  return (((uintptr_t)p % 16 == 0) && ...);
}

// What the launches of a call share
struct Products {
  ProductArgs base{};
  Shape shape;
  bool fast, large;
  int dtype;
  int64_t slots;
  hipStream_t stream;

  // kKind's launch; `m`: rows of the weights' gradient, else 0; n: columns
  template <int kKind>
  hipError_t run(const void *a, const void *b, void *out, int m, int n, void *more = nullptr,
                 const void *pre = nullptr) const {
    ProductArgs g = base;
    g.a = a;
    g.b = b;
    g.out = out;
    g.more = more;
    g.pre = pre;
    const int per = kKind == kUp ? shape.cols / 2 : shape.cols;
    g.col_tiles = (n + per - 1) / per;
    g.row_tiles = (m + shape.rows - 1) / shape.rows;
    const int64_t entries = g.experts * (m ? g.row_tiles : (slots + shape.rows - 1) / shape.rows);
    // ids come in pieces of 32 by 8 XCDs
    const int64_t blocks = (entries * g.col_tiles + 255) / 256 * 256;
    const uint32_t bytes = 2 * (shape.rows + shape.cols) * kStepBytes;
    void *args[] = {&g};
    return hipLaunchKernel(product_of<kKind>(dtype, fast, large), dim3((uint32_t)blocks),
                           dim3(shape.threads), args, bytes, stream);
  }
};

template <class A>
hipError_t prepare(const A &a, const FfnSpace &sp, bool fast, int cus, void *zero,
                   hipStream_t stream, Products &p) {
  uint8_t *ws = (uint8_t *)a.workspace;
  const int64_t size = a.dtype == TACCL_F32 ? 4 : 2;
  p.dtype = a.dtype;
  p.fast = fast;
  p.slots = a.sources * a.capacity;
  p.stream = stream;
  // the large tile where it leaves every CU two tiles of the smaller product
  const int64_t tiles = a.num_experts * ((p.slots + 255) / 256) *
                        ((std::min(a.cols, 2 * a.hidden) + 255) / 256);
  p.large = fast && size == 2 && tiles >= 2 * cus;
  p.shape = p.large ? kLarge : kSmall;
  ProductArgs &g = p.base;
  g.rows = (const int32_t *)(ws + sp.rows);
  g.num_tiles = (const int32_t *)(ws + sp.num_tiles);
  g.tiles = (const FfnTile *)(ws + sp.tiles);
  g.map = a.sources > 1 ? (const int32_t *)(ws + sp.map) : nullptr;
  g.slots = p.slots;
  g.cols = a.cols;
  g.hidden = a.hidden;
  g.experts = a.num_experts;
  PlanArgs q{};
  q.counts = a.counts;
  q.capacity = a.capacity;
  q.sources = a.sources;
  q.experts = a.num_experts;
  q.tile = p.shape.rows;
  q.parts = zero || g.map ? (int)std::max<int64_t>(1, std::min<int64_t>(
                                p.slots, (4 * (int64_t)cus + q.experts - 1) / q.experts))
                          : 0;
  q.rows = (int32_t *)(ws + sp.rows);
  q.num_tiles = (int32_t *)(ws + sp.num_tiles);
  q.map = (int32_t *)g.map;
  q.tiles = (FfnTile *)(ws + sp.tiles);
  q.zero = (uint8_t *)zero;
  q.row_bytes = a.cols * size;
  void *args[] = {&q};
  return hipLaunchKernel((const void *)ffn_plan_kernel,
                         dim3(1 + (uint32_t)q.experts * (uint32_t)q.parts), dim3(kPlanThreads),
                         args, 0, stream);
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
  Products p;
  hipError_t e = prepare(a, sp, fast, cus, a.out, stream, p);
  void *act = (uint8_t *)a.workspace + sp.act;
  if (e == hipSuccess) e = p.run<kUp>(a.buffer, a.w_in, act, 0, a.hidden, a.pre);
  if (e == hipSuccess) e = p.run<kDown>(act, a.w_out, a.out, 0, a.cols);
  return e;
}

hipError_t launch_ffn_backward(const taccl_ffn_backward_t &a, int cus, hipStream_t stream) {
  const FfnSpace sp = ffn_space(a.sources, a.num_experts, a.capacity, a.hidden, a.dtype, true);
  const bool fast =
      whole_chunks(a.dtype, a.cols, a.hidden) &&
      aligned16(a.dout, a.buffer, a.w_in, a.w_out, a.pre, a.dbuffer, a.dw_in, a.dw_out);
  Products p;
  hipError_t e = prepare(a, sp, fast, cus, a.dbuffer, stream, p);
  void *act = (uint8_t *)a.workspace + sp.act, *dpre = (uint8_t *)a.workspace + sp.dpre;
  if (e == hipSuccess) e = p.run<kGrad>(a.dout, a.w_out, dpre, 0, a.hidden, act, a.pre);
  if (e == hipSuccess && a.dbuffer) e = p.run<kDx>(dpre, a.w_in, a.dbuffer, 0, a.cols);
  if (e == hipSuccess && a.dw_out) e = p.run<kDwOut>(a.dout, act, a.dw_out, a.cols, a.hidden);
  if (e == hipSuccess && a.dw_in) e = p.run<kDwIn>(dpre, a.buffer, a.dw_in, 2 * a.hidden, a.cols);
  return e;
}

}  // namespace taccl
