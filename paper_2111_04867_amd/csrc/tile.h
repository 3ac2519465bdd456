// Matrix products on tiles in LDS for the experts' feed-forward (gfx950).
//
// A block multiplies BM rows of one operand by BN rows of the other over steps
// of 128 bytes of the shared axis (kStepK elements). Either operand is stored
// with the shared axis contiguous ("along") or as rows of it ("across"); its
// tile lies in LDS the way it is stored, in 16-byte chunks whose order within a
// row is permuted so that the reads of a matrix instruction's operand touch
// every bank equally often. Loads go straight to LDS where every chunk is
// aligned and whole (kFast), else through registers.
#pragma once

#include <hip/hip_runtime.h>

#include "elem.h"

namespace taccl {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));

// what lanes past the shared axis' end load; never written
static __device__ Chunk zero_chunk;

__device__ __forceinline__ void load_to_lds(const void *p, void *lds) {
  __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)p,
                                   (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}
// all of the block's loads to LDS are there, and all its reads of LDS are done
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One operand's part of a step: 16 rows by 64 bytes of the shared axis, a chunk
// per lane. Lane l holds row l % 16; the elements of the shared axis are dealt
// out to lane groups l / 16 alike for both operands.
template <class T>
struct Frag {
  typename Vec<T>::V v;
};
__device__ __forceinline__ F4 multiply(const Frag<bf16_t> &a, const Frag<bf16_t> &b, F4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ F4 multiply(const Frag<f16_t> &a, const Frag<f16_t> &b, F4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ F4 multiply(const Frag<float> &a, const Frag<float> &b, F4 c) {
#pragma unroll
  for (int i = 0; i < 4; i++)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
  return c;
}

// An operand in memory: `rows` rows (tile rows where the shared axis is along
// them, else rows of that axis), `ld` elements apart from `p`, or where `map`
// says.
template <class T>
struct Operand {
  const T *p;
  int64_t ld;
  const int32_t *map;  // row numbers, or null
  __device__ __forceinline__ const T *row(int64_t i) const {
    return p + (map ? (int64_t)map[i] : i) * ld;
  }
};

constexpr int kStepBytes = 128;
template <class T>
constexpr int kStepK = kStepBytes / (int)sizeof(T);

// The place of chunk `c` in row r of a tile across the shared axis, whose rows
// have kChunks chunks. A 16-bit operand is read 32 bytes (two chunks) from each
// of the rows 8 g + 0..3 (g < 4), a 32-bit one 64 bytes from each of 4 g + i.
template <class T, int kChunks>
__device__ __forceinline__ int across_place(int r, int c) {
  if (sizeof(T) == 2) return c ^ ((((r & 3) | (r >> 3 & 3) << 2) << 1) & (kChunks - 1));
  return c ^ (((r >> 2 & 3) << 2) & (kChunks - 1));
}

// The loads of an operand's tile of kRows rows (columns where the shared axis
// is across) by a block of kThreads threads.
template <class T, bool kAcross, bool kFast, int kRows, int kThreads>
struct Loader {
  static constexpr int kLoads = kRows * 8 / kThreads;
  static constexpr int kN = Vec<T>::kN;
  static constexpr int kChunks = kAcross ? kRows / kN : 8;  // per row in LDS
  static_assert(kRows * 8 % kThreads == 0);

  Operand<T> o;
  const T *at[kLoads];  // along: the row's next chunk
  int K;                // the shared axis' length
  int col, cols;        // across: the tile's first column and their number
  Chunk held[kFast ? 1 : kLoads];

  static __device__ __forceinline__ int chunk_id(int i) { return i * kThreads + threadIdx.x; }
  // row of load i in LDS and the chunk of the operand that belongs there
  static __device__ __forceinline__ int row(int i) { return chunk_id(i) / kChunks; }
  static __device__ __forceinline__ int source(int i) {
    const int c = chunk_id(i) % kChunks, r = row(i);
    return kAcross ? across_place<T, kChunks>(r, c) : c ^ (r & 7);
  }

  // tile row r is row `from(r)` of the operand
  template <class F>
  __device__ __forceinline__ void along(const Operand<T> &op, int k, F from) {
    o = op;
    K = k;
#pragma unroll
    for (int i = 0; i < kLoads; i++) at[i] = o.row(from(row(i))) + source(i) * kN;
  }
  // columns from `c` on, of n
  __device__ __forceinline__ void across(const Operand<T> &op, int k, int c, int n) {
    o = op;
    K = k;
    col = c;
    cols = n;
    if (!o.map) {
#pragma unroll
      for (int i = 0; i < kLoads; i++) at[i] = o.p + (int64_t)row(i) * o.ld + column(i);
    }
  }
  // a chunk past the last column takes the tile's first one: its results are
  // not stored
  __device__ __forceinline__ int column(int i) const {
    const int c = col + source(i) * kN;
    return c < cols ? c : col;
  }

  // Step k0 of the tile, to `lds` (kFast) or on its way to `held`.
  __device__ __forceinline__ void load(int k0, char *lds) {
    const bool last = k0 + kStepK<T> > K;
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
      const T *p;
      int left;  // elements of the chunk that exist
      if (kAcross) {
        const int r = k0 + row(i);
        if (o.map) {
          p = r < K ? o.row(r) + column(i) : nullptr;
        } else {
          p = at[i];
          at[i] += kStepK<T> * o.ld;
        }
        left = !last || r < K ? (kFast ? kN : min(cols - column(i), kN)) : 0;
      } else {
        p = at[i];
        at[i] += kStepK<T>;
        left = last ? K - k0 - source(i) * kN : kN;
      }
      if (kFast) {
        if (last && left <= 0) p = (const T *)&zero_chunk;
        load_to_lds(p, lds + (i * kThreads + (threadIdx.x & ~63)) * 16);
      } else {
        held[i] = __builtin_bit_cast(Chunk, load_vec<T, true>(p, left));
      }
    }
  }
  __device__ __forceinline__ void store(char *lds) const {
    if (kFast) return;
#pragma unroll
    for (int i = 0; i < kLoads; i++) *(Chunk *)(lds + chunk_id(i) * 16) = held[i];
  }
};

// Operand of rows r0..r0+15 of a tile, half `step` of its 128 bytes
template <class T, bool kAcross, int kRows>
__device__ __forceinline__ Frag<T> read_frag(const char *lds, int r0, int step) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  constexpr int kN = Vec<T>::kN, kChunks = kRows / kN;
  Frag<T> f;
  if constexpr (!kAcross) {
    const int row = r0 + r;
    f.v = *(const typename Vec<T>::V *)(lds + row * kStepBytes + ((step * 4 + g) ^ (row & 7)) * 16);
  } else if constexpr (sizeof(T) == 2) {
    // Two transposing reads: of the 16 lanes of a group lanes 4 j + i read 4
    // columns each of row j, and lane r gets column r of rows 0 to 3.
    typedef short S4 __attribute__((ext_vector_type(4)));
    S4 h[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int k = step * 32 + g * 8 + j * 4 + (r >> 2), c = r0 + (r & 3) * 4;
      const char *p = lds + k * (kRows * 2) + across_place<T, kChunks>(k, c >> 3) * 16 + (c & 7) * 2;
      h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)p);
    }
    typedef short S8 __attribute__((ext_vector_type(8)));
    f.v = __builtin_bit_cast(typename Vec<T>::V,
                             (S8)__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    const int c = r0 + r;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int k = step * 16 + g * 4 + i;
      f.v[i] = *(const float *)(lds + k * (kRows * 4) + across_place<T, kChunks>(k, c >> 2) * 16 +
                                (c & 3) * 4);
    }
  }
  return f;
}

// Rows r of zeros: pieces of memory dealt out to blocks of kThreads threads
template <int kThreads>
__device__ __forceinline__ void zero_piece(uint8_t *p, int64_t n, int part, int parts) {
  typedef Chunk ChunkU __attribute__((aligned(1)));
  int64_t i = (int64_t)part * kThreads + threadIdx.x;
  const int64_t step = (int64_t)parts * kThreads;
  if (n < 16) {
    if (i < n) p[i] = 0;
    return;
  }
  const Chunk zero = {0, 0, 0, 0};
  for (; i < n / 16; i += step) *(ChunkU *)(p + 16 * i) = zero;
  if (part == 0 && threadIdx.x == 0) *(ChunkU *)(p + n - 16) = zero;
}

}  // namespace taccl
