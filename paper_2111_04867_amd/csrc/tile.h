// Matrix products on tiles in LDS for the experts' feed-forward (gfx950).
//
// A block multiplies BM rows of one operand by BN rows of the other over steps
// of 128 bytes of the shared axis, a cache line of every row (steps of 64 bytes,
// twice as many on their way, were 5 to 25% slower). Either operand is stored with the
// shared axis contiguous ("along") or as rows of it ("across"); its tile lies
// in LDS the way it is stored, in 16-byte chunks whose order within a row is
// permuted so that the reads of a matrix instruction's operand touch every bank
// equally often (no conflict by the counters). Where every chunk is aligned and
// whole (kFast), loads go straight to LDS; else through registers.
#pragma once

#include <hip/hip_runtime.h>

#include "elem.h"

namespace taccl {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;

// what lanes past the shared axis' end load; never written
static __device__ Chunk zero_chunk;

// 16 bytes per lane from p to LDS, the wavefront's from `lds` on. As a builtin
// the compiler waits for all such loads before every transposing read, which
// it takes to read what they write; so it does not see them, and whoever reads
// their LDS waits for them itself (tile_barrier). There is no register that they
// write.
__device__ __forceinline__ void load_to_lds(const void *p, char *lds) {
  const uint32_t at = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds);
  // m0 is declared so that no move to it is carried past this one; that it is
  // not kept for the code behind, which the compiler warns of, is meant.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(p), "s"(at)
               : "memory", "m0");
#pragma clang diagnostic pop
}
// All but the newest kLater of the wavefront's loads are there and its reads of
// LDS are done, and the same holds for the block's other wavefronts.
template <int kLater>
__device__ __forceinline__ void tile_barrier() {
  static_assert(kLater < 64);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater) : "memory");
}

// Stores and loads that other XCDs' blocks see and have made: a block that has
// waited for its stores (vmcnt) and then counts itself as done, atomically, is
// read by the one that finds all counted. Fences in their place write back and
// drop a whole L2.
__device__ __forceinline__ void put(float *p, F4 v) {
#pragma unroll
  for (int i = 0; i < 4; i++)
    __hip_atomic_store(p + i, v[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ F4 get(const float *p) {
  F4 v;
#pragma unroll
  for (int i = 0; i < 4; i++)
    v[i] = __hip_atomic_load(p + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return v;
}
// The same for a tile: chunks of 64 lanes' 16 bytes, 1 KB apart, N of them on
// their way at once (4 bytes at a time, as atomics: 32 tiles of 128 x 256 in four
// parts each took 70 us longer). The compiler does not look into the assembly, so
// its wait states are placed here: 12 behind a matrix instruction whose results are
// put (put_ready, once for all of them) and 2 before a store's registers are
// written again.
__device__ __forceinline__ void put_ready() { asm volatile("s_nop 15" ::: "memory"); }
__device__ __forceinline__ void put_chunk(float *p, F4 v) {
  asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" : : "v"(p), "v"(v) : "memory");
}
template <int N>
__device__ __forceinline__ void get_chunks(F4 (&v)[N], const float *p) {
  static_assert(N == 2 || N == 4 || N == 16);
  if constexpr (N == 2) {
    asm volatile(
        "global_load_dwordx4 %0, %2, off sc1\n\t"
        "global_load_dwordx4 %1, %2, off offset:1024 sc1\n\t"
        "s_waitcnt vmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1])
        : "v"(p)
        : "memory");
  } else if constexpr (N == 4) {
    asm volatile(
        "global_load_dwordx4 %0, %4, off sc1\n\t"
        "global_load_dwordx4 %1, %4, off offset:1024 sc1\n\t"
        "global_load_dwordx4 %2, %4, off offset:2048 sc1\n\t"
        "global_load_dwordx4 %3, %4, off offset:3072 sc1\n\t"
        "s_waitcnt vmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
        : "v"(p)
        : "memory");
  } else {
    asm volatile(
        "global_load_dwordx4 %0, %16, off sc1\n\t"
        "global_load_dwordx4 %1, %16, off offset:1024 sc1\n\t"
        "global_load_dwordx4 %2, %16, off offset:2048 sc1\n\t"
        "global_load_dwordx4 %3, %16, off offset:3072 sc1\n\t"
        "global_load_dwordx4 %4, %17, off sc1\n\t"
        "global_load_dwordx4 %5, %17, off offset:1024 sc1\n\t"
        "global_load_dwordx4 %6, %17, off offset:2048 sc1\n\t"
        "global_load_dwordx4 %7, %17, off offset:3072 sc1\n\t"
        "global_load_dwordx4 %8, %18, off sc1\n\t"
        "global_load_dwordx4 %9, %18, off offset:1024 sc1\n\t"
        "global_load_dwordx4 %10, %18, off offset:2048 sc1\n\t"
        "global_load_dwordx4 %11, %18, off offset:3072 sc1\n\t"
        "global_load_dwordx4 %12, %19, off sc1\n\t"
        "global_load_dwordx4 %13, %19, off offset:1024 sc1\n\t"
        "global_load_dwordx4 %14, %19, off offset:2048 sc1\n\t"
        "global_load_dwordx4 %15, %19, off offset:3072 sc1\n\t"
        "s_waitcnt vmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]),
          "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7]), "=&v"(v[8]), "=&v"(v[9]),
          "=&v"(v[10]), "=&v"(v[11]), "=&v"(v[12]), "=&v"(v[13]), "=&v"(v[14]),
          "=&v"(v[15])
        : "v"(p), "v"(p + 1024), "v"(p + 2048), "v"(p + 3072)
        : "memory");
  }
}
// By all threads of a block behind their put()s: whether it is the last of
// `parts` blocks to come here. `word` lies in LDS.
__device__ __forceinline__ bool last_of(int32_t *done, int parts, int32_t *word) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    *word = __hip_atomic_fetch_add(done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return *word == parts - 1;
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

// An operand in memory: rows (tile rows where the shared axis is along them,
// else rows of that axis) `ld` elements apart from `p`, or where `map` says, of
// an array that ends before `end`.
template <class T>
struct Operand {
  const T *p, *end;
  int64_t ld;
  const int32_t *map;  // row numbers, or null
  __device__ __forceinline__ const T *row(int64_t i) const {
    return p + (map ? (int64_t)map[i] : i) * ld;
  }
};

// The place of chunk `c` in row r of a tile whose rows have kChunks chunks.
// Along: sixteen rows' chunks of one number are read at a time, eight of them
// in each pass over the banks. Across: a 16-bit operand is read 32 bytes (two
// chunks) from each of the rows 8 g + 0..3 (g < 4), a 32-bit one 64 bytes from
// each of 4 g + i.
template <class T, bool kAcross, int kChunks>
__device__ __forceinline__ int chunk_place(int r, int c) {
  if (!kAcross) return c ^ (r & 7);
  if (sizeof(T) == 2) return c ^ ((((r & 3) | (r >> 3 & 3) << 2) << 1) & (kChunks - 1));
  return c ^ (((r >> 2 & 3) << 2) & (kChunks - 1));
}

// The loads of an operand's tile of kRows rows (columns where the shared axis
// is across), by kThreads threads.
template <class T, bool kAcross, bool kMapped, bool kFast, int kRows, int kThreads>
struct Loader {
  static constexpr int kLoads = kRows * kStepBytes / 16 / kThreads;
  static constexpr int kN = Vec<T>::kN, kStep = kStepBytes / (int)sizeof(T);
  static constexpr int kChunks = kAcross ? kRows / kN : 8;  // per row in LDS
  static_assert(kRows * 8 % kThreads == 0 && (kChunks & (kChunks - 1)) == 0);

  Operand<T> o;
  const T *at[kLoads];  // the chunk of the first step
  int K;                // the shared axis' length
  int col, cols;        // across: the tile's first column and their number
  int32_t mapped[kMapped ? kLoads : 1];  // the rows of the next step to load

  static __device__ __forceinline__ int chunk_id(int i) { return i * kThreads + threadIdx.x; }
  // row of load i in LDS and the chunk of the operand that belongs there
  static __device__ __forceinline__ int row(int i) { return chunk_id(i) / kChunks; }
  static __device__ __forceinline__ int source(int i) {
    return chunk_place<T, kAcross, kChunks>(row(i), chunk_id(i) % kChunks);
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
#pragma unroll
    for (int i = 0; i < kLoads; i++)
      at[i] = o.p + (kMapped ? 0 : (int64_t)row(i) * o.ld) + column(i);
  }
  // a chunk past the last column takes the tile's first one: its results are
  // not stored
  __device__ __forceinline__ int column(int i) const {
    const int c = col + source(i) * kN;
    return c < cols ? c : col;
  }
  // The map's entries for the step from k0 on, a step before its loads need them
  // and ahead of those that are started between: loads arrive in order.
  __device__ __forceinline__ void look_up(int k0) {
    if (!kMapped) return;
#pragma unroll
    for (int i = 0; i < kLoads; i++) mapped[i] = o.map[max(min(k0 + row(i), K - 1), 0)];
  }

  // Chunk i of the step from k0 on; `left` elements of it exist
  __device__ __forceinline__ const T *chunk(int i, int k0, int &left) const {
    const bool last = k0 + kStep > K;
    left = kN;
    if (kAcross) {
      if (!kFast) left = min(cols - column(i), kN);
      if (last && k0 + row(i) >= K) left = 0;
      return at[i] + (int64_t)(kMapped ? mapped[kMapped ? i : 0] : k0) * o.ld;
    }
    if (last) left = K - k0 - source(i) * kN;
    return at[i] + k0;
  }
  // to `lds`; past the end zeros (kFast)
  __device__ __forceinline__ void load(int i, int k0, char *lds) const {
    int left;
    const T *p = chunk(i, k0, left);
    if (left <= 0) p = (const T *)&zero_chunk;
    load_to_lds(p, lds + (i * kThreads + (threadIdx.x & ~63)) * 16);
  }
  // Steps whose chunks can be read whole: to the shared axis' end along it; of
  // an operand across it the last chunk of a row may reach into the next row
  // (columns that are not stored), but not past the array.
  __device__ __forceinline__ int whole_steps() const {
    int n = K / kStep;
    if (kAcross && col + kRows > cols) {
      if (kMapped) {  // rows in ascending order: only the last may be the array's last
        if (cols < kN) return 0;
        if (n > 0 && n * kStep == K && o.end - o.row(K - 1) < cols + kN - 1) n--;
        return n;
      }
      while (n > 0 && o.end - (o.p + ((int64_t)n * kStep - 1) * o.ld) < cols + kN - 1) n--;
    }
    return n;
  }
  // Chunk i of the step from k0 on, whole or as much of it as exists
  __device__ __forceinline__ Chunk fetch_whole(int i, int k0) const {
    int left;
    return __builtin_bit_cast(Chunk, load_vec<T, false>(chunk(i, k0, left), kN));
  }
  __device__ __forceinline__ Chunk fetch(int i, int k0) const {
    int left;
    const T *p = chunk(i, k0, left);
    return __builtin_bit_cast(Chunk, load_vec<T, true>(p, left));
  }
};

// Operand of rows r0..r0+15 of a tile, half `part` of its step
template <class T, bool kAcross, int kRows>
__device__ __forceinline__ Frag<T> read_frag(const char *lds, int r0, int part) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  constexpr int kN = Vec<T>::kN, kChunks = kAcross ? kRows / kN : 8;
  Frag<T> f;
  if constexpr (!kAcross) {
    const int row = r0 + r;
    f.v = *(const typename Vec<T>::V *)(lds + row * kStepBytes +
                                        chunk_place<T, false, kChunks>(row, part * 4 + g) * 16);
  } else if constexpr (sizeof(T) == 2) {
    // Two transposing reads: of the 16 lanes of a group lanes 4 j + i read 4
    // columns each of row j, and lane r gets column r of rows 0 to 3.
    typedef short S4 __attribute__((ext_vector_type(4)));
    S4 h[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int k = part * 32 + g * 8 + j * 4 + (r >> 2), c = r0 + (r & 3) * 4;
      const char *p = lds + k * (kRows * 2) + chunk_place<T, true, kChunks>(k, c >> 3) * 16 +
                      (c & 7) * 2;
      h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)p);
    }
    typedef short S8 __attribute__((ext_vector_type(8)));
    f.v = __builtin_bit_cast(typename Vec<T>::V,
                             (S8)__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    const int c = r0 + r;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int k = part * 16 + g * 4 + i;
      f.v[i] = *(const float *)(lds + k * (kRows * 4) +
                                chunk_place<T, true, kChunks>(k, c >> 2) * 16 + (c & 3) * 4);
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
