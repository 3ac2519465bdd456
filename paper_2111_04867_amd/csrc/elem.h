// Rows of 16-byte vectors and wavefront reductions of the expert-layer
// kernels (gfx950).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "wave.h"

namespace taccl {

using bf16_t = __bf16;
using f16_t = _Float16;

// VE elements of one 16-byte vector; the global access needs only the
// element's alignment (gfx950 takes any address).
template <class T>
struct Vec {
  static constexpr int kN = 16 / (int)sizeof(T);
  typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef V U __attribute__((aligned(sizeof(T))));
};

// The vector at p. Of the columns from `left` on nothing is read or written
// and they come as zero; kTail: fewer than kN may be left (else none or kN).
// Such a rest is read and written as its binary digits: 4, 2 and 1 elements.
template <class T, bool kTail>
__device__ __forceinline__ typename Vec<T>::V load_vec(const T *p, int left) {
  constexpr int N = Vec<T>::kN;
  typedef T T4 __attribute__((ext_vector_type(4)));
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef T4 U4 __attribute__((aligned(sizeof(T))));
  typedef T2 U2 __attribute__((aligned(sizeof(T))));
  typename Vec<T>::V v;
#pragma unroll
  for (int i = 0; i < N; i++) v[i] = (T)0.0f;
  if (left >= N) {
    v = *(const typename Vec<T>::U *)p;
  } else if (kTail && left > 0) {
    T4 w4 = {(T)0.0f, (T)0.0f, (T)0.0f, (T)0.0f};
    T2 w2 = {(T)0.0f, (T)0.0f};
    T w1 = (T)0.0f;
    if (N == 8 && (left & 4)) w4 = *(const U4 *)p;
    if (left & 2) w2 = *(const U2 *)(p + (left & 4));
    if (left & 1) w1 = p[left & 6];
    if constexpr (N == 8) {
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] = w4[i];
#pragma unroll
      for (int i = 0; i < 2; i++) {
        v[i] = left & 4 ? v[i] : w2[i];
        v[4 + i] = left & 4 ? w2[i] : (T)0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) v[i] = (left & 1) && (left & 6) == i ? w1 : v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 2; i++) v[i] = w2[i];
      v[0] = left == 1 ? w1 : v[0];
      v[2] = left == 3 ? w1 : (T)0.0f;
    }
  }
  return v;
}

template <class T, bool kTail>
__device__ __forceinline__ void store_vec(T *p, typename Vec<T>::V v, int left) {
  constexpr int N = Vec<T>::kN;
  typedef T T4 __attribute__((ext_vector_type(4)));
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef T4 U4 __attribute__((aligned(sizeof(T))));
  typedef T2 U2 __attribute__((aligned(sizeof(T))));
  if (left >= N) {
    *(typename Vec<T>::U *)p = v;
  } else if (kTail && left > 0) {
    T2 w2 = {v[0], v[1]};
    T w1 = v[0];
    if constexpr (N == 8) {
      if (left & 4) {
        *(U4 *)p = T4{v[0], v[1], v[2], v[3]};
        w2 = T2{v[4], v[5]};
      }
#pragma unroll
      for (int i = 2; i < 8; i += 2) w1 = (left & 6) == i ? v[i] : w1;
    } else {
      w1 = left & 2 ? v[2] : w1;
    }
    if (left & 2) *(U2 *)(p + (left & 4)) = w2;
    if (left & 1) p[left & 6] = w1;
  }
}

// The same vector, whose conversions to float are not kept across this point:
// 16-bit rows held as they are stored take half the registers.
template <class V>
__device__ __forceinline__ void as_stored(V &v) {
  asm volatile("" : "+v"(v));
}

// Moves within a row of 16 lanes, every lane of it active: with the bound
// control set there is no old value to keep, and the move becomes an operand
// of what uses it.
template <int Ctrl>
__device__ __forceinline__ int dppi(int v) {
  return __builtin_amdgcn_update_dpp(0, v, Ctrl, 0xf, 0xf, true);
}
template <int Ctrl>
__device__ __forceinline__ float dppf(float v) {
  return __builtin_bit_cast(float, dppi<Ctrl>(__builtin_bit_cast(int, v)));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
constexpr int kRor8 = 0x128, kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;

// Sums and maxima over groups of L lanes (16: one DPP row; 32; 64: the
// wavefront), the same in every lane of the group. Sums go down a fixed tree.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dppf<kRor8>(v);
  v += dppf<kRor4>(v);
  v += dppf<kRor2>(v);
  v += dppf<kRor1>(v);
  if (L >= 32) v += __shfl_xor(v, 16);
  if (L == 64) v += __shfl_xor(v, 32);
  return v;
}
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, dppf<kRor8>(v));
  v = fmaxf(v, dppf<kRor4>(v));
  v = fmaxf(v, dppf<kRor2>(v));
  v = fmaxf(v, dppf<kRor1>(v));
  if (L >= 32) v = fmaxf(v, __shfl_xor(v, 16));
  if (L == 64) v = fmaxf(v, __shfl_xor(v, 32));
  return v;
}
template <int L>
__device__ __forceinline__ uint32_t lanes_min(uint32_t v) {
  v = min(v, (uint32_t)dppi<kRor8>((int)v));
  v = min(v, (uint32_t)dppi<kRor4>((int)v));
  v = min(v, (uint32_t)dppi<kRor2>((int)v));
  v = min(v, (uint32_t)dppi<kRor1>((int)v));
  if (L >= 32) v = min(v, (uint32_t)__shfl_xor((int)v, 16));
  if (L == 64) v = min(v, (uint32_t)__shfl_xor((int)v, 32));
  return v;
}

}  // namespace taccl
