// Rows of activations in registers, shared by the operators that normalise them (norm.hip, resnorm.h): pieces of 16 bytes on any
// element, sums over a row's waves.
#pragma once

#include "ff_internal.h"

namespace ff {
namespace norm {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 Loose __attribute__((aligned(2)));   // on any element

// A piece of 16 bytes as it lies in memory, on any element: rows of odd widths start anywhere, and the memory unit
// takes such pieces whole.
template <class E>
struct Pack {
  static constexpr int kN = 16 / (int)sizeof(E);
  typedef u32x4 Raw;
  static __device__ __forceinline__ Raw load(const E* p) { return *reinterpret_cast<const Loose*>(p); }
  static __device__ __forceinline__ void widen(Raw w, float* v) {
    if constexpr (sizeof(E) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned u = w[i];
        v[i] = __builtin_bit_cast(float, u);
      }
    }
  }
  static __device__ __forceinline__ void put(E* p, const float* v) {
    u32x4 w;
    if constexpr (sizeof(E) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = (unsigned)__builtin_bit_cast(unsigned short, (__bf16)v[2 * i]) |
               (unsigned)__builtin_bit_cast(unsigned short, (__bf16)v[2 * i + 1]) << 16;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(unsigned, v[i]);
    }
    *reinterpret_cast<Loose*>(p) = w;
  }
};

// N values of weight or bias from column c (absent: `none`)
template <int N>
__device__ __forceinline__ void vector_at(const void* p, int bf16, float none, int c, float* v) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = none;
  } else if (bf16) {
    const __bf16* q = static_cast<const __bf16*>(p) + c;
    if constexpr (N == 8) {
      Pack<__bf16>::widen(Pack<__bf16>::load(q), v);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = (float)q[i];
    }
  } else {
    const float* q = static_cast<const float*>(p) + c;
    if constexpr (N >= 4) {
#pragma unroll
      for (int i = 0; i < N; i += 4) Pack<float>::widen(Pack<float>::load(q + i), v + i);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = q[i];
    }
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Sums over the WV waves of a row (the whole workgroup when WV > 1); `sh` has two floats per wave.
template <int WV>
__device__ __forceinline__ float2 row_sum(float2 v, float2* sh) {
  v.x = wave_sum(v.x);
  v.y = wave_sum(v.y);
  if constexpr (WV > 1) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int i = 1; i < WV; ++i) v.x += sh[i].x, v.y += sh[i].y;
  }
  return v;
}

constexpr int threads_of(int wv) { return wv == 1 ? 256 : wv * 64; }

// The pieces of a thread in a row of n elements: piece i WV 64 + l from its element at(i) on, of which those below skip(i)
// are another piece's (all of them: no piece).  PART: n is no whole number of pieces; the last one then is the 16 bytes
// that end with the row, so that every access is whole.  What it shares with the piece before is computed by both
// alike, and enters sums once.
template <class E, int NV, int WV, bool PART>
struct Row {
  static constexpr int kN = Pack<E>::kN;
  u32x4 raw[NV];
  static __device__ __forceinline__ int skip(int i, int l, int n) {
    const int left = n - (i * WV * 64 + l) * kN;
    if (!PART) return left > 0 ? 0 : kN;
    return left >= kN ? 0 : (left > 0 ? kN - left : kN);
  }
  static __device__ __forceinline__ int at(int i, int l, int n) {
    const int c = (i * WV * 64 + l) * kN;
    return PART && c > n - kN ? n - kN : c;
  }
  __device__ __forceinline__ void load(const void* base, int64_t ld, int64_t t, int l, int n) {
    const E* p = static_cast<const E*>(base) + t * ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (skip(i, l, n) < kN) raw[i] = Pack<E>::load(p + at(i, l, n));
      else raw[i] = u32x4{0u, 0u, 0u, 0u};
    }
  }
};

}  // namespace norm
}  // namespace ff
