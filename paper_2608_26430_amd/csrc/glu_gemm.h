// Matrix products of the gated feed-forward (glu.hip has the calls), on the operand tiles of xent_gemm.h.
//
//   G = X Wg^T [+ Ag],  U = X Wu^T [+ Au],  H = f(G) U                 projection_kernel, kForward (G and U kept or not)
//   dU = dH f(G),  dG = dH U f'(G), G and U made again                 projection_kernel, kBackward
//   dX = dG Wg + dU Wu                                                 gradient_kernel, one sum over both halves of k
//   dWg = dG^T X,  dWu = dU^T X                                        gradient_kernel, two results
// Here i runs along the rows of memory of a result, j over its rows, and every product is out[j][i] = sum_k A(i, k) B(j, k).
//
// projection_kernel: a workgroup's tile of BM has BM / 2 columns of both products: the same columns of G and U end in the same lane's
// registers, and f needs nothing from elsewhere.  Its end reads and writes rows of memory, 16 bytes a lane in bf16 where a wave has
// 32 columns or more.
//
// Large products are bound by the matrix units and the LDS reads that feed them, about alike (a step of 256 x 256 x 64 is 2048
// cycles of either), middle ones by LDS and a tile's start and end, those of few tokens by reading the weights.  Measured, bf16:
// 4096 tokens of 4096 -> 11008 with addends and G, U kept 660 to 700 us (1.06 to 1.12 PFLOP/s), dX 531 to 575 (1.28 to 1.39);
// 2003 tokens of 1024 -> 4096 with addends and GELU 40 us; one token of 4096 -> 11008 33 to 36 us (5.1 TB/s).  fp32, 500 tokens of
// 768 -> 2048: 33 to 35 us each product (90 to 94 TFLOP/s).
#pragma once

#include "xent_gemm.h"

namespace ff {
namespace glu {

using xent::f32x4;
using xent::load4;
using xent::Mma;
using xent::Operand;
using xent::ring_wait;
using xent::store4;
using xent::store8;
using xent::u32x4;
using xent::up;

enum Mode { kForward = 0, kBackward = 1 };

// The lane's number, made anew: where a tile starts and ends it would otherwise take a register (and with it a spill) over the
// whole main loop.
__device__ __forceinline__ int fresh_lane() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

struct ProjArgs {
  const void* Wg;
  const void* Wu;
  const void* X;
  int64_t ldw, ldx;
  int F, T, n;            // columns and rows of the results, length of the sums
  int tm, tn;             // tiles along the columns and the rows
  int rest;               // of them, those that are halved (at most as many as half of the workgroups)
  int kt;                 // k tiles
  const void* Ag;         // NULL: none
  const void* Au;
  int64_t lda;
  const void* dH;         // kBackward
  int64_t lddh;
  void* H;                // kForward
  int64_t ldh;
  void* G;                // kForward: NULL if not kept (Kept words); kBackward: dG
  void* U;                //           dU
  int64_t ldg;
};

// f(g) and f'(g).  Fast: 1 ulp exponentials and reciprocals, for results that are rounded to bf16.
__device__ __forceinline__ float exp_of(float x, bool fast) { return fast ? __builtin_amdgcn_exp2f(x * 1.4426950408889634f) : expf(x); }
__device__ __forceinline__ float inverse(float x, bool fast) { return fast ? __builtin_amdgcn_rcpf(x) : 1.f / x; }

constexpr float kSaturated = 0x1p60f;      // f' is 1 or 0 there, and from 1e3 on

template <int FN, bool FAST>
__device__ __forceinline__ float2 gated(float g) {
  if constexpr (FN == FF_GLU_SILU) {
    const float s = inverse(1.f + exp_of(-g, FAST), FAST);
    return make_float2(g * s, s * fmaf(g, 1.f - s, 1.f));
  } else if constexpr (FN == FF_GLU_GELU) {
    const float e = exp_of(-0.5f * g * g, FAST);
    float cdf;
    if constexpr (FAST) {
      // erfc(x) = exp(-x^2) Q(1 / (1 + 0.33 x)) for x = |g| / sqrt 2: Q is the polynomial of the least relative error over x from 0 to
      // 10, 1e-7 (at most 1.1e-6 in fp32 arithmetic; tests/test_glu_function.py has the fit and the bound).  The library's erfc took 7
      // of 41 us (2003 tokens, 1024 -> 4096).
      const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.33f * 0.70710678118654752f, 1.f));
      float q = fmaf(t, -0.135348532f, 0.460249317f);
      q = fmaf(t, q, -0.351171446f);
      q = fmaf(t, q, 0.408520793f);
      q = fmaf(t, q, 0.0472091254f);
      q = fmaf(t, q, 0.201227576f);
      q = fmaf(t, q, 0.182955311f);
      q = fmaf(t, q, 0.186357848f);
      const float half = 0.5f * t * q * e;
      cdf = g < 0.f ? half : 1.f - half;
    } else {
      cdf = 0.5f * erfcf(g * -0.70710678118654752f);   // keeps the digits of f where g is far below zero
    }
    return make_float2(g * cdf, fmaf(g, 0.39894228040143268f * e, cdf));
  } else {
    // sqrt(2 / pi) (g + 0.044715 g^3), whose tanh is 2 s - 1
    constexpr float c = 0.79788456080286536f;
    const float s = inverse(1.f + exp_of(-2.f * c * g * fmaf(0.044715f * g, g, 1.f), FAST), FAST);
    const float b = __builtin_amdgcn_fmed3f(g, -kSaturated, kSaturated);    // whose square is a number; g s (1 - s) is zero long before
    return make_float2(g * s, fmaf(g * s * (1.f - s), 2.f * c * fmaf(3.f * 0.044715f * b, b, 1.f), s));
  }
}

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// W (4 or 8) consecutive elements.
template <int W>
__device__ __forceinline__ void load_run(const __bf16* p, float (&v)[W]) {
  if constexpr (W == 8) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
    }
  } else {
    const f32x4 w = load4(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
  }
}
template <int W>
__device__ __forceinline__ void load_run(const float* p, float (&v)[W]) {
#pragma unroll
  for (int q = 0; q < W; q += 4) {
    const f32x4 w = load4(p + q);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[q + i] = w[i];
  }
}
template <int W>
__device__ __forceinline__ void store_run(__bf16* p, const float (&v)[W]) {
  if constexpr (W == 8) store8(p, f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]});
  else store4(p, f32x4{v[0], v[1], v[2], v[3]});
}
template <int W>
__device__ __forceinline__ void store_run(float* p, const float (&v)[W]) {
#pragma unroll
  for (int q = 0; q < W; q += 4) store4(p + q, f32x4{v[q], v[q + 1], v[q + 2], v[q + 3]});
}

// G and U as they are kept: fp32 as they are, for bf16 activations words of 16 bits with ten significant ones: a sign, 6 bits of
// exponent (bias 37: 1.5e-11 to 6.7e7 in full, smaller ones as subnormals, larger ones as infinity), 9 of mantissa.  In bf16, with
// eight, their roundings would be as large as those of dG and dU themselves and add to them: 4096 tokens 4096 -> 11008, dU 0.0030
// off and dX 0.0031 (relative norm), 0.0018 and 0.0024 so.  A NaN is kept as the positive infinity, whose f is infinite too.
constexpr float kKeepDown = 0x1p-90f, kKeepUp = 0x1p90f;     // fp32's exponent to the words' and back
constexpr float kKeepMost = 0x1p-64f;                        // of a value times kKeepDown: the word of infinity
template <class E>
struct Kept;
template <>
struct Kept<float> {
  typedef float Word;
  template <int W>
  static __device__ __forceinline__ void put(float* p, const float (&v)[W]) {
    store_run<W>(p, v);
  }
  typedef f32x4 Raw;
  static __device__ __forceinline__ bool infinite(Raw, Raw) { return false; }
  static __device__ __forceinline__ float any_value(float x) { return x; }
  static __device__ __forceinline__ void get(Raw r, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r[i];
  }
};
template <>
struct Kept<__bf16> {
  typedef uint16_t Word;
  static __device__ __forceinline__ unsigned word(float x) {
    // rounded to nearest, halves away from zero; the sign moves down beside the six bits of exponent.  (Of -x, as a NaN comes out as the
    // lower limit; the sum turns the sign back.)
    const unsigned b = (__builtin_bit_cast(unsigned, __builtin_amdgcn_fmed3f(x * -kKeepDown, -kKeepMost, kKeepMost)) + 0x80002000u) >> 14;
    return (b & 0x7fffu) | (b >> 2 & 0x8000u);
  }
  // of a word that is not infinite, and of any
  static __device__ __forceinline__ float value(unsigned w) {
    return __builtin_bit_cast(float, (w & 0x7fffu) << 14 | (w & 0x8000u) << 16) * kKeepUp;
  }
  static __device__ __forceinline__ float any_value(unsigned w) {
    const float x = value(w);
    return fabsf(x) < kKeepMost * kKeepUp ? x : x * INFINITY;
  }
  template <int W>
  static __device__ __forceinline__ void put(uint16_t* p, const float (&v)[W]) {
    unsigned x[W / 2];
#pragma unroll
    for (int i = 0; i < W / 2; ++i) x[i] = word(v[2 * i]) | word(v[2 * i + 1]) << 16;
    if constexpr (W == 8) *reinterpret_cast<u32x4*>(p) = u32x4{x[0], x[1], x[2], x[3]};
    else *reinterpret_cast<u32x2*>(p) = u32x2{x[0], x[1]};
  }
  typedef u32x4 Raw;
  // Whether one of two pieces' words has an exponent of ones: it then carries into the sign's place.
  static __device__ __forceinline__ bool infinite(Raw a, Raw b) {
    unsigned any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) any |= ((a[i] & 0x7e007e00u) + 0x02000200u) | ((b[i] & 0x7e007e00u) + 0x02000200u);
    return any & 0x80008000u;
  }
  static __device__ __forceinline__ void get(Raw r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = value(r[i] & 0xffffu), v[2 * i + 1] = value(r[i] >> 16);
  }
};

// What the end of a tile reads, W columns from c of row t, as it lies in memory: all of a wave's are on their way at once.
template <class E, int W, int MODE>
struct RawExtra {
  typedef unsigned Raw __attribute__((ext_vector_type(W * (int)sizeof(E) / 4)));
  Raw g, u, x;
  __device__ __forceinline__ void load(const ProjArgs& a, int64_t t, int c) {
    if (a.Ag) g = *reinterpret_cast<const Raw*>(static_cast<const E*>(a.Ag) + t * a.lda + c);
    if (a.Au) u = *reinterpret_cast<const Raw*>(static_cast<const E*>(a.Au) + t * a.lda + c);
    if constexpr (MODE == kBackward) x = *reinterpret_cast<const Raw*>(static_cast<const E*>(a.dH) + t * a.lddh + c);
  }
  static __device__ __forceinline__ float at(const Raw& r, int i) {
    if constexpr (sizeof(E) == 4) {
      const unsigned v = r[i];
      return __builtin_bit_cast(float, v);
    } else {
      const unsigned v = r[i / 2];
      return __builtin_bit_cast(float, i % 2 ? v & 0xffff0000u : v << 16);
    }
  }
};

// The end of W columns from c of row t: what is added, f, and what is written.
template <class E, int FN, int MODE, int W>
__device__ __forceinline__ void finish_run(const ProjArgs& a, int64_t t, int c, float (&g)[W], float (&u)[W],
                                           const RawExtra<E, W, MODE>& r) {
  constexpr bool kFast = sizeof(E) == 2;
  if (a.Ag) {
#pragma unroll
    for (int i = 0; i < W; ++i) g[i] += r.at(r.g, i);
  }
  if (a.Au) {
#pragma unroll
    for (int i = 0; i < W; ++i) u[i] += r.at(r.u, i);
  }
  if constexpr (MODE == kForward) {
    typedef typename Kept<E>::Word Word;
    if (a.G) {
      Kept<E>::put(static_cast<Word*>(a.G) + t * a.ldg + c, g);
      Kept<E>::put(static_cast<Word*>(a.U) + t * a.ldg + c, u);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) g[i] = gated<FN, kFast>(g[i]).x * u[i];
    store_run<W>(static_cast<E*>(a.H) + t * a.ldh + c, g);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float2 f = gated<FN, kFast>(g[i]);
      const float x = r.at(r.x, i);
      g[i] = x * u[i] * f.y;
      u[i] = x * f.x;
    }
    store_run<W>(static_cast<E*>(a.G) + t * a.ldg + c, g);
    store_run<W>(static_cast<E*>(a.U) + t * a.ldg + c, u);
  }
}

constexpr int kHalfNB = 3;      // buffers of a halved large tile, which take its 128 KB and 16 more
constexpr int lds_bytes(int BM, int BN, int NB) {
  const int whole = NB * (BM + BN), half = BN == 256 ? kHalfNB * (BM + BN / 2) : 0;
  return (whole > half ? whole : half) * xent::kTileBytes;
}

// A workgroup's share of `total` tiles: numbers wg, wg + step, ..; place(number, &i0, &j0) is where a tile is.
template <class E, int BM, int BN, int WVM, int WVN, int NB, int FN, int MODE, class Place>
__device__ __forceinline__ void project(const ProjArgs& a, char* lds, int wg, int step, int total, const Place& place_of) {
  constexpr int NW = WVM * WVN;
  constexpr int TH = BM / 2 / WVM, TN = BN / WVN;        // columns of each product, rows of a wave
  constexpr int FH = TH / 16, FM = 2 * FH, FNT = TN / 16;
  constexpr int PF = sizeof(E) == 2 && FH >= 2 ? 2 : 0;
  typedef Operand<E, BM / 2, NW, false, PF> OpA;
  typedef Operand<E, BN, NW, false, 0> OpB;
  constexpr int kBuf = 2 * OpA::kBytes + OpB::kBytes;
  constexpr int kLoads = 2 * OpA::kLoads + OpB::kLoads;
  constexpr int kK = OpA::kK;
  constexpr bool kAhead = BN > 32;     // a half tile's fragments are read under the other half's products
  constexpr int kReads = FM * OpA::kReads + FNT * OpB::kReads;
  constexpr int kMmas = FM * FNT * (sizeof(E) == 2 ? 1 : 4);

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WVM, wn = wave / WVM;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  OpA og, ou;
  OpB ob;
  og.init(a.ldw, wave, lane);
  ou.init(a.ldw, wave, lane);
  ob.init(a.ldx, wave, lane);
  int i0, j0, i_next, j_next;
  // (the same for all lanes: kept in scalar registers)
  auto place = [&](int at) {
    int i, j;
    place_of(at, &i, &j);
    i_next = __builtin_amdgcn_readfirstlane(i), j_next = __builtin_amdgcn_readfirstlane(j);
  };
  auto issue_last = [&]() {
    const int left = a.n - (a.kt - 1) * kK;
    const int own = fresh_lane();
    og.issue_last(a.kt - 1, left, a.ldw, i0, a.F, lds0, wave, own);
    ou.issue_last(a.kt - 1, left, a.ldw, i0, a.F, lds0 + OpA::kBytes, wave, own);
    ob.issue_last(a.kt - 1, left, a.ldx, j0, a.T, lds0 + 2 * OpA::kBytes, wave, own);
  };
  auto issue = [&](int t, int buf) {
    const unsigned to = lds0 + buf * kBuf;
    og.issue(t < a.kt, to, wave);
    ou.issue(t < a.kt, to + OpA::kBytes, wave);
    ob.issue(t < a.kt, to + 2 * OpA::kBytes, wave);
  };
  // k is walked with its last tile first, so that only the first loads look at its end
  auto start = [&]() {
    i0 = i_next, j0 = j_next;
    og.seek(a.Wg, a.ldw, i0, a.F, 0);
    ou.seek(a.Wu, a.ldw, i0, a.F, 0);
    ob.seek(a.X, a.ldx, j0, a.T, 0);
    issue_last();
#pragma unroll
    for (int t = 1; t < (kAhead ? NB : NB - 1); ++t) issue(t, t);
  };

  place(wg);
  start();
  for (;;) {
    place(wg + step);
    f32x4 acc[FM][FNT];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int j = 0; j < FNT; ++j) acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // fp32: sums of 128 k, then their sum, so that rounding grows with the length of both
    constexpr bool kBlocked = sizeof(E) == 4;
    f32x4 sum[kBlocked ? FM : 1][kBlocked ? FNT : 1] = {};
    auto close_block = [&](bool end) {
      if constexpr (kBlocked) {
        if (!end) return;
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int j = 0; j < FNT; ++j) {
            sum[f][j] += acc[f][j];
            acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
      }
    };
    auto read = [&](int buf, int kk, f32x4 (&fa)[FM], f32x4 (&fb)[FNT]) {
      const char* la = lds + buf * kBuf;
#pragma unroll
      for (int j = 0; j < FNT; ++j) fb[j] = OpB::read(la + 2 * OpA::kBytes, wn * TN, j, kk, lane);
#pragma unroll
      for (int f = 0; f < FH; ++f) {
        fa[f] = OpA::read(la, wm * TH, f, kk, lane);
        fa[FH + f] = OpA::read(la + OpA::kBytes, wm * TH, f, kk, lane);
      }
    };
    auto multiply = [&](const f32x4 (&fa)[FM], const f32x4 (&fb)[FNT]) {
#pragma unroll
      for (int k = 0; k < Mma<E>::kSteps; ++k)
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int j = 0; j < FNT; ++j) acc[f][j] = Mma<E>::step(k, fa[f], fb[j], acc[f][j]);
    };
    if constexpr (kAhead) {
      f32x4 fa[2][FM], fb[2][FNT];
      ring_wait<(NB - 1) * kLoads>();
      read(0, 0, fa[0], fb[0]);
      for (int t0 = 0; t0 < a.kt; t0 += NB) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (t0 + b >= a.kt) break;
          read(b, 1, fa[1], fb[1]);
          multiply(fa[0], fb[0]);
          xent::interleave<kReads, kMmas>();
          ring_wait<(NB - 2) * kLoads>();
          if (NB > 2 || t0 + b + 2 < a.kt) issue(t0 + b + NB, b);
          read((b + 1) % NB, 0, fa[0], fb[0]);
          multiply(fa[1], fb[1]);
          xent::interleave<kReads, kMmas>();
          close_block((t0 + b) % 4 == 3);
        }
      }
    } else {
      for (int t0 = 0; t0 < a.kt; t0 += NB) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (t0 + b >= a.kt) break;
          ring_wait<(NB - 2) * kLoads>();
          issue(t0 + b + NB - 1, (b + NB - 1) % NB);
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            f32x4 fa[FM], fb[FNT];
            read(b, kk, fa, fb);
            multiply(fa, fb);
          }
          close_block((t0 + b) % 4 == 3);
        }
      }
    }
    if constexpr (kBlocked) {
#pragma unroll
      for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int j = 0; j < FNT; ++j) acc[f][j] += sum[f][j];
    }
    const int ci = i0 + wm * TH, cj = j0 + wn * TN;
    wg += step;
    const bool more = wg < total;
    if (more) {
      ring_wait<0>();      // every wave's reads of the buffers are done
      start();
    }
    const int own = fresh_lane();
    const int g = own >> 4, r = own & 15;
    constexpr int P = PF ? PF : 1, W = 4 * P;
    constexpr int JB = FNT > 2 && sizeof(E) == 2 ? 2 : 1;    // more rows' at once would spill
#pragma unroll
    for (int j0 = 0; j0 < FNT; j0 += JB) {
      RawExtra<E, W, MODE> extra[JB][FH / P];
      if (MODE == kBackward || a.Ag || a.Au) {
        // (rows and columns past the last read those of the last, and are not written)
#pragma unroll
        for (int j = 0; j < JB; ++j)
#pragma unroll
          for (int f = 0; f < FH; f += P) {
            const int row = cj + (j0 + j) * 16 + r, c = ci + f * 16 + g * W;
            extra[j][f / P].load(a, row < a.T ? row : a.T - 1, c < a.F ? c : a.F - W);
          }
      }
#pragma unroll
      for (int j = 0; j < JB; ++j) {
        const int row = cj + (j0 + j) * 16 + r;
#pragma unroll
        for (int f = 0; f < FH; f += P) {
          const int c = ci + f * 16 + g * W;
          float x[W], y[W];
#pragma unroll
          for (int q = 0; q < P; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * q + i] = acc[f + q][j0 + j][i], y[4 * q + i] = acc[FH + f + q][j0 + j][i];
          if (row < a.T && c < a.F) finish_run<E, FN, MODE, W>(a, row, c, x, y, extra[j][f / P]);
        }
      }
    }
    if (!more) break;
  }
  // no direct load may be in flight when the workgroup's LDS is given to another one
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <class E, int BM, int BN, int WVM, int WVN, int NB, int WPE, int FN, int MODE>
__global__ void __launch_bounds__(WVM * WVN * 64, WPE) projection_kernel(ProjArgs a) {
  __shared__ __align__(1024) char lds[lds_bytes(BM, BN, NB)];
  const int full = a.tm * a.tn - a.rest;
  // Large tiles: those of a last (or only) round that would leave half of the CUs idle go out as halves of fewer rows.  They come first: their
  // workgroups' tiles then end at other times than the others', and the ends share the memory.
  if constexpr (BN == 256) {
    const int halves = 2 * a.rest;
    auto half = [&](int at, int* i, int* j) {
      const int id = xent::share_of(at, halves);
      int im, in;
      xent::tile_of(full + id / 2, a.tm, a.tn, &im, &in);
      *i = im * (BM / 2), *j = in * BN + id % 2 * (BN / 2);
    };
    if ((int)blockIdx.x < halves) {
      int i, j;
      half(blockIdx.x, &i, &j);
      // (not the second half of a last tile of few rows)
      if (j < a.T) project<E, BM, BN / 2, 2 * WVM, WVN / 2, kHalfNB, FN, MODE>(a, lds, blockIdx.x, halves, halves, half);
      __syncthreads();
    }
  }
  if ((int)blockIdx.x < full)
    project<E, BM, BN, WVM, WVN, NB, FN, MODE>(a, lds, blockIdx.x, gridDim.x, full, [&](int at, int* i, int* j) {
      int im, in;
      xent::tile_of(xent::share_of(at, full), a.tm, a.tn, &im, &in);
      *i = im * (BM / 2), *j = in * BN;
    });
}

// Few tokens, or few columns: 16 FNT rows, 16 columns of each product a workgroup.  Its KS waves share k in chunks of 256 bytes and read the
// weights straight into the registers of the MFMA (64 bytes of a row in four lanes), the next chunk under the products of one; nothing
// is read twice but X, which is small.  The waves' sums are added up in a fixed order.
template <class E, int FNT, int KS, int FN, int MODE>
__global__ void __launch_bounds__(KS * 64) narrow_kernel(ProjArgs a) {
  constexpr int kPer = 16 / (int)sizeof(E), kStep = 4 * kPer, kSteps = 4, kChunk = kSteps * kStep;
  __shared__ f32x4 part[KS][2 * FNT][64];
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // an XCD's workgroups take all rows of a run of columns, whose weights are then read into one L2
  const int rows = (a.T + 16 * FNT - 1) / (16 * FNT), id = xent::share_of(blockIdx.x, gridDim.x);
  const int c0 = id / rows * 16, t0 = id % rows * (16 * FNT);
  // columns past the last read its weights, and their results are not written
  const int64_t row = c0 + r < a.F ? c0 + r : a.F - 1;
  const E* wg = static_cast<const E*>(a.Wg) + row * a.ldw + g * kPer;
  const E* wu = static_cast<const E*>(a.Wu) + row * a.ldw + g * kPer;
  const E* x[FNT];
#pragma unroll
  for (int j = 0; j < FNT; ++j) x[j] = static_cast<const E*>(a.X) + (int64_t)(t0 + j * 16 + r < a.T ? t0 + j * 16 + r : 0) * a.ldx + g * kPer;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 ag[FNT], au[FNT];
#pragma unroll
  for (int j = 0; j < FNT; ++j) ag[j] = au[j] = zero;
  f32x4 fg[kSteps], fu[kSteps], fx[kSteps][FNT];
  auto load = [&](int k0) {
    const bool whole = k0 + kChunk <= a.n;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int k = k0 + s * kStep;
      const bool in = whole || k + g * kPer < a.n;
      fg[s] = fu[s] = zero;
      if (in) {
        fg[s] = *reinterpret_cast<const f32x4*>(wg + k);
        fu[s] = *reinterpret_cast<const f32x4*>(wu + k);
      }
#pragma unroll
      for (int j = 0; j < FNT; ++j) {
        fx[s][j] = zero;
        if (in && t0 + j * 16 + r < a.T) fx[s][j] = *reinterpret_cast<const f32x4*>(x[j] + k);
      }
    }
  };
  int k0 = wave * kChunk;
  if (k0 < a.n) load(k0);
  while (k0 < a.n) {
    f32x4 cg[kSteps], cu[kSteps], cx[kSteps][FNT];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      cg[s] = fg[s], cu[s] = fu[s];
#pragma unroll
      for (int j = 0; j < FNT; ++j) cx[s][j] = fx[s][j];
    }
    k0 += KS * kChunk;
    if (k0 < a.n) load(k0);
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int q = 0; q < Mma<E>::kSteps; ++q)
#pragma unroll
        for (int j = 0; j < FNT; ++j) {
          ag[j] = Mma<E>::step(q, cg[s], cx[s][j], ag[j]);
          au[j] = Mma<E>::step(q, cu[s], cx[s][j], au[j]);
        }
  }
#pragma unroll
  for (int j = 0; j < FNT; ++j) part[wave][2 * j][lane] = ag[j], part[wave][2 * j + 1][lane] = au[j];
  __syncthreads();
  if (wave >= FNT) return;
  f32x4 sg = part[0][2 * wave][lane], su = part[0][2 * wave + 1][lane];
#pragma unroll
  for (int w = 1; w < KS; ++w) sg += part[w][2 * wave][lane], su += part[w][2 * wave + 1][lane];
  const int t = t0 + wave * 16 + r, c = c0 + g * 4;
  if (t >= a.T || c >= a.F) return;
  float vg[4], vu[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) vg[i] = sg[i], vu[i] = su[i];
  RawExtra<E, 4, MODE> extra;
  extra.load(a, t, c);
  finish_run<E, FN, MODE, 4>(a, t, c, vg, vu, extra);
}

struct GradArgs {
  const void* A[2];       // dX: Wg, Wu; dW: X
  const void* B[2];       // dG, dU
  int64_t lda, ldb;
  int M, N, K;            // dX: n, T, F (of each half of the sum); dW: n, F (of each result), T
  int tm, tn;             // tiles along i, and j (dW: of one result)
  int kt, kt_split;       // k tiles (dX: of each half), and those of one split
  int splits;
  int rest;               // of all tiles, those that are halved
  void* out[2];           // dX: the first; dW: dWg, dWu
  int64_t ldo;
  float beta;
  float* part;            // with splits > 1: [splits][N, dW: 2 N][M] fp32
};

// Where a tile is: which result, split of k, first column and row.
struct GradPlace {
  int which, split, i, j;
};

// A workgroup's share of `total` tiles: numbers wg, wg + step, ..  TRB: dG and dU stored along j (dW); otherwise along k (dX).
template <class E, int BM, int BN, int WVM, int WVN, int NB, bool TRB, class Place>
__device__ __forceinline__ void gradient(const GradArgs& a, char* lds, int wg, int step, int total, const Place& place_of) {
  constexpr int NW = WVM * WVN;
  constexpr int TM = BM / WVM, TN = BN / WVN;
  constexpr int FM = TM / 16, FNT = TN / 16;
  typedef Operand<E, BM, NW, true, 0> OpA;
  typedef Operand<E, BN, NW, TRB, 0> OpB;
  constexpr int kBuf = OpA::kBytes + OpB::kBytes;
  constexpr int kLoads = OpA::kLoads + OpB::kLoads;
  constexpr int kK = OpA::kK;
  constexpr bool kAhead = BN > 32;     // a half tile's fragments are read under the other half's products
  constexpr int kReads = FM * OpA::kReads + FNT * OpB::kReads;
  constexpr int kMmas = FM * FNT * (sizeof(E) == 2 ? 1 : 4);
  constexpr int kHalves = TRB ? 1 : 2, kOuts = TRB ? 2 : 1;
  static_assert((kAhead ? NB : NB - 1) >= kHalves, "the halves' last tiles are read before the loop");

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WVM, wn = wave / WVM;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  OpA oa;
  OpB ob;
  oa.init(a.lda, wave, lane);
  ob.init(a.ldb, wave, lane);
  int i0, j0, which, split, nk;          // the tile whose operands are being read; nk: its k tiles of a half
  GradPlace next;
  uint64_t second_a = 0, second_b = 0;   // where the second half starts
  // Large tiles of dX: the places that A's fragments are read from (as Operand::read has them) differ in three bits, and are made
  // from the first one's for each half tile.  Kept over the loop they leave no room for the places of the loads, whose reloading from
  // scratch waits for every load on its way (4096 tokens, 4096 <- 2 x 11008: 709 us, 545 without).
  constexpr bool kLean = sizeof(E) == 2 && BM == 256 && !TRB;
  unsigned a0 = 0;
  if constexpr (kLean) {
    const int k = (lane >> 4) * 8 + ((lane & 15) >> 2), cb = wm * TM * 2 + (lane & 3) * 8;
    a0 = k * OpA::kRow + (((cb >> 4) ^ OpA::swizzle(k)) << 4 | (cb & 15));
  }
  auto place = [&](int at) {
    const GradPlace p = place_of(at);
    next.which = __builtin_amdgcn_readfirstlane(p.which), next.split = __builtin_amdgcn_readfirstlane(p.split);
    next.i = __builtin_amdgcn_readfirstlane(p.i), next.j = __builtin_amdgcn_readfirstlane(p.j);
  };
  // A half's last k tile comes first, so that only the first loads look at its end: the sequence is the last tiles of the
  // halves, then the others of the first, then those of the second.
  auto issue_last = [&](int h) {
    const int last = a.K - (split * a.kt_split + nk - 1) * kK;
    const unsigned to = lds0 + h * kBuf;
    const int own = fresh_lane();
    oa.issue_last(nk - 1, last < kK ? last : kK, a.lda, i0, a.M, to, wave, own);
    ob.issue_last(nk - 1, last < kK ? last : kK, a.ldb, j0, a.N, to + OpA::kBytes, wave, own);
  };
  auto issue = [&](int t, int buf) {
    if (kHalves == 2 && t == nk + 1) oa.base = second_a, ob.base = second_b;
    const unsigned to = lds0 + buf * kBuf;
    oa.issue(t < kHalves * nk, to, wave);
    ob.issue(t < kHalves * nk, to + OpA::kBytes, wave);
  };
  auto start = [&]() {
    i0 = next.i, j0 = next.j, which = next.which, split = next.split;
    const int kt0 = split * a.kt_split;
    nk = a.kt - kt0 < a.kt_split ? a.kt - kt0 : a.kt_split;
    if constexpr (kHalves == 2) {
      oa.seek(a.A[1], a.lda, i0, a.M, kt0);
      ob.seek(a.B[1], a.ldb, j0, a.N, kt0);
      second_a = oa.base, second_b = ob.base;
    }
    oa.seek(a.A[0], a.lda, i0, a.M, kt0);
    ob.seek(a.B[TRB ? which : 0], a.ldb, j0, a.N, kt0);
    issue_last(0);
    if constexpr (kHalves == 2) {
      const uint64_t first_a = oa.base, first_b = ob.base;
      oa.base = second_a, ob.base = second_b;
      issue_last(1);
      oa.base = first_a, ob.base = first_b;
    }
#pragma unroll
    for (int t = kHalves; t < (kAhead ? NB : NB - 1); ++t) issue(t, t);
  };

  place(wg);
  start();
  for (;;) {
    place(wg + step);
    const int nkt = kHalves * nk;
    f32x4 acc[FM][FNT];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int j = 0; j < FNT; ++j) acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr bool kBlocked = sizeof(E) == 4;
    f32x4 sum[kBlocked ? FM : 1][kBlocked ? FNT : 1] = {};
    auto close_block = [&](bool end) {
      if constexpr (kBlocked) {
        if (!end) return;
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int j = 0; j < FNT; ++j) {
            sum[f][j] += acc[f][j];
            acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
      }
    };
    auto read = [&](int buf, int kk, f32x4 (&fa)[FM], f32x4 (&fb)[FNT]) {
      const char* la = lds + buf * kBuf;
#pragma unroll
      for (int j = 0; j < FNT; ++j) fb[j] = OpB::read(la + OpA::kBytes, wn * TN, j, kk, lane);
      if constexpr (kLean) {
        unsigned at = a0;
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          const char* p = la + (at ^ (f * 32)) + kk * 32 * OpA::kRow;
          const xent::s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) xent::s16x4*)p);
          const xent::s16x4 hi =
              __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) xent::s16x4*)(p + 4 * OpA::kRow));
          fa[f] = __builtin_bit_cast(f32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
      } else {
#pragma unroll
        for (int f = 0; f < FM; ++f) fa[f] = OpA::read(la, wm * TM, f, kk, lane);
      }
    };
    auto multiply = [&](const f32x4 (&fa)[FM], const f32x4 (&fb)[FNT]) {
#pragma unroll
      for (int k = 0; k < Mma<E>::kSteps; ++k)
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int j = 0; j < FNT; ++j) acc[f][j] = Mma<E>::step(k, fa[f], fb[j], acc[f][j]);
    };
    if constexpr (kAhead) {
      f32x4 fa[2][FM], fb[2][FNT];
      ring_wait<(NB - 1) * kLoads>();
      read(0, 0, fa[0], fb[0]);
      for (int t0 = 0; t0 < nkt; t0 += NB) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (t0 + b >= nkt) break;
          read(b, 1, fa[1], fb[1]);
          multiply(fa[0], fb[0]);
          xent::interleave<kReads, kMmas>();
          ring_wait<(NB - 2) * kLoads>();
          if (NB > 2 || t0 + b + 2 < nkt) issue(t0 + b + NB, b);
          read((b + 1) % NB, 0, fa[0], fb[0]);
          multiply(fa[1], fb[1]);
          xent::interleave<kReads, kMmas>();
          close_block((t0 + b) % 4 == 3);
        }
      }
    } else {
      for (int t0 = 0; t0 < nkt; t0 += NB) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (t0 + b >= nkt) break;
          ring_wait<(NB - 2) * kLoads>();
          issue(t0 + b + NB - 1, (b + NB - 1) % NB);
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            f32x4 fa[FM], fb[FNT];
            read(b, kk, fa, fb);
            multiply(fa, fb);
          }
          close_block((t0 + b) % 4 == 3);
        }
      }
    }
    if constexpr (kBlocked) {
#pragma unroll
      for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int j = 0; j < FNT; ++j) acc[f][j] += sum[f][j];
    }
    const int ci = i0 + wm * TM, cj = j0 + wn * TN, out = which, part = split;
    wg += step;
    const bool more = wg < total;
    if (more) {
      ring_wait<0>();      // every wave's reads of the buffers are done
      start();
    }
    const int own = fresh_lane();
    const int g = own >> 4, r = own & 15;
#pragma unroll
    for (int j = 0; j < FNT; ++j) {
      const int row = cj + j * 16 + r;
      if (row >= a.N) continue;
#pragma unroll
      for (int f = 0; f < FM; ++f) {
        const int c = ci + f * 16 + g * 4;
        if (c >= a.M) continue;
        f32x4 v = acc[f][j];
        if (a.splits > 1) {
          store4(a.part + (((int64_t)part * kOuts + out) * a.N + row) * a.M + c, v);
        } else {
          E* p = static_cast<E*>(a.out[out]) + (int64_t)row * a.ldo + c;
          if (a.beta != 0.f) v += a.beta * load4(p);
          store4(p, v);
        }
      }
    }
    if (!more) break;
  }
  // no direct load may be in flight when the LDS is given to another tile or workgroup
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <class E, int BM, int BN, int WVM, int WVN, int NB, bool TRB, int WPE>
__global__ void __launch_bounds__(WVM * WVN * 64, WPE) gradient_kernel(GradArgs a) {
  constexpr int kOuts = TRB ? 2 : 1;
  __shared__ __align__(1024) char lds[lds_bytes(BM, BN, NB)];
  const int tiles = a.tm * a.tn * kOuts, full = tiles * a.splits - a.rest;
  auto tile = [&](int id) {
    GradPlace p;
    p.split = id / tiles;
    int im, in;
    xent::tile_of(id - p.split * tiles, a.tm, a.tn * kOuts, &im, &in);
    p.which = kOuts == 2 && in >= a.tn;
    p.i = im * BM, p.j = (in - p.which * a.tn) * BN;
    return p;
  };
  if ((int)blockIdx.x < full)
    gradient<E, BM, BN, WVM, WVN, NB, TRB>(a, lds, blockIdx.x, gridDim.x, full,
                                           [&](int at) { return tile(xent::share_of(at, full)); });
  // as in projection_kernel
  if constexpr (BN == 256) {
    const int halves = 2 * a.rest;
    if ((int)blockIdx.x >= halves) return;
    auto half = [&](int at) {
      const int id = xent::share_of(at, halves);
      GradPlace p = tile(full + id / 2);
      p.j += id % 2 * (BN / 2);
      return p;
    };
    if (half(blockIdx.x).j >= a.N) return;
    __syncthreads();
    gradient<E, BM, BN / 2, 2 * WVM, WVN / 2, kHalfNB, TRB>(a, lds, blockIdx.x, halves, halves, half);
  }
}

// G and U kept: dG and dU element by element, 16 bytes a thread (4096 x 11008 bf16 82 us, 70 behind the forward that kept them: 451 MB
// at 5.5 and 6.4 TB/s, part of it from the last-level cache).
struct PointArgs {
  const void* dH;
  const void* G;
  const void* U;
  void* dG;
  void* dU;
  int64_t lddh, ldg, lddg;
  int64_t first, items;   // pieces of 16 bytes
  int pieces;             // of a row
};

template <class E, int FN>
__global__ void __launch_bounds__(256) point_kernel(PointArgs a) {
  constexpr int W = 16 / (int)sizeof(E);
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= a.items) return;
  const int64_t item = a.first + at;
  const int64_t t = item <= 0xffffffffll ? (int64_t)((unsigned)item / (unsigned)a.pieces) : item / a.pieces;
  const int c = (int)(item - t * a.pieces) * W;
  float g[W], u[W], x[W];
  typedef typename Kept<E>::Word Word;
  typedef typename Kept<E>::Raw Raw;
  const Word* pg = static_cast<const Word*>(a.G) + t * a.ldg + c;
  const Word* pu = static_cast<const Word*>(a.U) + t * a.ldg + c;
  const E* px = static_cast<const E*>(a.dH) + t * a.lddh + c;
  E* og = static_cast<E*>(a.dG) + t * a.lddg + c;
  E* ou = static_cast<E*>(a.dU) + t * a.lddg + c;
  const Raw rg = *reinterpret_cast<const Raw*>(pg), ru = *reinterpret_cast<const Raw*>(pu);
  load_run<W>(px, x);
#pragma unroll
  for (int i = 0; i < W; ++i) asm volatile("" : "+v"(x[i]));     // read with the words, not behind the question
  if (Kept<E>::infinite(rg, ru)) {
    // An infinite word stands for a value that is not known but large: f' is that of any such value, f zero below and infinite above,
    // and a factor of zero gives zero (rows that are masked by dH = 0 would otherwise reach dX and every weight's gradient as NaN).
    // Few pieces have one: element by element, from memory again.
#pragma unroll 1
    for (int i = 0; i < W; ++i) {
      const float gi = Kept<E>::any_value(pg[i]), ui = Kept<E>::any_value(pu[i]), xi = (float)px[i];
      const float2 f = gated<FN, sizeof(E) == 2>(__builtin_amdgcn_fmed3f(gi, -kSaturated, kSaturated));
      const bool none = xi == 0.f;
      og[i] = (E)(none || f.y == 0.f ? 0.f : xi * ui * f.y);
      ou[i] = (E)(none ? 0.f : xi * (gi > kSaturated ? gi : f.x));
    }
    return;
  }
  Kept<E>::get(rg, g);
  Kept<E>::get(ru, u);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float2 f = gated<FN, sizeof(E) == 2>(g[i]);
    g[i] = x[i] * u[i] * f.y;
    u[i] = x[i] * f.x;
  }
  store_run<W>(og, g);
  store_run<W>(ou, u);
}

// tile: xent::Tile, or the few-token kernel (ks waves) where ks > 0
hipError_t launch_projection(int bf16, int fn, int mode, int tile, int ks, const ProjArgs& a, hipStream_t s);
hipError_t launch_point(int bf16, int fn, const PointArgs& a, hipStream_t s);
hipError_t launch_gradient(int bf16, int trb, int tile, const GradArgs& a, hipStream_t s);

}  // namespace glu
}  // namespace ff
