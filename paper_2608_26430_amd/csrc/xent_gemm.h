// Matrix products of the head's loss (xent.hip), one kernel template for all of them.
//
// Every product has the form out[j][i] = sum_k A(i, k) B(j, k): i runs along the rows of memory of the
// result, j over its rows.
//   logits  z[t][v]  = sum_c W[v][c] H[t][c]      A = W, B = H, both stored along k
//   dH      dH[t][c] = sum_v W[v][c] P[t][v]      A = W stored along i, B = P stored along k
//   dW      dW[v][c] = sum_t H[t][c] P[t][v]      A = H, B = P, both stored along i / j
// An operand stored along k goes to LDS as rows of 128 bytes (64 bf16 or 32 fp32 values of one i) and
// is read with 16-byte reads; one stored along i goes there as rows of k, read with the transposing
// 16-bit read (bf16) or element by element (fp32).  Both kinds are XOR-swizzled in pieces of 16 bytes
// so that the lanes of a read fall on different banks; the swizzle is applied to the source address of
// the direct loads into LDS, whose destination is linear.
//
// A workgroup computes a BM x BN tile (BM along i), its waves as WVM x WVN; NB tiles of 128 bytes
// of k are in flight.  In a 16 x 16 MFMA the lane holds four consecutive i of one j, so that results are
// stored along the rows of memory and the softmax statistics of one token stay in one lane's registers.
// For bf16 logits the rows of A are dealt to the MFMA in an order that gives a lane eight consecutive
// vocabulary entries over two tiles (PF = 2), one store of 16 bytes; the four lanes of a token store 64 bytes.  kExp's
// results are stored as fp16 either way.
//
// Bound by the matrix units.  4096 tokens, 4096 wide, 32,000 entries, bf16 (1.07 TFLOP a product): dH 770 to 830 us,
// logits with P's stores 840 to 960 us, alternately run; a large library product reaches 1.44 to 1.49 PFLOP/s on this
// card, which is 745 and 720 us.  Matrix units busy 64 to 70% of the cycles, LDS reads 25%, no bank conflicts; what is
// left is the end of a tile (maximum, exponentials, 33 MB of P a round: 75 us of the logits) and the last round of tiles
// (32,000 x 4096: 2000 tiles of 256 x 256, 7.8 rounds).  fp32: 100 to 120 of the library's 154 TFLOP/s.
// With few tokens it is bound by reading W: 1 token, 32,000 x 4096: 42 us, 6.2 TB/s.
#pragma once

#include "ff_internal.h"
#include "xent_plan.h"
#include "xent_span.h"

namespace ff {
namespace xent {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

enum Mode {
  kStats = 0,     // logits: maximum and sum of exponentials of each wave's columns, the target left out, and its logit
  kExp = 1,       // the same, and exp(z - maximum) to out (bf16 activations: store8_half)
  kGrad = 2,      // logits: out = (softmax - onehot) dloss from the saved log-sum-exp
  kOut = 3,       // out = beta out + alpha product
  kPart = 4,      // alpha times fp32 partial sums of one share of k
};

struct GemmArgs {
  const void* A;
  const void* B;
  int64_t lda, ldb;       // elements
  int M, N, K;            // extents of i, j, k
  int tm, tn;             // tiles along i and j
  int kt;                 // k tiles in all
  int kt_split;           // k tiles of one split
  int splits;
  int mode;
  void* out;              // [N][ldo], written up to column ocols (columns past M as zero: P's padding)
  int64_t ldo;
  int64_t rest;           // kGrad: elements from a row of out to that of what its rounding left, 0: not kept
  int ocols;
  float beta;
  float* part;            // [splits][N][M] fp32
  int part_add;           // 1: added to what is there (an earlier piece of the vocabulary)
  // logits
  float2* stats;          // [wave columns][N] (maximum, sum of exponentials), the target left out
  const int64_t* target;  // [N]
  int64_t v0;             // first vocabulary entry of A
  int64_t vocab;          // entries of the whole vocabulary
  float* zt;              // [N] the target's logit
  const float* lse;       // [N]
  const float* loss;      // [N] or NULL (kGrad: the target's value from it)
  const float* dloss;     // [N] or NULL
  float alpha;            // kOut, kPart: factor of the product
};

template <class E>
struct ElemTraits;
template <>
struct ElemTraits<__bf16> {
  static constexpr int kSize = 2;
};
template <>
struct ElemTraits<float> {
  static constexpr int kSize = 4;
};

constexpr unsigned kFar = 0x80000000u;   // a byte offset past every range: the load gives zero

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 bytes per lane from rsrc + voff to LDS address lds + 16 lane (zero where voff is out of range).  The compiler
// does not see the write: the main loop waits for it by count (ring_wait).
__device__ __forceinline__ void load_lds(unsigned voff, u32x4 rsrc, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds)
               : "m0");
}
#pragma clang diagnostic pop

// All of this wave's direct loads but the last N have landed and its LDS reads are done; then the workgroup's barrier.
template <int N>
__device__ __forceinline__ void ring_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(N) : "memory");
}

__device__ __forceinline__ u32x4 make_rsrc(uint64_t base, unsigned bytes) {
  u32x4 r = {(unsigned)__builtin_amdgcn_readfirstlane((int)(uint32_t)base),
             (unsigned)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
             (unsigned)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
  return r;
}

// One operand's tile of BX along i (or j) and 128 bytes of k.  PF > 0: rows in the order of 4 PF consecutive
// entries per lane (K-major operands only).
template <class E, int BX, int NW, bool TR, int PF>
struct Operand {
  static constexpr int kE = ElemTraits<E>::kSize;
  static constexpr int kPer = 16 / kE;            // elements of a 16-byte piece
  static constexpr int kK = kTileBytes / kE;      // k of a tile
  static constexpr int kBytes = BX * kTileBytes;
  static constexpr int kLoads = kBytes / 1024 / NW;
  static constexpr int kRow = TR ? BX * kE : 128; // bytes of an LDS row
  static constexpr int kPieces = kRow / 16;
  static constexpr int kReads = !TR ? 1 : (kE == 2 ? 2 : 4);   // LDS reads of a fragment
  static_assert(kBytes % (1024 * NW) == 0, "a whole number of loads per wave");

  uint64_t base;      // next k tile
  uint64_t step;      // bytes per k tile
  unsigned records;   // bytes of a whole k tile that may be read
  unsigned voff[kLoads];

  static __device__ __forceinline__ int swizzle(int row) {
    if (!TR) {
      if (PF == 0) return row & 7;
      return (row & 3) | (((row >> 3) & 1) << 2);
    }
    if (kE == 2 && kPieces == 4) return row & 2;
    const int s = kE == 2 ? (((row & 3) << 1) ^ (((row >> 3) & 1) << 3)) : (((row >> 2) & 3) << 2);
    return s & (kPieces - 1);
  }

  __device__ __forceinline__ void init(int64_t ld, int wave, int lane) {
    step = (uint64_t)k_step(!TR, kE, ld);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int byte = (wave * kLoads + q) * 1024 + lane * 16;
      const int row = byte / kRow, piece = (byte % kRow / 16) ^ swizzle(row);
      voff[q] = (unsigned)((int64_t)row * ld * kE) + piece * 16;
    }
  }

  // x0: first i (j) of the tile, X its extent, kt0: first k tile
  __device__ __forceinline__ void seek(const void* p, int64_t ld, int x0, int X, int kt0) {
    const Span s = span_of(!TR, kE, BX, ld, x0, X, kt0, kK);
    base = (uint64_t)((const char*)p + s.first);
    records = s.bytes;
  }

  // The last k tile of the tile at x0, `tile` steps on, of which `left` of k remain: zero beyond them.
  __device__ __forceinline__ void issue_last(int tile, int left, int64_t ld, int x0, int X, unsigned lds, int wave,
                                             int lane) const {
    const int pieces = (left + kPer - 1) / kPer;
    const unsigned n = span_of(!TR, kE, BX, ld, x0, X, 0, left).bytes;
    asm volatile("" : "+v"(lane));   // places made here, not kept (and spilled) from one tile to the next
    const u32x4 r = make_rsrc(base + tile * step, n);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      unsigned v = voff[q];
      if (!TR) {
        const int byte = (wave * kLoads + q) * 1024 + lane * 16;
        v = ((byte % kRow / 16) ^ swizzle(byte / kRow)) < pieces ? v : kFar;
      }
      load_lds(v, r, lds + (wave * kLoads + q) * 1024);
    }
  }

  // The next whole k tile (nothing, as zeros, unless `more`).
  __device__ __forceinline__ void issue(bool more, unsigned lds, int wave) {
    const u32x4 r = make_rsrc(base, more ? records : 0u);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) load_lds(voff[q], r, lds + (wave * kLoads + q) * 1024);
    base += step;
  }

  // Fragment of 16 i starting at x (a multiple of 16; PF > 0: tile f of the wave's part at x) of half kk of the tile.
  typedef __attribute__((ext_vector_type(4))) float Frag;
  static __device__ __forceinline__ Frag read(const char* lds, int x, int f, int kk, int lane) {
    const int g = lane >> 4, r = lane & 15;
    if (!TR) {
      int row;
      if (PF == 0) row = x + f * 16 + r;
      else row = x + (f / (PF ? PF : 1)) * PF * 16 + (r >> 2) * PF * 4 + (f % (PF ? PF : 1)) * 4 + (r & 3);
      return *reinterpret_cast<const Frag*>(lds + row * 128 + (((kk * 4 + g) ^ (r & 7)) << 4));
    }
    if (kE == 2) {
      // rows k = 32 kk + 8 g + 4 h + j, j = r / 4; the lane gives 4 columns, and gets column r of 4 rows
      const int j = r >> 2, cb = (x + f * 16) * 2 + (r & 3) * 8;
      const int k = kk * 32 + g * 8 + j;
      const char* a = lds + k * kRow + ((((cb >> 4) ^ swizzle(k)) << 4) | (cb & 15));
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(a));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(a + 4 * kRow));
      return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    const int k = kk * 16 + g * 4, cb = (x + f * 16 + r) * 4;
    const char* a = lds + k * kRow + ((((cb >> 4) ^ swizzle(k)) << 4) | (cb & 15));
    Frag v;
#pragma unroll
    for (int s = 0; s < 4; ++s) v[s] = *reinterpret_cast<const float*>(a + s * kRow);
    return v;
  }
};

template <class E>
struct Mma;
template <>
struct Mma<__bf16> {
  static constexpr int kSteps = 1;
  static __device__ __forceinline__ f32x4 step(int, f32x4 a, f32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
  }
};
// fp32: lane group g holds k = 4 g + s in element s, so that step s of the four covers k = s, s + 4, s + 8, s + 12
template <>
struct Mma<float> {
  static constexpr int kSteps = 4;
  static __device__ __forceinline__ f32x4 step(int s, f32x4 a, f32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[s], c, 0, 0, 0);
  }
};

// Asks the scheduler to spread READS LDS reads evenly over the MMAS multiplications beside them.
template <int READS, int MMAS, int I = 0>
__device__ __forceinline__ void interleave() {
  if constexpr (I < READS) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                                         // one LDS read
    __builtin_amdgcn_sched_group_barrier(0x008, MMAS * (I + 1) / READS - MMAS * I / READS, 0);   // its share of MFMA
    interleave<READS, MMAS, I + 1>();
  }
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ unsigned short bf16_bits(float x) {
  return __builtin_bit_cast(unsigned short, (__bf16)x);
}
__device__ __forceinline__ float bf16_value(unsigned short b) { return __builtin_bit_cast(float, (unsigned)b << 16); }

// What rounding to bf16 leaves of v.
__device__ __forceinline__ f32x4 rounding_of(f32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] -= bf16_value(bf16_bits(v[i]));
  return v;
}
// eight consecutive results
__device__ __forceinline__ void store8(__bf16* p, f32x4 v, f32x4 w) {
  const u32x4 x = {(unsigned)bf16_bits(v[0]) | (unsigned)bf16_bits(v[1]) << 16,
                   (unsigned)bf16_bits(v[2]) | (unsigned)bf16_bits(v[3]) << 16,
                   (unsigned)bf16_bits(w[0]) | (unsigned)bf16_bits(w[1]) << 16,
                   (unsigned)bf16_bits(w[2]) | (unsigned)bf16_bits(w[3]) << 16};
  *reinterpret_cast<u32x4*>(p) = x;
}
// and eight exponentials of kExp, times 2^kExpShift, in fp16: its 11 bits leave the rounding of P to bf16 nearly the only
// one, and the shift keeps them down to 2^-29 of the columns' maximum (the target, which may be far above, left out)
constexpr int kExpShift = 15;
__device__ __forceinline__ void store8_half(void* p, f32x4 v, f32x4 w) {
  typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
  const f16x8 x = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3],
                   (_Float16)w[0], (_Float16)w[1], (_Float16)w[2], (_Float16)w[3]};
  *reinterpret_cast<f16x8*>(p) = x;
}
__device__ __forceinline__ void store4_half(void* p, f32x4 v) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  const f16x4 x = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
  *reinterpret_cast<f16x4*>(p) = x;
}
// four consecutive results (the address is a multiple of four elements)
__device__ __forceinline__ void store4(__bf16* p, f32x4 v) {
  u32x2 w = {(unsigned)bf16_bits(v[0]) | (unsigned)bf16_bits(v[1]) << 16,
             (unsigned)bf16_bits(v[2]) | (unsigned)bf16_bits(v[3]) << 16};
  *reinterpret_cast<u32x2*>(p) = w;
}
__device__ __forceinline__ void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ f32x4 load4(const __bf16* p) {
  const u32x2 w = *reinterpret_cast<const u32x2*>(p);
  f32x4 v = {bf16_value(w[0] & 0xffff), bf16_value(w[0] >> 16), bf16_value(w[1] & 0xffff), bf16_value(w[1] >> 16)};
  return v;
}
__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// The results of a wave's tile: FM x FN tiles of 16 x 16 from (i0, j0).
template <class E, int FM, int FN, int TM, int PF, bool TRA>
__device__ __forceinline__ void finish(const GemmArgs& a, f32x4 (&acc)[FM][FN], const int (&target)[FN], int i0, int j0,
                                       int split, int lane) {
  const int g = lane >> 4, r = lane & 15;
  // first of the four i of tile f that the lane holds
  auto col = [&](int f) {
    if (TRA) return i0 + f * 16 + g * 4;
    constexpr int P = PF ? PF : 1;
    return i0 + (f / P) * P * 16 + g * (P * 4) + (f % P) * 4;
  };
  if constexpr (TRA) {
    const bool partial = a.mode == kPart;
    float* part = partial ? a.part + (int64_t)split * a.N * a.M : nullptr;
    const float alpha = a.alpha;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int row = j0 + j * 16 + r;
      if (row >= a.N) continue;
#pragma unroll
      for (int f = 0; f < FM; ++f) {
        const int c = col(f);
        if (c >= a.M) continue;
        f32x4 v = acc[f][j] * alpha;
        if (partial) {
          float* p = part + (int64_t)row * a.M + c;
          if (a.part_add) v += load4(p);
          store4(p, v);
        } else {
          E* p = static_cast<E*>(a.out) + (int64_t)row * a.ldo + c;
          if (a.beta != 0.f) v += a.beta * load4(p);
          store4(p, v);
        }
      }
    }
  } else {
    constexpr float kLog2e = 1.4426950408889634f;
    // tile f's results of a token: the two tiles of a pair go out together
    f32x4 first;
    auto put = [&](E* out, int f, f32x4 v, bool live) {
      if constexpr (PF == 2) {
        if (f % 2 == 0) {
          first = v;
        } else if (live && col(f - 1) < a.ocols) {
          if (a.mode == kExp) {
            store8_half(out + col(f - 1), first, v);
          } else {
            store8(out + col(f - 1), first, v);
            if (a.rest) store8(out + a.rest + col(f - 1), rounding_of(first), rounding_of(v));
          }
        }
      } else if (live && col(f) < a.ocols) {
        if (sizeof(E) == 2 && a.mode == kExp) {
          store4_half(out + col(f), v);
        } else {
          store4(out + col(f), v);
          if (sizeof(E) == 2 && a.rest) store4(out + a.rest + col(f), rounding_of(v));
        }
      }
    };
    const bool edge = i0 + TM > a.M;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int row = j0 + j * 16 + r;
      const bool live = row < a.N;
      const bool counted = target[j] != -1;
      const int at = target[j] >= i0 && target[j] < i0 + TM ? target[j] : -1;
      const bool hit = __any(at >= 0);      // a token of the wave has its target in these columns
      E* out = static_cast<E*>(a.out) + (int64_t)row * a.ldo;
      if (a.mode == kGrad) {
        const float lse = live ? a.lse[row] : 0.f;
        const float w = counted ? (a.dloss ? a.dloss[row] : 1.f) : 0.f;
        const float own = at >= 0 && a.loss ? expm1f(-a.loss[row]) : 0.f;
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          const int c = col(f);
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = sizeof(E) == 2 ? exp2_fast((acc[f][j][i] - lse) * kLog2e) : expf(acc[f][j][i] - lse);
            v[i] = counted ? p * w : 0.f;
          }
          if (hit) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (c + i == at) v[i] = (a.loss ? own : expm1f(acc[f][j][i] - lse)) * w;
          }
          if (edge) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = c + i < a.M ? v[i] : 0.f;
          }
          put(out, f, v, live);
        }
        continue;
      }
      if (edge) {
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (col(f) + i >= a.M) acc[f][j][i] = -INFINITY;
      }
      // the target stays out of the maximum as well as of the sum: the others' exponentials would leave fp16's range
      // where its logit is far above theirs
      if (hit) {
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (col(f) + i == at) {
              a.zt[row] = acc[f][j][i];
              acc[f][j][i] = -INFINITY;
            }
      }
      float top = -INFINITY;
#pragma unroll
      for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, acc[f][j][i]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float ref = top == -INFINITY ? 0.f : top;    // columns of nothing: exp(-inf) = 0, not NaN
      // bf16: all exponentials of this mode carry the shift of their storage
      float sum = 0.f;
#pragma unroll
      for (int f = 0; f < FM; ++f) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = sizeof(E) == 2 ? exp2_fast(fmaf(acc[f][j][i] - ref, kLog2e, (float)kExpShift)) : expf(acc[f][j][i] - ref);
        if (a.mode == kExp) put(out, f, v, live);
        sum += (v[0] + v[1]) + (v[2] + v[3]);
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (sizeof(E) == 2) sum *= 1.f / (1 << kExpShift);
      if (g == 0 && live && i0 < a.M) a.stats[(int64_t)(i0 / TM) * a.N + row] = make_float2(top, sum);
    }
  }
}

template <class E, int BM, int BN, int WVM, int WVN, int NB, bool TRA, bool TRB, int WPE>
__global__ void __launch_bounds__(WVM * WVN * 64, WPE) gemm_kernel(GemmArgs a) {
  constexpr int NW = WVM * WVN;
  constexpr int TM = BM / WVM, TN = BN / WVN;
  constexpr int FM = TM / 16, FN = TN / 16;
  constexpr int PF = TRA || sizeof(E) == 4 || FM < 2 ? 0 : 2;
  typedef Operand<E, BM, NW, TRA, PF> OpA;
  typedef Operand<E, BN, NW, TRB, 0> OpB;
  constexpr int kBuf = OpA::kBytes + OpB::kBytes;
  constexpr int kLoads = OpA::kLoads + OpB::kLoads;
  constexpr int kK = OpA::kK;
  constexpr int kReads = FM * OpA::kReads + FN * OpB::kReads;      // LDS reads and MFMA of half a tile
  constexpr int kMmas = FM * FN * (sizeof(E) == 2 ? 1 : 4);
  __shared__ __align__(1024) char lds[NB * kBuf];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WVM, wn = wave / WVM;
  const int tiles = a.tm * a.tn, total = tiles * a.splits;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  OpA oa;
  OpB ob;
  oa.init(a.lda, wave, lane);
  ob.init(a.ldb, wave, lane);
  int i0, j0, split, nkt;      // the tile whose operands are being read
  int i_next, j_next, split_next;
  auto place = [&](int wg) {   // of a workgroup's next tile: divisions, done while its loads are awaited
    const int id = share_of(wg, total);
    split_next = id / tiles;
    int im, in;
    tile_of(id - split_next * tiles, a.tm, a.tn, &im, &in);
    i_next = im * BM, j_next = in * BN;
  };
  auto seek = [&]() {
    split = split_next, i0 = i_next, j0 = j_next;
    const int kt0 = split * a.kt_split;
    nkt = a.kt - kt0 < a.kt_split ? a.kt - kt0 : a.kt_split;
    oa.seek(a.A, a.lda, i0, a.M, kt0);
    ob.seek(a.B, a.ldb, j0, a.N, kt0);
  };
  // k is walked with its last tile first, so that only the first loads look at its end
  auto issue_last = [&]() {
    if (nkt <= 0) return;
    const int last = a.K - (split * a.kt_split + nkt - 1) * kK;
    oa.issue_last(nkt - 1, last < kK ? last : kK, a.lda, i0, a.M, lds0, wave, lane);
    ob.issue_last(nkt - 1, last < kK ? last : kK, a.ldb, j0, a.N, lds0 + OpA::kBytes, wave, lane);
  };
  auto issue = [&](int t, int buf) {
    oa.issue(t < nkt, lds0 + buf * kBuf, wave);
    ob.issue(t < nkt, lds0 + buf * kBuf + OpA::kBytes, wave);
  };
  int64_t raw[FN];             // targets of that tile's tokens
  auto start = [&]() {
    seek();
    if constexpr (!TRA) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int row = j0 + wn * TN + j * 16 + (lane & 15);
        raw[j] = row < a.N ? a.target[row] : -1;
      }
    }
    issue_last();
#pragma unroll
    for (int t = 1; t < (NB == 2 ? 2 : NB - 1); ++t) issue(t, t);
  };

  place(blockIdx.x);
  start();
  for (int wg = blockIdx.x;;) {
  place(wg + gridDim.x);
  // the token's target as a column of A (-1: none, -2: in another piece of the vocabulary)
  int target[FN] = {};
  if constexpr (!TRA) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
      target[j] = raw[j] < 0 || raw[j] >= a.vocab ? -1 : (raw[j] >= a.v0 && raw[j] - a.v0 < a.M ? (int)(raw[j] - a.v0) : -2);
  }
  f32x4 acc[FM][FN];
#pragma unroll
  for (int f = 0; f < FM; ++f)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // fp32 (128 k at a time), and the logits of few tokens (one k tile): sums of a block, then their sum, so that rounding
  // grows with the length of both, not of k (fp32, 1024 wide, 44 entries: the loss's error 1.2e-6 -> 3.4e-7, costs 3%;
  // bf16, 1 to 64 tokens: the mean error 3.5e-7 -> 1.6e-7 with the exponentials' difference taken before it is scaled, and
  // no cost)
  constexpr bool kFew = NB == 4 && !TRA, kBlocked = sizeof(E) == 4 || kFew;
  f32x4 total_acc[kBlocked ? FM : 1][kBlocked ? FN : 1] = {};
  auto close_block = [&](bool end) {
    if constexpr (kBlocked) {
      if (!end) return;
#pragma unroll
      for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          total_acc[f][j] += acc[f][j];
          acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
  };
  auto read = [&](int buf, int kk, f32x4 (&fa)[FM], f32x4 (&fb)[FN]) {
    const char* la = lds + buf * kBuf;
    const char* lb = la + OpA::kBytes;
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[j] = OpB::read(lb, wn * TN, j, kk, lane);
#pragma unroll
    for (int f = 0; f < FM; ++f) fa[f] = OpA::read(la, wm * TM, f, kk, lane);
  };
  auto multiply = [&](const f32x4 (&fa)[FM], const f32x4 (&fb)[FN]) {
    // fp32: a step of k over all tiles, so that no product waits for the one before
#pragma unroll
    for (int k = 0; k < Mma<E>::kSteps; ++k)
#pragma unroll
      for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[f][j] = Mma<E>::step(k, fa[f], fb[j], acc[f][j]);
  };

  if constexpr (NB == 2) {
    // Two buffers.  The fragments of a half tile are read while the other half is multiplied; in the middle of tile
    // t every wave has read all of it, so that its buffer takes tile t + 2.
    f32x4 fa[2][FM], fb[2][FN];
    ring_wait<kLoads>();
    read(0, 0, fa[0], fb[0]);
    for (int t0 = 0; t0 < nkt; t0 += 2) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (t0 + b >= nkt) break;
        read(b, 1, fa[1], fb[1]);
        multiply(fa[0], fb[0]);
        interleave<kReads, kMmas>();
        ring_wait<0>();
        if (t0 + b + 2 < nkt) issue(t0 + b + 2, b);
        read(1 - b, 0, fa[0], fb[0]);
        multiply(fa[1], fb[1]);
        interleave<kReads, kMmas>();
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
          f32x4 fa[FM], fb[FN];
          read(b, kk, fa, fb);
          multiply(fa, fb);
        }
        close_block(kFew || (t0 + b) % 4 == 3);
      }
    }
  }
  if constexpr (kBlocked) {
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[f][j] += total_acc[f][j];
  }
  // this tile's place, and the next one's first loads under the results' arithmetic and stores
  const int wi0 = i0 + wm * TM, wj0 = j0 + wn * TN, wsplit = split;
  wg += gridDim.x;
  const bool more = wg < total;
  if (more) {
    ring_wait<0>();      // every wave's reads of the buffers are done
    start();
  }
  finish<E, FM, FN, TM, PF, TRA>(a, acc, target, wi0, wj0, wsplit, lane);
  if (!more) break;
  }
  // no direct load may be in flight when the workgroup's LDS is given to another one
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// layout 0: logits, 1: dH, 2: dW
hipError_t launch_gemm(int layout, int bf16, int tile, const GemmArgs& a, hipStream_t s);

}  // namespace xent
}  // namespace ff
