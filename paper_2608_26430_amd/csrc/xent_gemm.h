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
// For logits the rows of A are dealt to the MFMA in an order that gives a lane 4 PF consecutive
// vocabulary entries over PF tiles.
#pragma once

#include "ff_internal.h"

namespace ff {
namespace xent {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

enum Mode {
  kStats = 0,     // logits: maximum and sum of exponentials (the target's left out) of each wave's columns, the target's logit
  kExp = 1,       // the same, and exp(z - maximum) to out
  kGrad = 2,      // logits: out = (softmax - onehot) weight from the saved log-sum-exp
  kOut = 3,       // out = beta out + product
  kPart = 4,      // fp32 partial sums of one share of k
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
  int ocols;
  float beta;
  float* part;            // [splits][N][M] fp32
  int part_add;           // 1: added to what is there (an earlier piece of the vocabulary)
  // logits
  float2* stats;          // [wave columns][N] (maximum, sum of exponentials)
  const int64_t* target;  // [N]
  int64_t v0;             // first vocabulary entry of A
  int64_t vocab;          // entries of the whole vocabulary
  float* zt;              // [N] the target's logit
  const float* lse;       // [N]
  const float* loss;      // [N] or NULL (kGrad: the target's value from it)
  const float* dloss;     // [N] or NULL
  float scale;
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

__device__ __forceinline__ u32x4 make_rsrc(uint64_t base, int64_t bytes) {
  const uint32_t n = bytes <= 0 ? 0u : (bytes > 0x7fffffffll ? 0x7fffffffu : (uint32_t)bytes);
  u32x4 r = {(unsigned)__builtin_amdgcn_readfirstlane((int)(uint32_t)base),
             (unsigned)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
             (unsigned)__builtin_amdgcn_readfirstlane((int)n), 0x00020000u};
  return r;
}

// One operand's tile of BX along i (or j) and 128 bytes of k.  PF > 0: rows in the order of 4 PF consecutive
// entries per lane (K-major operands only).
template <class E, int BX, int NW, bool TR, int PF>
struct Operand {
  static constexpr int kE = ElemTraits<E>::kSize;
  static constexpr int kPer = 16 / kE;            // elements of a 16-byte piece
  static constexpr int kK = 128 / kE;             // k of a tile
  static constexpr int kBytes = BX * 128;
  static constexpr int kLoads = kBytes / 1024 / NW;
  static constexpr int kRow = TR ? BX * kE : 128; // bytes of an LDS row
  static constexpr int kPieces = kRow / 16;
  static_assert(kBytes % (1024 * NW) == 0, "a whole number of loads per wave");

  uint64_t base;
  int64_t total;      // bytes from base to the operand's end
  int64_t step;       // bytes per k tile
  unsigned voff[kLoads];
  int kq[kLoads];     // first k of the lane's piece within the tile (K-major)

  static __device__ __forceinline__ int swizzle(int row) {
    if (!TR) {
      if (PF == 0) return row & 7;
      constexpr int lg = PF == 4 ? 4 : 3;
      return (row & 3) | (((row >> lg) & 1) << 2);
    }
    const int s = kE == 2 ? (((row & 3) << 1) ^ (((row >> 3) & 1) << 3)) : (((row >> 2) & 3) << 2);
    return s & (kPieces - 1);
  }

  // x0: first i (j) of the tile, X its extent, kt0: first k tile.  The memory of a row reaches to the next whole
  // piece (H and W by their widths, P by its zero padding).
  __device__ __forceinline__ void init(const void* p, int64_t ld, int x0, int X, int K, int kt0, int wave, int lane) {
    const char* b = static_cast<const char*>(p);
    X = (X + kPer - 1) / kPer * kPer;
    K = TR ? K : (K + kPer - 1) / kPer * kPer;
    if (TR) {
      step = (int64_t)kK * ld * kE;
      base = (uint64_t)(b + (int64_t)x0 * kE + kt0 * step);
      total = ((int64_t)(K - 1) * ld + X - x0) * kE - kt0 * step;
    } else {
      step = 128;
      base = (uint64_t)(b + (int64_t)x0 * ld * kE + kt0 * step);
      const int rows = X - x0 < BX ? X - x0 : BX;
      total = ((int64_t)(rows - 1) * ld + K) * kE - kt0 * step;
    }
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int byte = (wave * kLoads + q) * 1024 + lane * 16;
      const int row = byte / kRow, piece = (byte % kRow / 16) ^ swizzle(row);
      voff[q] = (unsigned)((int64_t)row * ld * kE) + piece * 16;
      kq[q] = piece * kPer;
    }
  }

  // k tile t (counted from init's) into the LDS buffer; left: k from that tile's start on
  __device__ __forceinline__ void issue(int t, int left, unsigned lds, int wave) const {
    const u32x4 r = make_rsrc(base + t * step, left > 0 ? total - t * step : 0);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      unsigned v = voff[q];
      if (!TR && left < kK) v = kq[q] < left ? v : kFar;
      load_lds(v, r, lds + (wave * kLoads + q) * 1024);
    }
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
__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 mma<__bf16>(f32x4 a, f32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// fp32: lane group g holds k = 4 g + s in element s, so that step s of the four covers k = s, s + 4, s + 8, s + 12
template <>
__device__ __forceinline__ f32x4 mma<float>(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[s], c, 0, 0, 0);
  return c;
}

template <class E>
__device__ __forceinline__ float exp_of(float x) {
  return sizeof(E) == 2 ? __expf(x) : expf(x);
}

__device__ __forceinline__ unsigned short bf16_bits(float x) {
  return __builtin_bit_cast(unsigned short, (__bf16)x);
}
__device__ __forceinline__ float bf16_value(unsigned short b) { return __builtin_bit_cast(float, (unsigned)b << 16); }

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

// Tile of a workgroup.  Workgroups go round the eight XCDs; each XCD takes a contiguous run of tiles, in groups of
// eight along j and then along i, so that the tiles that run at once on an XCD share their operands in its L2.
__device__ __forceinline__ void tile_of(int wg, int total, int tm, int tn, int* im, int* in) {
  const int xcd = wg & 7, idx = wg >> 3;
  const int per = total >> 3, rem = total & 7;
  const int id = xcd * per + (xcd < rem ? xcd : rem) + idx;
  const int group = 8 * tm;
  const int g = id / group, first = g * 8;
  const int w = tn - first < 8 ? tn - first : 8;
  const int in_group = id - g * group;
  *in = first + in_group % w;
  *im = in_group / w;
}

template <class E, int BM, int BN, int WVM, int WVN, int NB, bool TRA, bool TRB, int WPE>
__global__ void __launch_bounds__(WVM * WVN * 64, WPE) gemm_kernel(GemmArgs a) {
  constexpr int NW = WVM * WVN;
  constexpr int TM = BM / WVM, TN = BN / WVN;
  constexpr int FM = TM / 16, FN = TN / 16;
  constexpr int PF = TRA ? 0 : (FM < 4 ? FM : 4);
  typedef Operand<E, BM, NW, TRA, PF> OpA;
  typedef Operand<E, BN, NW, TRB, 0> OpB;
  constexpr int kBuf = OpA::kBytes + OpB::kBytes;
  constexpr int kLoads = OpA::kLoads + OpB::kLoads;
  constexpr int kK = OpA::kK;
  __shared__ __align__(1024) char lds[NB * kBuf];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WVM, wn = wave / WVM;
  const int tiles = a.tm * a.tn;
  const int split = blockIdx.x / tiles;
  int im, in;
  tile_of(blockIdx.x - split * tiles, tiles, a.tm, a.tn, &im, &in);
  const int kt0 = split * a.kt_split;
  const int nkt = a.kt - kt0 < a.kt_split ? a.kt - kt0 : a.kt_split;

  OpA oa;
  OpB ob;
  oa.init(a.A, a.lda, im * BM, a.M, a.K, kt0, wave, lane);
  ob.init(a.B, a.ldb, in * BN, a.N, a.K, kt0, wave, lane);
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int kleft = a.K - kt0 * kK;
  auto issue = [&](int t, int buf) {
    const int left = t < nkt ? kleft - t * kK : 0;
    oa.issue(t, left, lds0 + buf * kBuf, wave);
    ob.issue(t, left, lds0 + buf * kBuf + OpA::kBytes, wave);
  };

  f32x4 acc[FM][FN];
#pragma unroll
  for (int f = 0; f < FM; ++f)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int t = 0; t < NB - 1; ++t) issue(t, t);
  for (int t0 = 0; t0 < nkt; t0 += NB) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (t0 + b >= nkt) break;
      ring_wait<(NB - 2) * kLoads>();
      issue(t0 + b + NB - 1, (b + NB - 1) % NB);
      const char* la = lds + b * kBuf;
      const char* lb = la + OpA::kBytes;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        f32x4 fa[FM], fb[FN];
#pragma unroll
        for (int f = 0; f < FM; ++f) fa[f] = OpA::read(la, wm * TM, f, kk, lane);
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[j] = OpB::read(lb, wn * TN, j, kk, lane);
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[f][j] = mma<E>(fa[f], fb[j], acc[f][j]);
      }
    }
  }
  // no direct load may be in flight when the workgroup's LDS is given to another one
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  const int g = lane >> 4, r = lane & 15;
  const int i0 = im * BM + wm * TM, j0 = in * BN + wn * TN;
  // first of the four i of tile f that the lane holds
  auto col = [&](int f) {
    if (TRA) return i0 + f * 16 + g * 4;
    constexpr int P = PF ? PF : 1;
    return i0 + (f / P) * P * 16 + g * (P * 4) + (f % P) * 4;
  };
  if constexpr (TRA) {
    if (a.mode == kPart) {
      float* part = a.part + (int64_t)split * a.N * a.M;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int row = j0 + j * 16 + r;
        if (row >= a.N) continue;
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          const int c = col(f);
          if (c >= a.M) continue;
          float* p = part + (int64_t)row * a.M + c;
          f32x4 v = acc[f][j];
          if (a.part_add) v += load4(p);
          store4(p, v);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int row = j0 + j * 16 + r;
        if (row >= a.N) continue;
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          const int c = col(f);
          if (c >= a.M) continue;
          E* p = static_cast<E*>(a.out) + (int64_t)row * a.ldo + c;
          f32x4 v = acc[f][j];
          if (a.beta != 0.f) v += a.beta * load4(p);
          store4(p, v);
        }
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int row = j0 + j * 16 + r;
      const bool live = row < a.N;
      const int64_t tg = live ? a.target[row] : -1;
      const bool counted = tg >= 0 && tg < a.vocab;
      const int at = counted && tg >= a.v0 && tg - a.v0 < a.M ? (int)(tg - a.v0) : -1;
      E* out = static_cast<E*>(a.out) + (int64_t)row * a.ldo;
      if (a.mode == kGrad) {
        const float lse = live ? a.lse[row] : 0.f;
        const float own = at >= 0 && a.loss ? expm1f(-a.loss[row]) : 0.f;
        const float w = counted ? a.scale * (a.dloss ? a.dloss[row] : 1.f) : 0.f;
#pragma unroll
        for (int f = 0; f < FM; ++f) {
          const int c = col(f);
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float z = acc[f][j][i] - lse;
            const float p = c + i == at ? (a.loss ? own : expm1f(z)) : exp_of<E>(z);
            v[i] = counted && c + i < a.M ? p * w : 0.f;
          }
          if (live && c < a.ocols) store4(out + c, v);
        }
        continue;
      }
      float top = -INFINITY;
#pragma unroll
      for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = col(f) + i;
          if (c >= a.M) acc[f][j][i] = -INFINITY;
          if (c == at) a.zt[row] = acc[f][j][i];
          top = fmaxf(top, acc[f][j][i]);
        }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float ref = top == -INFINITY ? 0.f : top;    // columns of nothing: exp(-inf) = 0, not NaN
      float sum = 0.f;
#pragma unroll
      for (int f = 0; f < FM; ++f) {
        const int c = col(f);
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = exp_of<E>(acc[f][j][i] - ref);
          sum += c + i == at ? 0.f : v[i];
        }
        if (a.mode == kExp && live && c < a.ocols) store4(out + c, v);
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (g == 0 && live && i0 < a.M) a.stats[(int64_t)(i0 / TM) * a.N + row] = make_float2(top, sum);
    }
  }
}

// Tile sizes of the instances: large (256 x 256, wave 128 x 64), medium (128 x 128, wave 64 x 64), small (128 x 32,
// wave 32 x 32).
enum Tile { kLarge = 0, kMedium = 1, kSmall = 2 };
constexpr int tile_m(int t) { return t == kLarge ? 256 : 128; }
constexpr int tile_n(int t) { return t == kLarge ? 256 : (t == kMedium ? 128 : 32); }
// columns of one entry of the logits' statistics
constexpr int stat_cols(int t) { return t == kLarge ? 128 : (t == kMedium ? 64 : 32); }

// layout 0: logits, 1: dH, 2: dW
hipError_t launch_gemm(int layout, int bf16, int tile, const GemmArgs& a, hipStream_t s);

}  // namespace xent
}  // namespace ff
