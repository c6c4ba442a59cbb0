// Dropout from a counter-based generator: the mask is a function of (seed, offset, row, column, width), computed where
// it is needed and never stored; the backward pass is the same call on the gradient.
//
//   y = [r +] m x / (1 - p'),   m = 0 for a share p' = D / 65536 of the elements, D = round(65536 p).
// A row is cut into blocks of eight elements.  Block b = t ceil(n / 8) + i / 8 draws four 32-bit words of Philox 4x32
// with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), counter
// (b, offset), key seed; element j of the block takes 16 bits, of word j / 2 the low (j even) or high half, and is
// dropped where they are below D.  16 bits an element halve the generator's 20 wide products per word set against 32
// bits; the kept elements are scaled by the share that is kept in fact, so that the expectation is exact.
// Bound by memory: 4 bytes (bf16, no residual; with one 6) an element; 8192 x 28,672 with a residual 280 us, 5.0 TB/s,
// where a large copy has 5.2.  A thread takes one block at a time of a grid-wide stride, row and column carried along
// by additions; a launch of 64 x 256 is 3 us.
#include <cmath>

#include "ff_internal.h"

namespace ff {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes on any element: rows of odd widths start anywhere, and the memory unit takes such pieces whole
typedef u32x4 Loose __attribute__((aligned(2)));

struct DropArgs {
  const void* X;
  const void* R;
  void* Y;
  int64_t ldx, ldr, ldy;
  int64_t T, blocks;       // blocks = T ceil(n / 8)
  int n, nb;               // nb = ceil(n / 8)
  int64_t seed_lo_hi;      // the key
  uint64_t offset;
  const uint64_t* offset_dev;
  unsigned drop;           // D
  float scale;
};

__device__ __forceinline__ u32x4 philox(uint64_t block, uint64_t offset, uint64_t seed) {
  unsigned c0 = (unsigned)block, c1 = (unsigned)(block >> 32), c2 = (unsigned)offset, c3 = (unsigned)(offset >> 32);
  unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
    c1 = (unsigned)b;
    c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
    c3 = (unsigned)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  u32x4 w = {c0, c1, c2, c3};
  return w;
}

template <class E>
__device__ __forceinline__ void get8(const E* p, float* v);
template <>
__device__ __forceinline__ void get8<__bf16>(const __bf16* p, float* v) {
  const u32x4 w = *reinterpret_cast<const Loose*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void get8<float>(const float* p, float* v) {
  const u32x4 a = reinterpret_cast<const Loose*>(p)[0], b = reinterpret_cast<const Loose*>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned x = a[i], y = b[i];
    v[i] = __builtin_bit_cast(float, x), v[4 + i] = __builtin_bit_cast(float, y);
  }
}
template <class E>
__device__ __forceinline__ void put8(E* p, const float* v);
template <>
__device__ __forceinline__ void put8<__bf16>(__bf16* p, const float* v) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (unsigned)__builtin_bit_cast(unsigned short, (__bf16)v[2 * i]) |
           (unsigned)__builtin_bit_cast(unsigned short, (__bf16)v[2 * i + 1]) << 16;
  *reinterpret_cast<Loose*>(p) = w;
}
template <>
__device__ __forceinline__ void put8<float>(float* p, const float* v) {
  u32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = __builtin_bit_cast(unsigned, v[i]), b[i] = __builtin_bit_cast(unsigned, v[4 + i]);
  reinterpret_cast<Loose*>(p)[0] = a;
  reinterpret_cast<Loose*>(p)[1] = b;
}

template <class E, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(DropArgs a) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (b >= a.blocks) return;
  int64_t t = b / a.nb;
  int c = (int)(b - t * a.nb);
  const int64_t dt = stride / a.nb;
  const int dc = (int)(stride - dt * a.nb);
  const uint64_t offset = a.offset + (a.offset_dev ? *a.offset_dev : 0);
  for (; b < a.blocks; b += stride) {
    const E* x = static_cast<const E*>(a.X) + t * a.ldx + c * 8;
    const E* r = RES ? static_cast<const E*>(a.R) + t * a.ldr + c * 8 : nullptr;
    E* y = static_cast<E*>(a.Y) + t * a.ldy + c * 8;
    const int left = a.n - c * 8;
    float v[8], q[8];
    if (left >= 8) {
      get8<E>(x, v);
      if (RES) get8<E>(r, q);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = i < left ? (float)x[i] : 0.f;
        if (RES) q[i] = i < left ? (float)r[i] : 0.f;
      }
    }
    const u32x4 w = philox((uint64_t)b, offset, (uint64_t)a.seed_lo_hi);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned u = (i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
      v[i] = u >= a.drop ? v[i] * a.scale : 0.f;     // a dropped NaN or infinity is zero
      if (RES) v[i] += q[i];
    }
    if (left >= 8) {
      put8<E>(y, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) y[i] = (E)v[i];
    }
    t += dt;
    c += dc;
    if (c >= a.nb) c -= a.nb, ++t;
  }
}

template <class E>
void launch(const DropArgs& a, hipStream_t s) {
  int64_t grid = (a.blocks + 255) / 256;
  if (grid > 256 * 32) grid = 256 * 32;
  const dim3 g((unsigned)grid), t(256);
  if (a.R) hipLaunchKernelGGL((dropout_kernel<E, true>), g, t, 0, s, a);
  else hipLaunchKernelGGL((dropout_kernel<E, false>), g, t, 0, s, a);
}

ff_status check_rows(const char* name, const void* p, int64_t ld, int64_t n, int esz) {
  if (!p) return fail(FF_EINVAL, "%s is NULL", name);
  if (ld < n) return fail(FF_EINVAL, "leading dimension of %s (%lld) < %lld", name, (long long)ld, (long long)n);
  if ((uintptr_t)p % esz) return fail(FF_EINVAL, "%s is misaligned", name);
  return FF_OK;
}

}  // namespace
}  // namespace ff

extern "C" ff_status ff_dropout(int64_t T, int64_t n, int act, const void* X, int64_t ldx, double p, uint64_t seed,
                                uint64_t offset, const uint64_t* offset_dev, const void* R, int64_t ldr, void* Y,
                                int64_t ldy, void* stream) {
  ff::clear_error();
  if (act != FF_F32 && act != FF_BF16) return ff::fail(FF_EINVAL, "unknown activation dtype %d", act);
  if (T < 0 || T > ((int64_t)1 << 40) || n < 1 || n > ((int64_t)1 << 28))
    return ff::fail(FF_EINVAL, "T=%lld or n=%lld out of range", (long long)T, (long long)n);
  // no card holds so many; the blocks' numbers and places stay within 64 bits
  const int64_t nb = (n + 7) / 8;
  if (T > ((int64_t)1 << 44) / nb) return ff::fail(FF_EINVAL, "T=%lld rows of n=%lld: too many", (long long)T, (long long)n);
  if (!(p >= 0.0 && p <= 1.0)) return ff::fail(FF_EINVAL, "p=%g outside [0, 1]", p);
  if (T == 0) return FF_OK;
  const int esz = act == FF_BF16 ? 2 : 4;
  ff_status st;
  if ((st = ff::check_rows("X", X, ldx, n, esz)) != FF_OK) return st;
  if ((st = ff::check_rows("Y", Y, ldy, n, esz)) != FF_OK) return st;
  if (R && (st = ff::check_rows("R", R, ldr, n, esz)) != FF_OK) return st;
  if ((uintptr_t)offset_dev % 8) return ff::fail(FF_EINVAL, "offset_dev is not 8-byte aligned");
  const unsigned drop = p < 1.0 ? (unsigned)std::fmin(std::nearbyint(p * 65536.0), 65535.0) : 65536u;
  ff::DropArgs a{X, R, Y, ldx, R ? ldr : 0, ldy, T, T * nb, (int)n, (int)nb, (int64_t)seed, offset, offset_dev, drop,
                 drop < 65536u ? 65536.f / (float)(65536u - drop) : 0.f};
  if (act == FF_BF16) ff::launch<__bf16>(a, (hipStream_t)stream);
  else ff::launch<float>(a, (hipStream_t)stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FF_OK : ff::fail(FF_EDEVICE, "dropout launch: %s", hipGetErrorString(e));
}
