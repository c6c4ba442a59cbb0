// One AdamW step over a set of tensors of any lengths, moments in fp32 or in 8 bits.
//
//   c <- c (1 - lr wd);  g <- s g;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   c <- c - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// A table made with the set deals chunks of 4096 elements of the tensors to workgroups; the gradients' addresses, which may
// differ from step to step, travel as kernel arguments, so that a step copies nothing to the device and one launch serves
// kGrads tensors.
//
// Moments of 8 bits: blocks of 256 elements of a tensor share a unit 2^k; code a stands for a units below 16 and
// (8 + a % 8) 2^(a / 8 - 1) from there on: four significant bits.  m has a sign and 7 bits of code (up to 15 x 2^14 units), v
// 8 bits (up to 15 x 2^30, which is as far for its root).  k is the least that holds the block's largest value.  The step uses
// the new moments before they are rounded.  They are rounded up or down at random in proportion to what is left: to
// nearest, v would stand still wherever (1 - b2) g^2 stays below half a step, 6% of it.  A random fraction is (16 bits + 1/2) /
// 65536, the bits from Philox 4x32-10 of (element / 4, step, tensor): a function of the element alone, whatever the
// launch.  The moments and their place between codes are computed in fp64: in fp32 one element in a million would fall on the other
// side.
//
// With fp32 moments bound by memory: 28 bytes an element with fp32 gradients.  Measured: three tensors of 1000 and 256 elements 2.4 us; 289
// of 7000 to 20,000 and 4096, 92 MB, 16.7 us (5.5 TB/s, part of it from the last-level cache); three of 45, 27 and 38 million elements
// with bf16 gradients and copies, 28 bytes an element, 587 us (3.09 GB, 5.25 TB/s).
// In 8 bits, with bf16 gradients and copies, 16 bytes and 146 vector instructions an element: the same three tensors 412 to 475 us (1.76 GB,
// 3.7 to 4.3 TB/s; 246,000 vector instructions on each SIMD in 0.9 million cycles), their moments read in 155 to 162 (0.66 GB, 4.1 to
// 4.3 TB/s).
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <vector>

#include "ff_internal.h"

namespace ff {
namespace adamw {

constexpr int kChunk = 4096;     // elements of a workgroup
constexpr int kBlock = 256;      // elements of a shared unit
constexpr int kTopM = 14, kTopV = 30;   // the largest code is 15 x 2^top units
constexpr int kExpBias = 120;    // a stored exponent is k + 120; units stay normal fp32 and bf16 numbers

struct Tensor {
  float* c;
  __bf16* copy;        // NULL: none
  void* m;
  void* v;
  uint8_t* mx;         // 8 bits: exponents of the blocks
  uint8_t* vx;
  int64_t n;
  double decay;
};

struct Place {
  int tensor, chunk;
};

struct Hyper {
  double lr, b1, b2, scale;
  float eps;
  double ibc1, ibc2;               // 1 / (1 - b^step), unless step_dev
  int64_t step;
  uint64_t seed;
  const float* lr_dev;
  const float* scale_dev;
  const int64_t* step_dev;
};

// Gradients of tensors first .. first + G - 1, by value.
template <int G>
struct Grads {
  const void* g[G];
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 Loose4 __attribute__((aligned(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 Loose2 __attribute__((aligned(2)));
typedef unsigned Loose1 __attribute__((aligned(1)));

__device__ __forceinline__ f32x4 widen(u32x2 w) {
  return f32x4{__builtin_bit_cast(float, w[0] << 16), __builtin_bit_cast(float, w[0] & 0xffff0000u),
               __builtin_bit_cast(float, w[1] << 16), __builtin_bit_cast(float, w[1] & 0xffff0000u)};
}
__device__ __forceinline__ unsigned bf16_bits(float x) { return __builtin_bit_cast(unsigned short, (__bf16)x); }

// Four elements from i of an array of n (zero past its end), and back.
__device__ __forceinline__ f32x4 get(const float* p, int64_t i, int64_t n) {
  if (i + 4 <= n) return *reinterpret_cast<const Loose4*>(p + i);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (i + j < n) v[j] = p[i + j];
  return v;
}
__device__ __forceinline__ f32x4 get(const __bf16* p, int64_t i, int64_t n) {
  if (i + 4 <= n) return widen(*reinterpret_cast<const Loose2*>(p + i));
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (i + j < n) v[j] = (float)p[i + j];
  return v;
}
__device__ __forceinline__ void put(float* p, int64_t i, int64_t n, f32x4 v) {
  if (i + 4 <= n) {
    *reinterpret_cast<Loose4*>(p + i) = v;
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (i + j < n) p[i + j] = v[j];
}
__device__ __forceinline__ void put(__bf16* p, int64_t i, int64_t n, f32x4 v) {
  if (i + 4 <= n) {
    *reinterpret_cast<Loose2*>(p + i) = u32x2{bf16_bits(v[0]) | bf16_bits(v[1]) << 16, bf16_bits(v[2]) | bf16_bits(v[3]) << 16};
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (i + j < n) p[i + j] = (__bf16)v[j];
}
__device__ __forceinline__ unsigned get(const uint8_t* p, int64_t i, int64_t n) {
  if (i + 4 <= n) return *reinterpret_cast<const Loose1*>(p + i);
  unsigned v = 0;
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (i + j < n) v |= (unsigned)p[i + j] << (8 * j);
  return v;
}
__device__ __forceinline__ void put(uint8_t* p, int64_t i, int64_t n, unsigned v) {
  if (i + 4 <= n) {
    *reinterpret_cast<Loose1*>(p + i) = v;
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (i + j < n) p[i + j] = (uint8_t)(v >> (8 * j));
}

__device__ __forceinline__ double power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// What a workgroup needs of the hyperparameters.
struct Step {
  float lr, decay, ibc1, ibc2, eps;
  double scale;
  int64_t step;
};
__device__ __forceinline__ Step step_of(const Hyper& h, double wd) {
  Step s;
  const double lr = h.lr_dev ? h.lr * (double)*h.lr_dev : h.lr;
  double ibc1 = h.ibc1, ibc2 = h.ibc2;
  s.step = h.step;
  if (h.step_dev) {
    s.step += *h.step_dev;
    ibc1 = 1.0 / (1.0 - power(h.b1, s.step));
    ibc2 = 1.0 / (1.0 - power(h.b2, s.step));
  }
  s.lr = (float)lr;
  s.decay = (float)(1.0 - lr * wd);
  s.ibc1 = (float)ibc1;
  s.ibc2 = (float)ibc2;
  s.eps = h.eps;
  s.scale = h.scale_dev ? h.scale * (double)*h.scale_dev : h.scale;
  return s;
}
__device__ __forceinline__ float stepped(float c, float m, float v, const Step& s) {
  return c * s.decay - s.lr * ((m * s.ibc1) / (sqrtf(v * s.ibc2) + s.eps));
}

template <class E, int G>
__global__ void __launch_bounds__(256) step_kernel(const Tensor* tensors, const Place* places, Grads<G> grads, int first,
                                                   Hyper h) {
  const Place at = places[blockIdx.x];
  const E* g = static_cast<const E*>(grads.g[at.tensor - first]);
  if (!g) return;
  const Tensor t = tensors[at.tensor];
  const Step s = step_of(h, t.decay);
  // The moments are made in fp64 and rounded once: b and 1 - b rounded to fp32 each do not sum to one, and a long run's v would be
  // off by the rest over 1 - b2 (1.7e-4 for b2 = 0.9999, 1.3% for 0.999999).
  const double b1 = h.b1, a1 = 1.0 - h.b1, b2 = h.b2, a2 = 1.0 - h.b2;
  float* pm = static_cast<float*>(t.m);
  float* pv = static_cast<float*>(t.v);
  const int64_t i0 = (int64_t)at.chunk * kChunk + threadIdx.x * 4;
#pragma unroll
  for (int q = 0; q < kChunk / 1024; ++q) {
    const int64_t i = i0 + q * 1024;
    if (i >= t.n) break;
    f32x4 c = get(t.c, i, t.n), gg = get(g, i, t.n), m = get(pm, i, t.n), v = get(pv, i, t.n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double x = (double)gg[j] * s.scale;
      m[j] = (float)(b1 * (double)m[j] + a1 * x);
      v[j] = (float)(b2 * (double)v[j] + a2 * (x * x));
      c[j] = stepped(c[j], m[j], v[j], s);
    }
    put(t.c, i, t.n, c);
    put(pm, i, t.n, m);
    put(pv, i, t.n, v);
    if (t.copy) put(t.copy, i, t.n, c);
  }
}

// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).
__device__ __forceinline__ void philox(unsigned (&c)[4], unsigned k0, unsigned k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    const unsigned x0 = (unsigned)(b >> 32) ^ c[1] ^ k0, x2 = (unsigned)(a >> 32) ^ c[3] ^ k1;
    c[1] = (unsigned)b, c[3] = (unsigned)a, c[0] = x0, c[2] = x2;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
}

// 2^k as a double
__device__ __forceinline__ double two(int k) { return __builtin_bit_cast(double, (uint64_t)(k + 1023) << 52); }

// Value of code a (no sign) in units.
__device__ __forceinline__ float units_of(unsigned a) {
  const int e = (int)(a >> 3) - 1;
  return e < 1 ? (float)a : (float)(8u + (a & 7u)) * __builtin_bit_cast(float, (unsigned)(e + 127) << 23);
}

// The least k whose unit lets the largest code reach `most`, as it is stored.
__device__ __forceinline__ int unit_of(float most, int top) {
  const unsigned b = __builtin_bit_cast(unsigned, most);
  const int k = (int)(b >> 23) - 127 - 3 - top + ((b & 0x7fffffu) > 0x700000u);
  return (k < -kExpBias ? -kExpBias : k) + kExpBias;
}

// Code of |x| (finite) in units 2^k, up = 2^-k; r: 16 random bits.  From 8 units on, the exponent and three bits of the
// double are the code, and the random fraction is added to the bits below; below 8, eight units more have the same step.
__device__ __forceinline__ int code_of(double x, double up, unsigned r, int top) {
  double y = fabs(x) * up;
  const bool low = y < 8.0;
  y = low ? y + 8.0 : y;
  const unsigned hi = (unsigned)(__builtin_bit_cast(uint64_t, y) >> 32) + (r << 1 | 1u);
  const int a = (int)(hi >> 17) - (1026 * 8 - 8) - (low ? 8 : 0);
  return a < 8 * top + 15 ? a : 8 * top + 15;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// A wave takes a block of 256 elements at a time, four a lane.
template <class E, int G>
__global__ void __launch_bounds__(256) step8_kernel(const Tensor* tensors, const Place* places, Grads<G> grads, int first,
                                                    Hyper h) {
  const Place at = places[blockIdx.x];
  const E* g = static_cast<const E*>(grads.g[at.tensor - first]);
  if (!g) return;
  const Tensor t = tensors[at.tensor];
  const Step s = step_of(h, t.decay);
  uint8_t* pm = static_cast<uint8_t*>(t.m);
  uint8_t* pv = static_cast<uint8_t*>(t.v);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double b1 = h.b1, a1 = 1.0 - h.b1, b2 = h.b2, a2 = 1.0 - h.b2;
#pragma unroll
  for (int q = 0; q < kChunk / 1024; ++q) {
    const int64_t block = (int64_t)at.chunk * (kChunk / kBlock) + q * 4 + wave;
    if (block * kBlock >= t.n) break;      // whole waves
    const int64_t i = block * kBlock + lane * 4;
    f32x4 c = get(t.c, i, t.n), gg = get(g, i, t.n);
    const unsigned cm = get(pm, i, t.n), cv = get(pv, i, t.n);
    const double um = two((int)t.mx[block] - kExpBias), uv = two((int)t.vx[block] - kExpBias);
    double m[4], v[4];
    float top_m = 0.f, top_v = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned am = cm >> (8 * j) & 0xffu;
      const float mu = units_of(am & 0x7fu);
      const double x = (double)gg[j] * s.scale;
      m[j] = b1 * ((double)(am & 0x80u ? -mu : mu) * um) + a1 * x;
      v[j] = b2 * ((double)units_of(cv >> (8 * j) & 0xffu) * uv) + a2 * (x * x);
      const float mf = (float)m[j], vf = (float)v[j];
      c[j] = stepped(c[j], mf, vf, s);
      // what is not finite has no code: the state forgets the element
      const bool finite = fabsf(mf) <= 3.402823466e38f && vf <= 3.402823466e38f;
      m[j] = finite ? m[j] : 0.0;
      v[j] = finite ? v[j] : 0.0;
      top_m = fmaxf(top_m, finite ? fabsf(mf) : 0.f);
      top_v = fmaxf(top_v, finite ? vf : 0.f);
    }
    put(t.c, i, t.n, c);
    if (t.copy) put(t.copy, i, t.n, c);
    const int km = unit_of(wave_max(top_m), kTopM), kv = unit_of(wave_max(top_v), kTopV);
    const double dm = two(kExpBias - km), dv = two(kExpBias - kv);
    const int64_t b = i >> 2;
    unsigned w[4] = {(unsigned)b, (unsigned)(b >> 32), (unsigned)s.step, (unsigned)at.tensor};
    philox(w, (unsigned)h.seed, (unsigned)(h.seed >> 32));
    unsigned om = 0, ov = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int a = code_of(m[j], dm, w[j] & 0xffffu, kTopM);
      const int z = code_of(v[j], dv, w[j] >> 16, kTopV);
      om |= (unsigned)(a | (m[j] < 0.0 ? 0x80 : 0)) << (8 * j);
      ov |= (unsigned)(v[j] > 0.0 && z < 1 ? 1 : z) << (8 * j);
    }
    put(pm, i, t.n, om);
    put(pv, i, t.n, ov);
    if (lane == 0) {
      t.mx[block] = (uint8_t)km;
      t.vx[block] = (uint8_t)kv;
    }
  }
}

template <int G>
struct Outs {
  __bf16* m[G];
  __bf16* v[G];
};

// The values of 8-bit moments in bf16, which holds them exactly; zeros behind the end up to a whole block.
template <int G>
__global__ void __launch_bounds__(256) read8_kernel(const Tensor* tensors, const Place* places, Outs<G> outs, int first) {
  const Place at = places[blockIdx.x];
  const Tensor t = tensors[at.tensor];
  __bf16* om = outs.m[at.tensor - first];
  __bf16* ov = outs.v[at.tensor - first];
  const int64_t whole = (t.n + kBlock - 1) / kBlock * kBlock;
#pragma unroll
  for (int q = 0; q < kChunk / 1024; ++q) {
    const int64_t i = (int64_t)at.chunk * kChunk + q * 1024 + threadIdx.x * 4;
    if (i >= whole) break;
    const unsigned cm = get(static_cast<const uint8_t*>(t.m), i, t.n), cv = get(static_cast<const uint8_t*>(t.v), i, t.n);
    const float um = (float)two((int)t.mx[i / kBlock] - kExpBias), uv = (float)two((int)t.vx[i / kBlock] - kExpBias);
    f32x4 m, v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned a = cm >> (8 * j) & 0xffu;
      m[j] = units_of(a & 0x7fu) * (a & 0x80u ? -um : um);
      v[j] = units_of(cv >> (8 * j) & 0xffu) * uv;
    }
    if (om) put(om, i, whole, m);
    if (ov) put(ov, i, whole, v);
  }
}

constexpr int kGrads = 384;      // most of one launch: 3 KiB of its 4 KiB of arguments
constexpr int kFew = 16;         // sets up to this size: an eighth of a KiB

}  // namespace adamw
}  // namespace ff

struct ff_adamw_set {
  int device = 0;
  int64_t count = 0;
  int states = 0, g_dtype = 0;
  ff::adamw::Tensor* tensors = nullptr;   // device
  ff::adamw::Place* places = nullptr;     // device
  std::vector<int64_t> first;             // [count + 1] first chunk of each tensor
  ~ff_adamw_set() {
    if (tensors) (void)hipFree(tensors);
  }
};

namespace ff {
namespace adamw {
namespace {

template <int G, class F>
hipError_t over_tensors(const ff_adamw_set* s, const F& launch) {
  for (int64_t t0 = 0; t0 < s->count; t0 += G) {
    const int64_t t1 = t0 + G < s->count ? t0 + G : s->count;
    const int64_t chunks = s->first[t1] - s->first[t0];
    // a launch has fewer than 2^32 threads
    for (int64_t c = 0; c < chunks; c += (int64_t)1 << 23) {
      const int64_t n = chunks - c < ((int64_t)1 << 23) ? chunks - c : (int64_t)1 << 23;
      launch((int)t0, (int)(t1 - t0), s->places + s->first[t0] + c, (unsigned)n);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

template <class E, int G>
hipError_t run_step(const ff_adamw_set* s, const void* const* g, const Hyper& h, hipStream_t stream) {
  return over_tensors<G>(s, [&](int t0, int nt, const Place* places, unsigned chunks) {
    Grads<G> a{};
    for (int i = 0; i < nt; ++i) a.g[i] = g[t0 + i];
    if (s->states == FF_STATES_8BIT)
      hipLaunchKernelGGL((step8_kernel<E, G>), dim3(chunks), dim3(256), 0, stream, s->tensors, places, a, t0, h);
    else
      hipLaunchKernelGGL((step_kernel<E, G>), dim3(chunks), dim3(256), 0, stream, s->tensors, places, a, t0, h);
  });
}

// Memory that a step writes.
struct Written {
  uintptr_t first, end;
  int64_t tensor;
};

ff_status check_set(const ff_adamw_set* s) {
  if (!s) return fail(FF_EINVAL, "the set is NULL");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) (void)hipGetLastError(), dev = -1;
  if (dev != s->device) return fail(FF_EINVAL, "current device %d is not the set's device %d", dev, s->device);
  return FF_OK;
}

// A call of the runtime failed; the error is not left for the next launch, which asks for the last one as its own.
ff_status lost(ff_status st, const char* what) {
  (void)hipGetLastError();
  return fail(st, "%s", what);
}

}  // namespace
}  // namespace adamw
}  // namespace ff

extern "C" {

ff_status ff_adamw_set_create(int64_t count, const int64_t* n, int states, int g_dtype, float* const* c, void* const* copy,
                              void* const* m, void* const* v, uint8_t* const* m_exp, uint8_t* const* v_exp,
                              const double* weight_decay, ff_adamw_set** out) {
  using namespace ff::adamw;
  ff::clear_error();
  if (!out) return ff::fail(FF_EINVAL, "out is NULL");
  *out = nullptr;
  if (count < 1 || count > ((int64_t)1 << 20)) return ff::fail(FF_EINVAL, "count=%lld out of range", (long long)count);
  if (states != FF_STATES_F32 && states != FF_STATES_8BIT) return ff::fail(FF_EINVAL, "unknown states %d", states);
  if (g_dtype != FF_F32 && g_dtype != FF_BF16) return ff::fail(FF_EINVAL, "unknown gradient dtype %d", g_dtype);
  const bool eight = states == FF_STATES_8BIT;
  if (!n || !c || !m || !v || (eight && (!m_exp || !v_exp))) return ff::fail(FF_EINVAL, "NULL array");
  int64_t chunks = 0;
  for (int64_t i = 0; i < count; ++i) {
    const long long k = (long long)i;
    if (n[i] < 0 || n[i] > ((int64_t)1 << 40)) return ff::fail(FF_EINVAL, "length %lld of tensor %lld out of range", (long long)n[i], k);
    chunks += (n[i] + kChunk - 1) / kChunk;
    if (weight_decay && !(weight_decay[i] >= 0.0 && std::isfinite(weight_decay[i])))
      return ff::fail(FF_EINVAL, "weight decay of tensor %lld must be finite and >= 0", k);
    if (n[i] == 0) continue;
    if (!c[i] || !m[i] || !v[i] || (eight && (!m_exp[i] || !v_exp[i]))) return ff::fail(FF_EINVAL, "tensor %lld: NULL array", k);
    if ((uintptr_t)c[i] % 4 || (copy && (uintptr_t)copy[i] % 2) || (!eight && ((uintptr_t)m[i] % 4 || (uintptr_t)v[i] % 4)))
      return ff::fail(FF_EINVAL, "tensor %lld: misaligned array", k);
  }
  if (chunks > ((int64_t)1 << 30)) return ff::fail(FF_EINVAL, "the tensors' lengths sum to too much");
  std::unique_ptr<ff_adamw_set> s;
  std::vector<char> host;
  try {
    // a step's workgroups write all arrays at once: one element in two of them would have two writers
    std::vector<Written> written;
    written.reserve((size_t)count * 6);
    for (int64_t i = 0; i < count; ++i) {
      if (n[i] == 0) continue;
      const uintptr_t len = (uintptr_t)n[i], state = eight ? len : 4 * len, blocks = (len + kBlock - 1) / kBlock;
      auto add = [&](const void* p, uintptr_t bytes) { written.push_back(Written{(uintptr_t)p, (uintptr_t)p + bytes, i}); };
      add(c[i], 4 * len), add(m[i], state), add(v[i], state);
      if (copy && copy[i]) add(copy[i], 2 * len);
      if (eight) add(m_exp[i], blocks), add(v_exp[i], blocks);
    }
    std::sort(written.begin(), written.end(), [](const Written& a, const Written& b) { return a.first < b.first; });
    for (size_t i = 1; i < written.size(); ++i)
      if (written[i].first < written[i - 1].end)
        return ff::fail(FF_EINVAL, "arrays of tensors %lld and %lld overlap", (long long)written[i - 1].tensor,
                        (long long)written[i].tensor);
    s.reset(new ff_adamw_set);
    s->first.resize((size_t)count + 1);
    host.resize((size_t)count * sizeof(Tensor) + (size_t)chunks * sizeof(Place));
  } catch (const std::bad_alloc&) {
    return ff::fail(FF_ENOMEM, "host allocation failed");
  }
  s->count = count, s->states = states, s->g_dtype = g_dtype;
  Tensor* ht = reinterpret_cast<Tensor*>(host.data());
  Place* hp = reinterpret_cast<Place*>(ht + count);
  int64_t at = 0;
  for (int64_t i = 0; i < count; ++i) {
    ht[i] = Tensor{c[i], copy ? static_cast<__bf16*>(copy[i]) : nullptr, m[i], v[i], eight ? m_exp[i] : nullptr,
                   eight ? v_exp[i] : nullptr, n[i], weight_decay ? weight_decay[i] : 0.0};
    s->first[(size_t)i] = at;
    for (int64_t k = 0; k < (n[i] + kChunk - 1) / kChunk; ++k) hp[at++] = Place{(int)i, (int)k};
  }
  s->first[(size_t)count] = at;
  if (hipGetDevice(&s->device) != hipSuccess) return lost(FF_EDEVICE, "no HIP device");
  void* dev = nullptr;
  if (hipMalloc(&dev, host.size()) != hipSuccess) return lost(FF_ENOMEM, "device allocation of the set's table failed");
  s->tensors = static_cast<Tensor*>(dev);
  s->places = reinterpret_cast<Place*>(s->tensors + count);
  if (hipMemcpy(dev, host.data(), host.size(), hipMemcpyHostToDevice) != hipSuccess)
    return lost(FF_EDEVICE, "copy of the set's table failed");
  *out = s.release();
  return FF_OK;
}

void ff_adamw_set_destroy(ff_adamw_set* s) { delete s; }

ff_status ff_adamw_set_step(const ff_adamw_set* s, const void* const* g, const ff_adamw_hyper* p, void* stream) {
  using namespace ff::adamw;
  ff::clear_error();
  ff_status st = check_set(s);
  if (st != FF_OK) return st;
  if (!g || !p) return ff::fail(FF_EINVAL, "NULL array");
  if (p->step < 1 && !p->step_dev) return ff::fail(FF_EINVAL, "step numbers start at 1 (got %lld)", (long long)p->step);
  if (!(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0))
    return ff::fail(FF_EINVAL, "betas must lie in [0, 1)");
  if (!((float)p->eps > 0.f) || !std::isfinite(p->eps) || !std::isfinite(p->lr) || !(p->lr >= 0.0) || !std::isfinite(p->grad_scale))
    return ff::fail(FF_EINVAL, "need eps > 0, finite lr >= 0 and a finite grad_scale");
  if ((uintptr_t)p->lr_dev % 4 || (uintptr_t)p->grad_scale_dev % 4 || (uintptr_t)p->step_dev % 8)
    return ff::fail(FF_EINVAL, "a device value is misaligned");
  const int gsz = s->g_dtype == FF_BF16 ? 2 : 4;
  for (int64_t i = 0; i < s->count; ++i)
    if ((uintptr_t)g[i] % gsz) return ff::fail(FF_EINVAL, "gradient %lld is misaligned", (long long)i);
  Hyper h{p->lr, p->beta1, p->beta2, p->grad_scale, (float)p->eps, 0.0, 0.0, p->step, p->seed, p->lr_dev, p->grad_scale_dev,
          p->step_dev};
  if (!p->step_dev) {
    h.ibc1 = 1.0 / (1.0 - std::pow(p->beta1, (double)p->step));
    h.ibc2 = 1.0 / (1.0 - std::pow(p->beta2, (double)p->step));
  }
  const hipStream_t q = (hipStream_t)stream;
  hipError_t e;
  if (s->g_dtype == FF_BF16)
    e = s->count <= kFew ? run_step<__bf16, kFew>(s, g, h, q) : run_step<__bf16, kGrads>(s, g, h, q);
  else
    e = s->count <= kFew ? run_step<float, kFew>(s, g, h, q) : run_step<float, kGrads>(s, g, h, q);
  return e == hipSuccess ? FF_OK : ff::fail(FF_EDEVICE, "AdamW launch: %s", hipGetErrorString(e));
}

ff_status ff_adamw_set_read(const ff_adamw_set* s, void* const* m, void* const* v, void* stream) {
  using namespace ff::adamw;
  ff::clear_error();
  ff_status st = check_set(s);
  if (st != FF_OK) return st;
  if (s->states != FF_STATES_8BIT) return ff::fail(FF_EINVAL, "the set's states are fp32: read them where they are");
  if (!m || !v) return ff::fail(FF_EINVAL, "NULL array");
  for (int64_t i = 0; i < s->count; ++i)
    if ((uintptr_t)m[i] % 2 || (uintptr_t)v[i] % 2) return ff::fail(FF_EINVAL, "output %lld is misaligned", (long long)i);
  const hipError_t e = over_tensors<kGrads / 2>(s, [&](int t0, int nt, const Place* places, unsigned chunks) {
    Outs<kGrads / 2> a{};
    for (int i = 0; i < nt; ++i) a.m[i] = static_cast<__bf16*>(m[t0 + i]), a.v[i] = static_cast<__bf16*>(v[t0 + i]);
    hipLaunchKernelGGL(read8_kernel<kGrads / 2>, dim3(chunks), dim3(256), 0, (hipStream_t)stream, s->tensors, places, a, t0);
  });
  return e == hipSuccess ? FF_OK : ff::fail(FF_EDEVICE, "AdamW states: %s", hipGetErrorString(e));
}

}  // extern "C"
