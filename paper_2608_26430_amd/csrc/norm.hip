// Layer norm, forward and backward, with the reduction of the weight's and bias's gradients.
//
//   mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), h = (x - mu) r, y = w h + b          (a row x of n)
//   a = w g;  dx = beta dx + r (a - mean a - h mean(a h));  dw = sum_t g h;  db = sum_t g
// Every sum is in fp32; the variance is that of the centred row, which stays in registers, so that a large mean costs
// no digits.  A row belongs to WV waves (1 or 8) whose threads hold NV pieces of 16 bytes each;
// rows wider than that are read three times.  Workgroups walk the rows with a stride, the vectors of their columns in
// registers (fp32 weight and bias read for every row were twice a bf16 row's own bytes: 8192 x 8192 forward 67 -> 52
// us), reading the next row under the arithmetic of one.  The backward's also keep dw and db of their columns and leave one
// partial row each, added up in a fixed order by a second kernel: the same inputs give the same bits.  Bound by
// memory: forward 2 T n, backward 3 T n elements; 8192 x 8192 in bf16 52 and 84 + 5 us, 5.1 and 4.8 TB/s, where a large
// copy has 5.2; 12,608 x 768 11.8 and 14.7 + 3.9 us, of which a launch and the first row's latency are 4 each.
#include <cmath>

#include "ff_internal.h"

namespace ff {
namespace norm {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 Loose __attribute__((aligned(2)));   // on any element

struct Args {
  const void* X;
  const void* G;
  void* Y;             // forward: y, backward: dx
  int64_t ldx, ldg, ldy;
  int64_t T;
  int n;
  const void* weight;  // NULL: ones
  const void* bias;    // NULL: zeros
  int w_bf16;
  float eps;
  float* mean;
  float* rstd;
  float beta;
  float* part;         // [workgroups][2][n]: dw, db of a workgroup's rows (NULL: not wanted)
};

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

// A workgroup walks rows with a stride, weight and bias of its columns in registers; the next row is read while one is
// normalised.
template <class E, int NV, int WV, bool PART>
__global__ void __launch_bounds__(threads_of(WV), 2) fwd_kernel(Args a) {
  constexpr int kT = WV * 64, kRows = threads_of(WV) / kT, kN = Pack<E>::kN;
  typedef Row<E, NV, WV, PART> R;
  __shared__ float2 sh[2][WV];
  const int l = threadIdx.x % kT;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / kT;
  if (t >= a.T) return;      // whole waves; with WV > 1 a workgroup has one row at a time
  R x;
  x.load(a.X, a.ldx, t, l, a.n);
  float w[NV][kN], b[NV][kN];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (R::skip(i, l, a.n) < kN) {
      vector_at<kN>(a.weight, a.w_bf16, 1.f, R::at(i, l, a.n), w[i]);
      vector_at<kN>(a.bias, a.w_bf16, 0.f, R::at(i, l, a.n), b[i]);
    }
  }
  for (;;) {
    float v[NV][kN];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      Pack<E>::widen(x.raw[i], v[i]);
      const int skip = R::skip(i, l, a.n);
#pragma unroll
      for (int k = 0; k < kN; ++k) s += !PART || k >= skip ? v[i][k] : 0.f;
    }
    const int64_t next = t + stride;
    if (next < a.T) x.load(a.X, a.ldx, next, l, a.n);
    const float mu = row_sum<WV>(make_float2(s, 0.f), sh[0]).x / (float)a.n;
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int skip = R::skip(i, l, a.n);
#pragma unroll
      for (int k = 0; k < kN; ++k) {
        v[i][k] -= mu;
        q = (PART ? k >= skip : skip == 0) ? fmaf(v[i][k], v[i][k], q) : q;
      }
    }
    // (the barrier within keeps sh[0] until every wave has read it)
    const float var = row_sum<WV>(make_float2(q, 0.f), sh[1]).x / (float)a.n;
    const float r = 1.f / sqrtf(var + a.eps);
    E* y = static_cast<E*>(a.Y) + t * a.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (R::skip(i, l, a.n) < kN) {
        float o[kN];
#pragma unroll
        for (int k = 0; k < kN; ++k) o[k] = fmaf(v[i][k] * r, w[i][k], b[i][k]);
        Pack<E>::put(y + R::at(i, l, a.n), o);
      }
    }
    if (l == 0) {
      if (a.mean) a.mean[t] = mu;
      if (a.rstd) a.rstd[t] = r;
    }
    if (next >= a.T) break;
    t = next;
  }
}

// Rows too wide for the registers: read three times.  (sh[0] and sh[1] take turns, so that the barrier of one sum keeps
// the other's place until every wave has read it, over rows too.)
template <class E>
__global__ void __launch_bounds__(1024) fwd_wide_kernel(Args a) {
  __shared__ float2 sh[2][16];
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const E* x = static_cast<const E*>(a.X) + t * a.ldx;
    E* y = static_cast<E*>(a.Y) + t * a.ldy;
    float s = 0.f;
    for (int c = threadIdx.x; c < a.n; c += 1024) s += (float)x[c];
    const float mu = row_sum<16>(make_float2(s, 0.f), sh[0]).x / (float)a.n;
    float q = 0.f;
    for (int c = threadIdx.x; c < a.n; c += 1024) {
      const float d = (float)x[c] - mu;
      q = fmaf(d, d, q);
    }
    const float r = 1.f / sqrtf(row_sum<16>(make_float2(q, 0.f), sh[1]).x / (float)a.n + a.eps);
    for (int c = threadIdx.x; c < a.n; c += 1024) {
      float w, b;
      vector_at<1>(a.weight, a.w_bf16, 1.f, c, &w);
      vector_at<1>(a.bias, a.w_bf16, 0.f, c, &b);
      y[c] = (E)fmaf(((float)x[c] - mu) * r, w, b);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[t] = mu;
      if (a.rstd) a.rstd[t] = r;
    }
  }
}

template <class E, int NV, int WV, bool PART>
__global__ void __launch_bounds__(threads_of(WV), 2) bwd_kernel(Args a) {
  constexpr int kT = WV * 64, kRows = threads_of(WV) / kT, kN = Pack<E>::kN;
  typedef Row<E, NV, WV, PART> R;
  __shared__ float2 sh[2][WV];
  __shared__ float comb[kRows > 1 ? 2 * NV * kN * kT : 1];
  const int l = threadIdx.x % kT, sub = threadIdx.x / kT;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t t = (int64_t)blockIdx.x * kRows + sub;
  R x, g;
  float mu_next = 0.f, r_next = 0.f;
  auto fetch = [&](int64_t row) {
    if (row >= a.T) return;
    x.load(a.X, a.ldx, row, l, a.n);
    g.load(a.G, a.ldg, row, l, a.n);
    mu_next = a.mean[row];
    r_next = a.rstd[row];
  };
  fetch(t);
  float w[NV][kN], dw[NV][kN], db[NV][kN];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int k = 0; k < kN; ++k) w[i][k] = dw[i][k] = db[i][k] = 0.f;
    if (R::skip(i, l, a.n) < kN) vector_at<kN>(a.weight, a.w_bf16, 1.f, R::at(i, l, a.n), w[i]);
  }
  const float inv_n = 1.f / (float)a.n;
  int turn = 0;
  for (; t < a.T; t += stride, turn ^= 1) {
    const float mu = mu_next, r = r_next;
    float h[NV][kN], gg[NV][kN];
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      Pack<E>::widen(x.raw[i], h[i]);
      Pack<E>::widen(g.raw[i], gg[i]);
    }
    fetch(t + stride);
    // a piece that is not there has g = 0, so that nothing comes of it
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int skip = R::skip(i, l, a.n);
#pragma unroll
      for (int k = 0; k < kN; ++k) {
        h[i][k] = (h[i][k] - mu) * r;
        dw[i][k] = fmaf(gg[i][k], h[i][k], dw[i][k]);
        db[i][k] += gg[i][k];
        gg[i][k] *= w[i][k];
        const float q = !PART || k >= skip ? gg[i][k] : 0.f;
        s.x += q;
        s.y = fmaf(q, h[i][k], s.y);
      }
    }
    if (!a.Y) continue;
    s = row_sum<WV>(s, sh[turn]);
    const float ma = s.x * inv_n, mh = s.y * inv_n;
    E* dx = static_cast<E*>(a.Y) + t * a.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int skip = R::skip(i, l, a.n);
      if (skip < kN) {
        E* p = dx + R::at(i, l, a.n);
        float o[kN];
#pragma unroll
        for (int k = 0; k < kN; ++k) o[k] = r * (gg[i][k] - ma - h[i][k] * mh);
        if (a.beta == 0.f) {
          Pack<E>::put(p, o);
        } else if (!PART || skip == 0) {
          float old[kN];
          Pack<E>::widen(Pack<E>::load(p), old);
#pragma unroll
          for (int k = 0; k < kN; ++k) o[k] = fmaf(a.beta, old[k], o[k]);
          Pack<E>::put(p, o);
        } else {
          // the shared elements are added to once: this piece writes its own alone
#pragma unroll
          for (int k = 0; k < kN; ++k)
            if (k >= skip) p[k] = (E)fmaf(a.beta, (float)p[k], o[k]);
        }
      }
    }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.n;
  if constexpr (kRows > 1) {
    // the workgroup's rows in turn: a fixed order
    for (int q = 0; q < kRows; ++q) {
      if (q == sub)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int skip = R::skip(i, l, a.n);
          float* p = comb + R::at(i, l, a.n);
#pragma unroll
          for (int k = 0; k < kN; ++k)
            if (k >= skip) {
              p[k] = q ? p[k] + dw[i][k] : dw[i][k];
              p[NV * kN * kT + k] = q ? p[NV * kN * kT + k] + db[i][k] : db[i][k];
            }
        }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < a.n; c += threads_of(WV)) {
      part[c] = comb[c];
      part[a.n + c] = comb[NV * kN * kT + c];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int skip = R::skip(i, l, a.n), c = R::at(i, l, a.n);
#pragma unroll
      for (int k = 0; k < kN; ++k)
        if (k >= skip) {
          part[c + k] = dw[i][k];
          part[a.n + c + k] = db[i][k];
        }
    }
  }
}

// Rows too wide for the registers: dx row by row.
template <class E>
__global__ void __launch_bounds__(1024) bwd_wide_kernel(Args a) {
  __shared__ float2 sh[2][16];
  int turn = 0;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x, turn ^= 1) {
    const E* x = static_cast<const E*>(a.X) + t * a.ldx;
    const E* g = static_cast<const E*>(a.G) + t * a.ldg;
    E* dx = static_cast<E*>(a.Y) + t * a.ldy;
    const float mu = a.mean[t], r = a.rstd[t];
    float2 s = make_float2(0.f, 0.f);
    for (int c = threadIdx.x; c < a.n; c += 1024) {
      float w;
      vector_at<1>(a.weight, a.w_bf16, 1.f, c, &w);
      w *= (float)g[c];
      s.x += w;
      s.y = fmaf(w, ((float)x[c] - mu) * r, s.y);
    }
    s = row_sum<16>(s, sh[turn]);
    const float ma = s.x / (float)a.n, mh = s.y / (float)a.n;
    for (int c = threadIdx.x; c < a.n; c += 1024) {
      float w;
      vector_at<1>(a.weight, a.w_bf16, 1.f, c, &w);
      float o = r * (w * (float)g[c] - ma - ((float)x[c] - mu) * r * mh);
      if (a.beta != 0.f) o = fmaf(a.beta, (float)dx[c], o);
      dx[c] = (E)o;
    }
  }
}
// and dw, db: a workgroup takes 256 columns at a time of a share of the rows
template <class E>
__global__ void __launch_bounds__(256) bwd_wide_vectors_kernel(Args a) {
  for (int c = blockIdx.y * 256 + threadIdx.x; c < a.n; c += gridDim.y * 256) {
    float dw = 0.f, db = 0.f;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
      const float g = (float)(static_cast<const E*>(a.G) + t * a.ldg)[c];
      dw = fmaf(g, ((float)(static_cast<const E*>(a.X) + t * a.ldx)[c] - a.mean[t]) * a.rstd[t], dw);
      db += g;
    }
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.n;
    part[c] = dw;
    part[a.n + c] = db;
  }
}

// out (dw then db) = [out +] sum over the partial rows: 32 columns x 32 shares of the rows per workgroup.
__global__ void __launch_bounds__(1024) vector_sum_kernel(const float* part, int rows, int n, int add, float* dw, float* db) {
  __shared__ float sh[32][33];
  const int k = threadIdx.x & 31, c = blockIdx.x * 32 + k, q = threadIdx.x >> 5;
  float s = 0.f;
  if (c < 2 * n) {
#pragma unroll 8
    for (int r = q; r < rows; r += 32) s += part[(int64_t)r * 2 * n + c];
  }
  sh[q][k] = s;
  __syncthreads();
  if (q || c >= 2 * n) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) s += sh[i][k];
  float* out = c < n ? dw : db;
  if (!out) return;
  out += c < n ? c : c - n;
  *out = add ? *out + s : s;
}

// ------------------------------------------------------------------------------------------- dispatch

// The instance of a row of n: NV pieces of a thread and WV waves of a row.  A wave takes rows of up to four pieces a
// lane (bf16: 2048 wide; 2048 wide and 8192 rows, forward / backward: 14.6 / 20.8 us against 17.4 / 26.8 with four waves),
// eight waves up to four (8192 wide, two: 50.6 / 87 us against 51.1 / 94 with four waves of four and 65 / 90 with sixteen of
// one);
// rows wider than that (bf16 16384, fp32 8192), or narrower than a piece, are read three times.  A backward with a last
// piece that overlaps keeps to two pieces a lane of one wave: four spill (2047 wide and 8192 rows 47 us).
struct Shape {
  int nv, wv;   // wv 0: wide
  bool part;    // the last piece is a part
};
Shape shape_of(int64_t n, int esz, bool bwd) {
  const int per = 16 / esz;
  const int64_t p = (n + per - 1) / per;
  auto fit = [&](int wv, int limit) -> int {
    for (int nv : {1, 2, 4})
      if (nv <= limit && p <= (int64_t)nv * wv * 64) return nv;
    return 0;
  };
  const bool part = n % per != 0;
  if (n < per) return {0, 0, part};
  if (int nv = fit(1, bwd && part ? 2 : 4)) return {nv, 1, part};
  if (int nv = fit(8, 4)) return {nv, 8, part};
  return {0, 0, part};
}

// Workgroups of a forward: four of one-wave rows per CU (12,608 rows of 768: 11.8 us with 1024 workgroups, 13.1 with 512, 11.9
// with one per four rows; 8192 of 8192: 52, 50 and, one row each, 67).
int64_t fwd_groups(int64_t T, const Shape& s) {
  const int rows = s.wv == 1 ? 4 : 1;
  const int64_t g = (T + rows - 1) / rows;
  return g < 1024 ? g : 1024;
}
// And of a backward, each with a partial row of dw and db to write and add up (12,608 rows of 768: 14.8 us with 512, 18.6
// with 256, 16.9 with 1024; 8192 of 8192: 83 with 256, 92 with 512, 107 with 128).
constexpr int kGroups = 512;
int groups_of(int64_t T, int64_t n, const Shape& s) {
  const int rows = s.wv == 1 ? 4 : 1;
  const int64_t g = (T + rows - 1) / rows, most = n <= 4096 ? kGroups : kGroups / 2;
  return (int)(g < most ? g : most);
}

template <class E, int NV, int WV>
void launch(const Args& a, const Shape& sh, bool bwd, int groups, hipStream_t s) {
  const dim3 grid((unsigned)groups), block(threads_of(WV));
  if (bwd && sh.part) hipLaunchKernelGGL((bwd_kernel<E, NV, WV, true>), grid, block, 0, s, a);
  else if (bwd) hipLaunchKernelGGL((bwd_kernel<E, NV, WV, false>), grid, block, 0, s, a);
  else if (sh.part) hipLaunchKernelGGL((fwd_kernel<E, NV, WV, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((fwd_kernel<E, NV, WV, false>), grid, block, 0, s, a);
}

template <class E, int WV>
void launch_nv(const Args& a, const Shape& sh, bool bwd, int groups, hipStream_t s) {
  if (sh.nv == 1) launch<E, 1, WV>(a, sh, bwd, groups, s);
  else if (sh.nv == 2) launch<E, 2, WV>(a, sh, bwd, groups, s);
  else launch<E, 4, WV>(a, sh, bwd, groups, s);
}

template <class E>
hipError_t run(const Args& a, const Shape& sh, bool bwd, int groups, hipStream_t s) {
  if (sh.wv == 0) {
    // a launch has fewer than 2^32 threads
    const dim3 rows((unsigned)(a.T < (1 << 20) ? a.T : (1 << 20)));
    const dim3 columns((unsigned)groups, (unsigned)(a.n < (1 << 20) ? (a.n + 255) / 256 : 4096));
    if (!bwd) hipLaunchKernelGGL(fwd_wide_kernel<E>, rows, dim3(1024), 0, s, a);
    if (bwd && a.Y) hipLaunchKernelGGL(bwd_wide_kernel<E>, rows, dim3(1024), 0, s, a);
    if (bwd && a.part) hipLaunchKernelGGL(bwd_wide_vectors_kernel<E>, columns, dim3(256), 0, s, a);
  } else if (sh.wv == 1) {
    launch_nv<E, 1>(a, sh, bwd, groups, s);
  } else {
    launch_nv<E, 8>(a, sh, bwd, groups, s);
  }
  return hipGetLastError();
}

ff_status check_rows(const char* name, const void* p, int64_t ld, int64_t n, int esz) {
  if (!p) return fail(FF_EINVAL, "%s is NULL", name);
  if (ld < n) return fail(FF_EINVAL, "leading dimension of %s (%lld) < %lld", name, (long long)ld, (long long)n);
  if ((uintptr_t)p % esz) return fail(FF_EINVAL, "%s is misaligned", name);
  return FF_OK;
}

ff_status check_sizes(int64_t T, int64_t n, int act, int w_dtype) {
  if (act != FF_F32 && act != FF_BF16) return fail(FF_EINVAL, "unknown activation dtype %d", act);
  if (w_dtype != FF_F32 && w_dtype != FF_BF16) return fail(FF_EINVAL, "unknown weight dtype %d", w_dtype);
  if (T < 0 || T > ((int64_t)1 << 30) || n < 1 || n > ((int64_t)1 << 24))
    return fail(FF_EINVAL, "T=%lld or n=%lld out of range", (long long)T, (long long)n);
  return FF_OK;
}

}  // namespace norm
}  // namespace ff

extern "C" {

ff_status ff_layernorm_fwd(int64_t T, int64_t n, int act, const void* X, int64_t ldx, int w_dtype, const void* weight,
                           const void* bias, float eps, void* Y, int64_t ldy, float* mean, float* rstd, void* stream) {
  using namespace ff::norm;
  ff::clear_error();
  ff_status st = check_sizes(T, n, act, w_dtype);
  if (st != FF_OK) return st;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return ff::fail(FF_EINVAL, "eps=%g must be finite and >= 0", (double)eps);
  if (T == 0) return FF_OK;
  const int esz = act == FF_BF16 ? 2 : 4, wsz = w_dtype == FF_BF16 ? 2 : 4;
  if ((st = check_rows("X", X, ldx, n, esz)) != FF_OK) return st;
  if ((st = check_rows("Y", Y, ldy, n, esz)) != FF_OK) return st;
  if ((uintptr_t)weight % wsz || (uintptr_t)bias % wsz || (uintptr_t)mean % 4 || (uintptr_t)rstd % 4)
    return ff::fail(FF_EINVAL, "weight, bias, mean or rstd is misaligned");
  Args a{};
  a.X = X, a.Y = Y, a.ldx = ldx, a.ldy = ldy, a.T = T, a.n = (int)n, a.weight = weight, a.bias = bias;
  a.w_bf16 = w_dtype == FF_BF16, a.eps = eps, a.mean = mean, a.rstd = rstd;
  const Shape sh = shape_of(n, esz, false);
  const int groups = (int)fwd_groups(T, sh);
  const hipError_t e = act == FF_BF16 ? run<__bf16>(a, sh, false, groups, (hipStream_t)stream)
                                      : run<float>(a, sh, false, groups, (hipStream_t)stream);
  return e == hipSuccess ? FF_OK : ff::fail(FF_EDEVICE, "layer norm forward: %s", hipGetErrorString(e));
}

ff_status ff_layernorm_workspace(int64_t T, int64_t n, int64_t* bytes) {
  ff::clear_error();
  ff_status st = ff::norm::check_sizes(T, n, FF_F32, FF_F32);
  if (st != FF_OK) return st;
  if (!bytes) return ff::fail(FF_EINVAL, "bytes is NULL");
  const int64_t rows = T < ff::norm::kGroups ? (T ? T : 1) : ff::norm::kGroups;
  *bytes = rows * 2 * n * 4;
  return FF_OK;
}

ff_status ff_layernorm_bwd(int64_t T, int64_t n, int act, const void* X, int64_t ldx, const void* G, int64_t ldg,
                           int w_dtype, const void* weight, const float* mean, const float* rstd, float beta_dx, void* dX,
                           int64_t lddx, int accumulate_dw, float* dweight, float* dbias, void* workspace,
                           int64_t workspace_bytes, void* stream) {
  using namespace ff::norm;
  ff::clear_error();
  ff_status st = check_sizes(T, n, act, w_dtype);
  if (st != FF_OK) return st;
  if ((uintptr_t)dweight % 4 || (uintptr_t)dbias % 4) return ff::fail(FF_EINVAL, "dweight or dbias is misaligned");
  const bool vectors = dweight || dbias;
  if (!dX && !vectors) return FF_OK;
  const int esz = act == FF_BF16 ? 2 : 4, wsz = w_dtype == FF_BF16 ? 2 : 4;
  int groups = 0;
  Args a{};
  if (T > 0) {
    if ((st = check_rows("X", X, ldx, n, esz)) != FF_OK) return st;
    if ((st = check_rows("G", G, ldg, n, esz)) != FF_OK) return st;
    if (dX && (st = check_rows("dX", dX, lddx, n, esz)) != FF_OK) return st;
    if (!mean || !rstd) return ff::fail(FF_EINVAL, "mean or rstd is NULL");
    if ((uintptr_t)weight % wsz || (uintptr_t)mean % 4 || (uintptr_t)rstd % 4)
      return ff::fail(FF_EINVAL, "weight, mean or rstd is misaligned");
    const Shape sh = shape_of(n, esz, true);
    groups = groups_of(T, n, sh);
    if (vectors) {
      if (!workspace || (uintptr_t)workspace % 16) return ff::fail(FF_EINVAL, "the workspace is NULL or not 16-byte aligned");
      const int64_t need = (int64_t)groups * 2 * n * 4;
      if (workspace_bytes < need)
        return ff::fail(FF_EINVAL, "the workspace holds %lld bytes, the call needs %lld", (long long)workspace_bytes,
                        (long long)need);
    }
    a.X = X, a.G = G, a.Y = dX, a.ldx = ldx, a.ldg = ldg, a.ldy = lddx, a.T = T, a.n = (int)n, a.weight = weight;
    a.w_bf16 = w_dtype == FF_BF16, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd), a.beta = beta_dx;
    a.part = vectors ? static_cast<float*>(workspace) : nullptr;
    const hipError_t e = act == FF_BF16 ? run<__bf16>(a, sh, true, groups, (hipStream_t)stream)
                                        : run<float>(a, sh, true, groups, (hipStream_t)stream);
    if (e != hipSuccess) return ff::fail(FF_EDEVICE, "layer norm backward: %s", hipGetErrorString(e));
  }
  if (vectors) {
    hipLaunchKernelGGL(vector_sum_kernel, dim3((unsigned)((2 * n + 31) / 32)), dim3(1024), 0, (hipStream_t)stream, a.part,
                       groups, (int)n, accumulate_dw, dweight, dbias);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return ff::fail(FF_EDEVICE, "layer norm backward: %s", hipGetErrorString(e));
  }
  return FF_OK;
}

}  // extern "C"
