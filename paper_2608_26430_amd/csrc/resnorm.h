// Join of two blocks, forward and backward (kernels; resnorm.hip has the calls, resnorm_inst.hip the backward's instances).
//
//   p = post(b) = wp hp + bp, hp = (b - mp) rp;   x = c r + s gate p;   y = w h + bias, h = (x - m) q
// with the mean 0 for an RMS norm, and 1 / r, 1 / q the root of the centred row's mean square plus eps.  Backward, from dx
// of the stream and dy of the norm's result:
//   a = w dy;  D = dx + q (a - mean a - h mean(a h))      (the mean of a for a layer norm alone)
//   dr = c D;  dgate = s sum D p;  e = s gate D;  dwp = sum e hp, dbp = sum e;  f = wp e
//   db = rp (f - mean f - hp mean(f hp));  dw = sum dy h, dbias = sum dy
// Both passes read every row once and keep it in registers; x is made again in the backward from r and b in fp32, as the
// forward had it before its rounding, so that y's gradient is that of the y that was returned.  Sums and statistics are
// fp32.  Bound by memory: forward 4 T n, backward 6 T n elements moved.
//
// A row belongs to WV waves (1, 4 or 8) whose threads hold a piece of 16 bytes to 16 elements.  Workgroups walk the rows with a stride, the
// vectors of their columns in registers (forward) or LDS (backward), the next row read under the arithmetic of one.  The backward's walk a slice of the
// rows of one gate row at a time and leave one partial row of each vector's gradient, added up in a fixed order by a second
// launch: the same inputs give the same bits.
//
// Measured: 8192 x 8192 bf16, both norms RMS, forward 111 to 123 us (4.5 TB/s), backward 151 to 158 (5.2), sums 5; 12,608 x 768
// bf16, layer norm and gate, 18.7 + 24 + 4 us (77 MB and 116 MB); 1001 x 1000 fp32, both layer norms, seven gate rows, 8 + 11 + 5;
// 16 x 4096 forward 5.2.
#pragma once

#include "resnorm_plan.h"
#include "rows.h"

namespace ff {
namespace resnorm {

using norm::Pack;
using norm::Row;
using norm::row_sum;
using norm::threads_of;
using norm::vector_at;

enum Kind { kNone = 0, kRms = 1, kLayer = 2 };

struct Args {
  const void* R;
  const void* B;
  const void* dX;        // backward; NULL: zero
  const void* dY;        // backward, with a norm
  void* X;               // forward: x, backward: dr (NULL: not wanted)
  void* Y;               // forward: y, backward: db (NULL: not wanted)
  int64_t ldr, ldb, lddx, lddy, ldx, ldy;
  int64_t T;
  int n;
  int post, norm;        // Kind
  const void* pw;        // NULL: ones
  const void* pb;        // NULL: zeros
  const void* w;
  const void* b;
  int w_bf16;
  const void* gate;      // NULL: ones
  int64_t ldgate;
  int gate_bf16;
  unsigned group_rows;   // rows of one gate row
  unsigned groups;
  float res, block, post_eps, eps;
  float4* stats;         // [T] (mp, rp, m, q); forward: NULL if not wanted
  // backward
  unsigned slices;       // of all groups; of one: slices / groups
  float* part;           // [workgroups][4][n]: dwp, dbp, dw, dbias of a workgroup's rows (NULL: not wanted)
  float* gate_part;      // [slices][n] (NULL: not wanted)
  float* gate_out;       // dgate itself, where a group is one slice
  int gate_add;
  float4* sums;          // rows too wide for the registers: [T] mean a, mean a h, mean f, mean f hp
};

template <int NV, int KN>
__device__ __forceinline__ void fill(float (&v)[NV][KN], float x) {
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < KN; ++k) v[i][k] = x;
}

// Vector p (absent: none) of a thread's columns; zero where it has no piece.
template <class R, int NV, int KN>
__device__ __forceinline__ void columns(const void* p, int bf16, float none, int l, int n, float (&v)[NV][KN]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (R::skip(i, l, n) < KN) {
      vector_at<KN>(p, bf16, none, R::at(i, l, n), v[i]);
    } else {
#pragma unroll
      for (int k = 0; k < KN; ++k) v[i][k] = 0.f;
    }
  }
}

// A piece of a result.  Of a piece that overlaps the one before only its own elements: the result may lie over an input whose shared
// elements another wave has yet to read, or has written; what is read there in that case enters nothing.
template <class E, bool PART, int KN>
__device__ __forceinline__ void put_own(E* p, const float (&v)[KN], int skip) {
  if (PART && skip) {
#pragma unroll
    for (int k = 1; k < KN; ++k)
      if (k >= skip) p[k] = (E)v[k];
  } else {
    Pack<E>::put(p, v);
  }
}

__device__ __forceinline__ const void* gate_row(const Args& a, int64_t group) {
  return a.gate ? static_cast<const char*>(a.gate) + group * a.ldgate * (a.gate_bf16 ? 2 : 4) : nullptr;
}

// (mean, 1 / deviation) of the values v, which become v - mean.
template <class R, int WV, bool PART, int NV, int KN>
__device__ __forceinline__ float2 centre(float (&v)[NV][KN], int kind, float eps, int l, int n, float2* sh0, float2* sh1) {
  float mean = 0.f;
  if (kind == kLayer) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int skip = R::skip(i, l, n);
#pragma unroll
      for (int k = 0; k < KN; ++k) s += (PART ? k >= skip : skip == 0) ? v[i][k] : 0.f;
    }
    mean = row_sum<WV>(make_float2(s, 0.f), sh0).x / (float)n;
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int skip = R::skip(i, l, n);
#pragma unroll
    for (int k = 0; k < KN; ++k) {
      v[i][k] -= mean;
      q = (PART ? k >= skip : skip == 0) ? fmaf(v[i][k], v[i][k], q) : q;
    }
  }
  const float var = row_sum<WV>(make_float2(q, 0.f), sh1).x / (float)n;
  return make_float2(mean, 1.f / sqrtf(var + eps));
}

template <class E, int NV, int WV, bool PART>
__global__ void __launch_bounds__(threads_of(WV), 2) fwd_kernel(Args a) {
  constexpr int kT = WV * 64, kRows = threads_of(WV) / kT, kN = Pack<E>::kN;
  typedef Row<E, NV, WV, PART> Rw;
  __shared__ float2 sh[2][4][WV];
  const int l = threadIdx.x % kT;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / kT;
  if (t >= a.T) return;      // whole waves; with WV > 1 a workgroup has one row at a time
  Rw r, b;
  r.load(a.R, a.ldr, t, l, a.n);
  b.load(a.B, a.ldb, t, l, a.n);
  float pw[NV][kN], pb[NV][kN], w[NV][kN], bias[NV][kN], gt[NV][kN];
  if (a.post) {
    columns<Rw>(a.pw, a.w_bf16, 1.f, l, a.n, pw);
    columns<Rw>(a.pb, a.w_bf16, 0.f, l, a.n, pb);
  }
  if (a.norm) {
    columns<Rw>(a.w, a.w_bf16, 1.f, l, a.n, w);
    columns<Rw>(a.b, a.w_bf16, 0.f, l, a.n, bias);
  }
  const bool grouped = a.gate && a.groups > 1;
  if (!grouped) columns<Rw>(a.gate, a.gate_bf16, 1.f, l, a.n, gt);
  for (int turn = 0;; turn ^= 1) {
    if (grouped) columns<Rw>(gate_row(a, (unsigned)t / a.group_rows), a.gate_bf16, 1.f, l, a.n, gt);
    float x[NV][kN], p[NV][kN];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      Pack<E>::widen(r.raw[i], x[i]);
      Pack<E>::widen(b.raw[i], p[i]);
    }
    const int64_t next = t + stride;
    if (next < a.T) {
      r.load(a.R, a.ldr, next, l, a.n);
      b.load(a.B, a.ldb, next, l, a.n);
    }
    float2 ps = make_float2(0.f, 0.f), ns = make_float2(0.f, 0.f);
    if (a.post) {
      ps = centre<Rw, WV, PART>(p, a.post, a.post_eps, l, a.n, sh[turn][0], sh[turn][1]);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < kN; ++k) p[i][k] = fmaf(p[i][k] * ps.y, pw[i][k], pb[i][k]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < kN; ++k) x[i][k] = fmaf(a.block * gt[i][k], p[i][k], a.res * x[i][k]);
    E* xo = static_cast<E*>(a.X) + t * a.ldx;
    float y[NV][kN];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < kN; ++k) y[i][k] = x[i][k];
    if (a.norm) ns = centre<Rw, WV, PART>(y, a.norm, a.eps, l, a.n, sh[turn][2], sh[turn][3]);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (Rw::skip(i, l, a.n) < kN) put_own<E, PART>(xo + Rw::at(i, l, a.n), x[i], Rw::skip(i, l, a.n));
    if (a.norm) {
      E* yo = static_cast<E*>(a.Y) + t * a.ldy;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (Rw::skip(i, l, a.n) < kN) {
#pragma unroll
          for (int k = 0; k < kN; ++k) y[i][k] = fmaf(y[i][k] * ns.y, w[i][k], bias[i][k]);
          put_own<E, PART>(yo + Rw::at(i, l, a.n), y[i], Rw::skip(i, l, a.n));
        }
      }
    }
    if (l == 0 && a.stats) a.stats[t] = make_float4(ps.x, ps.y, ns.x, ns.y);
    if (next >= a.T) break;
    t = next;
  }
}

// Vectors of a thread's columns in LDS, in the order in which its row's waves read them back: [piece][quarter of a piece][thread]
// of four floats each.  In registers they cost 16 a vector, and the backward of both norms spilled (8192 x 8192, 590 us for both
// passes).
template <class R, int NV, int KN, int T>
struct Kept {
  static constexpr int kFloats = NV * KN * T;
  float* at;
  __device__ __forceinline__ void put(const void* p, int bf16, float none, float factor, int l, int n) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[KN];
#pragma unroll
      for (int k = 0; k < KN; ++k) v[k] = 0.f;      // zero where there is no piece
      if (R::skip(i, l, n) < KN) vector_at<KN>(p, bf16, none, R::at(i, l, n), v);
#pragma unroll
      for (int k = 0; k < KN; k += 4)
        *reinterpret_cast<float4*>(at + ((i * KN + k) * T + 4 * l)) =
            make_float4(v[k] * factor, v[k + 1] * factor, v[k + 2] * factor, v[k + 3] * factor);
    }
  }
  __device__ __forceinline__ void get(int i, int l, float (&v)[KN]) const {
#pragma unroll
    for (int k = 0; k < KN; k += 4) {
      const float4 q = *reinterpret_cast<const float4*>(at + ((i * KN + k) * T + 4 * l));
      v[k] = q.x, v[k + 1] = q.y, v[k + 2] = q.z, v[k + 3] = q.w;
    }
  }
};

// POST, NORM: there is such a norm.  BIAS: one of them may be a layer norm or have a bias (else both are RMS norms without;
// their code and the sums' registers are left out).  GATE: there is a gate.
template <class E, int NV, int WV, bool PART, bool POST, bool NORM, bool BIAS, bool GATE>
__global__ void __launch_bounds__(threads_of(WV), 2) bwd_kernel(Args a) {
  constexpr int kT = WV * 64, kThreads = threads_of(WV), kRows = kThreads / kT, kN = Pack<E>::kN;
  typedef Row<E, NV, WV, PART> Rw;
  typedef Kept<Rw, NV, kN, kT> Vec;
  constexpr int kVecs = (POST ? (BIAS ? 2 : 1) : 0) + (NORM ? 1 : 0) + (GATE ? 1 : 0);
  __shared__ float2 sh[2][2][WV];
  constexpr int kPlace = NV * kN * kT;
  __shared__ float comb[kRows > 1 ? 2 * kRows * kPlace : 1];
  int side = 0;
  __shared__ __align__(16) float kept[kVecs ? kVecs * Vec::kFloats : 4];
  const int l = threadIdx.x % kT, sub = threadIdx.x / kT;
  const float inv_n = 1.f / (float)a.n;
  const unsigned per_group = a.slices / a.groups;
  const Vec pw{kept}, w{kept + (POST ? 1 : 0) * Vec::kFloats}, gt{kept + ((POST ? 1 : 0) + (NORM ? 1 : 0)) * Vec::kFloats},
      pb{kept + (kVecs - 1) * Vec::kFloats};
  // (the waves of several rows write the same values)
  if constexpr (POST) Vec(pw).put(a.pw, a.w_bf16, 1.f, 1.f, l, a.n);
  if constexpr (POST && BIAS) Vec(pb).put(a.pb, a.w_bf16, 0.f, 1.f, l, a.n);
  if constexpr (NORM) Vec(w).put(a.w, a.w_bf16, 1.f, 1.f, l, a.n);
  // The gate is one row in a slice, so that sums of D hp and of D give its gradient and those of post's vectors.
  float sdh[NV][kN], sd[NV][kN], dw[NV][kN], db[NV][kN];
  if constexpr (NORM) fill(dw, 0.f);
  if constexpr (NORM && BIAS) fill(db, 0.f);
  // a thread's sums of its columns, over the workgroup's rows in a fixed order, to out[n]
  auto flush = [&](const float (&v)[NV][kN], float* out, int add) {
    if constexpr (kRows > 1) {
      // each row's waves their own place; two places in turn, so that a barrier a vector is enough
      float* p = comb + (side ^= 1) * kRows * kPlace;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int skip = Rw::skip(i, l, a.n);
#pragma unroll
        for (int k = 0; k < kN; ++k)
          if (k >= skip) p[sub * kPlace + Rw::at(i, l, a.n) + k] = v[i][k];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.n; c += kThreads) {
        float x = p[c];
#pragma unroll
        for (int q = 1; q < kRows; ++q) x += p[q * kPlace + c];
        out[c] = add ? out[c] + x : x;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int skip = Rw::skip(i, l, a.n), c = Rw::at(i, l, a.n);
#pragma unroll
        for (int k = 0; k < kN; ++k)
          if (k >= skip) out[c + k] = add ? out[c + k] + v[i][k] : v[i][k];
      }
    }
  };
  int turn = 0;
  for (unsigned slice = blockIdx.x; slice < a.slices; slice += gridDim.x) {
    const unsigned group = slice / per_group;
    if constexpr (GATE) {
      if (kRows > 1 && slice != blockIdx.x) __syncthreads();      // every wave is done with the last slice's gate
      Vec(gt).put(gate_row(a, group), a.gate_bf16, 1.f, a.block, l, a.n);
    }
    if constexpr (POST || GATE) fill(sdh, 0.f);
    if constexpr (POST && BIAS) fill(sd, 0.f);
    const int64_t first = (int64_t)group * a.group_rows, end = first + a.group_rows;
    const int64_t stride = (int64_t)per_group * kRows;
    int64_t t = first + (int64_t)(slice - group * per_group) * kRows + sub;
    Rw r, b, dx, dy;
    float4 st_next = make_float4(0.f, 0.f, 0.f, 0.f);
    auto fetch = [&](int64_t row) {
      if (row >= end) return;
      if constexpr (NORM) r.load(a.R, a.ldr, row, l, a.n);
      b.load(a.B, a.ldb, row, l, a.n);
      if (a.dX) dx.load(a.dX, a.lddx, row, l, a.n);
      if constexpr (NORM) dy.load(a.dY, a.lddy, row, l, a.n);
      st_next = a.stats[row];
    };
    fetch(t);
    for (; t < end; t += stride, turn ^= 1) {
      asm volatile("" ::: "memory");       // the vectors are read for every row, not kept in registers over all
      const float4 st = st_next;
      float hp[NV][kN], h[NV][kN], D[NV][kN], f[NV][kN];
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        Pack<E>::widen(b.raw[i], hp[i]);
        if (a.dX) {
          Pack<E>::widen(dx.raw[i], D[i]);
        } else {
#pragma unroll
          for (int k = 0; k < kN; ++k) D[i][k] = 0.f;
        }
        if constexpr (NORM) {
          Pack<E>::widen(r.raw[i], h[i]);
          Pack<E>::widen(dy.raw[i], f[i]);
        }
      }
      fetch(t + stride);
      // p and block gate of piece i
      auto p_of = [&](int i, float (&p)[kN]) {
        float q[kN], c[kN];
        if constexpr (POST) pw.get(i, l, q);
        if constexpr (POST && BIAS) pb.get(i, l, c);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
          if constexpr (!POST) p[k] = hp[i][k];
          else if constexpr (BIAS) p[k] = fmaf(hp[i][k], q[k], c[k]);
          else p[k] = hp[i][k] * q[k];
        }
      };
      auto gate_of = [&](int i, float (&g)[kN]) {
        if constexpr (GATE) gt.get(i, l, g);
        else {
          const float one = Rw::skip(i, l, a.n) < kN ? a.block : 0.f;
#pragma unroll
          for (int k = 0; k < kN; ++k) g[k] = one;
        }
      };
      if constexpr (POST) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int k = 0; k < kN; ++k) hp[i][k] = BIAS ? (hp[i][k] - st.x) * st.y : hp[i][k] * st.y;
      }
      if constexpr (NORM) {
        // a piece that is not there has dy = 0 and zero vectors, so that nothing comes of it
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int skip = Rw::skip(i, l, a.n);
          float p[kN], g[kN], wv[kN];
          p_of(i, p);
          gate_of(i, g);
          w.get(i, l, wv);
#pragma unroll
          for (int k = 0; k < kN; ++k) {
            const float x = fmaf(g[k], p[k], a.res * h[i][k]);
            h[i][k] = (BIAS ? x - st.z : x) * st.w;
            dw[i][k] = fmaf(f[i][k], h[i][k], dw[i][k]);
            if constexpr (BIAS) db[i][k] += f[i][k];
            f[i][k] *= wv[k];
            const float q = !PART || k >= skip ? f[i][k] : 0.f;
            if constexpr (BIAS) s.x += q;
            s.y = fmaf(q, h[i][k], s.y);
          }
        }
        s = row_sum<WV>(s, sh[turn][0]);
        const float ma = BIAS && a.norm == kLayer ? s.x * inv_n : 0.f, mh = s.y * inv_n;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int k = 0; k < kN; ++k) D[i][k] = fmaf(st.w, (BIAS ? f[i][k] - ma : f[i][k]) - h[i][k] * mh, D[i][k]);
      }
      float mf = 0.f, mp = 0.f;
      s = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int skip = Rw::skip(i, l, a.n);
        float g[kN], q[kN];
        gate_of(i, g);
        if constexpr (POST) pw.get(i, l, q);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
          if constexpr (POST || GATE) sdh[i][k] = fmaf(D[i][k], hp[i][k], sdh[i][k]);
          if constexpr (POST && BIAS) sd[i][k] += D[i][k];
          f[i][k] = g[k] * D[i][k];
          if constexpr (POST) {
            f[i][k] *= q[k];
            const float c = !PART || k >= skip ? f[i][k] : 0.f;
            if constexpr (BIAS) s.x += c;
            s.y = fmaf(c, hp[i][k], s.y);
          }
        }
      }
      if constexpr (POST) {
        s = row_sum<WV>(s, sh[turn][1]);
        mf = BIAS && a.post == kLayer ? s.x * inv_n : 0.f;
        mp = s.y * inv_n;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int skip = Rw::skip(i, l, a.n);
        if (skip < kN) {
          const int c = Rw::at(i, l, a.n);
          float o[kN];
          if (a.X) {
#pragma unroll
            for (int k = 0; k < kN; ++k) o[k] = a.res * D[i][k];
            put_own<E, PART>(static_cast<E*>(a.X) + t * a.ldx + c, o, skip);
          }
          if (a.Y) {
#pragma unroll
            for (int k = 0; k < kN; ++k) o[k] = POST ? st.y * (f[i][k] - mf - hp[i][k] * mp) : f[i][k];
            put_own<E, PART>(static_cast<E*>(a.Y) + t * a.ldy + c, o, skip);
          }
        }
      }
    }
    // the sums of the slice: a workgroup's first slice writes its partial rows, later ones (where there are more gate rows than
    // workgroups) add to them
    float* part = a.part + (int64_t)blockIdx.x * 4 * a.n;
    const int later = slice != blockIdx.x;
    if constexpr (GATE) {
      if (a.gate_out || a.gate_part) {
        float dg[NV][kN];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float q[kN], c[kN];
          if constexpr (POST) pw.get(i, l, q);
          if constexpr (POST && BIAS) pb.get(i, l, c);
#pragma unroll
          for (int k = 0; k < kN; ++k) {
            dg[i][k] = POST ? q[k] * sdh[i][k] : sdh[i][k];
            if constexpr (POST && BIAS) dg[i][k] = fmaf(c[k], sd[i][k], dg[i][k]);
            dg[i][k] *= a.block;
          }
        }
        if (a.gate_out) flush(dg, a.gate_out + (int64_t)group * a.n, a.gate_add);
        else flush(dg, a.gate_part + (int64_t)slice * a.n, 0);
      }
    }
    if constexpr (POST) {
      if (a.part) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float g[kN];
          if constexpr (GATE) gt.get(i, l, g);
#pragma unroll
          for (int k = 0; k < kN; ++k) {
            sdh[i][k] *= GATE ? g[k] : a.block;
            if constexpr (BIAS) sd[i][k] *= GATE ? g[k] : a.block;
          }
        }
        flush(sdh, part, later);
        if constexpr (BIAS) flush(sd, part + a.n, later);
      }
    }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 4 * a.n;
  if constexpr (NORM) flush(dw, part + 2 * (int64_t)a.n, 0);
  if constexpr (NORM && BIAS) flush(db, part + 3 * (int64_t)a.n, 0);
}

}  // namespace resnorm
}  // namespace ff
