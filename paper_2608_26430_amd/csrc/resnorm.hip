// Join of two blocks: the calls, the forward's instances, rows of any width, and the sums of the vectors' gradients
// (resnorm.h has the kernels and their formulas).
#include <cmath>
#include <initializer_list>
#include <utility>

#include "resnorm.h"

namespace ff {
namespace resnorm {

// ------------------------------------------------------------------------------------------- rows of any width

// Rows over 8192 elements, and those narrower than a piece: an element a thread and access, a row read up to five times forward (two layer
// norms) and four times backward.  4096 x 12,288 bf16, RMS norms on both sides: forward 305 us, backward 882 (1.3 and 0.7 TB/s of what a
// single reading moves; 4096 x 8192, held in registers, 4.4).

// What a column of a row comes to; the same steps as in the kernels that hold their rows.
template <class E>
struct Column {
  float pw, pb, w, b, gt;
  __device__ __forceinline__ Column(const Args& a, int64_t group, int c) {
    vector_at<1>(a.pw, a.w_bf16, 1.f, c, &pw);
    vector_at<1>(a.pb, a.w_bf16, 0.f, c, &pb);
    vector_at<1>(a.w, a.w_bf16, 1.f, c, &w);
    vector_at<1>(a.b, a.w_bf16, 0.f, c, &b);
    vector_at<1>(gate_row(a, group), a.gate_bf16, 1.f, c, &gt);
    gt *= a.block;
  }
  static __device__ __forceinline__ float get(const void* p, int64_t ld, int64_t t, int c) {
    return (float)static_cast<const E*>(p)[t * ld + c];
  }
  __device__ __forceinline__ float hp(const Args& a, int64_t t, int c, const float4& st) const {
    const float v = get(a.B, a.ldb, t, c);
    return a.post ? (v - st.x) * st.y : v;
  }
  __device__ __forceinline__ float p(const Args& a, float hp) const { return a.post ? fmaf(hp, pw, pb) : hp; }
  __device__ __forceinline__ float x(const Args& a, int64_t t, int c, float p) const {
    return fmaf(gt, p, a.res * get(a.R, a.ldr, t, c));
  }
  __device__ __forceinline__ float D(const Args& a, int64_t t, int c, float h, const float4& st, const float4& sums) const {
    float d = a.dX ? get(a.dX, a.lddx, t, c) : 0.f;
    if (a.norm) d = fmaf(st.w, w * get(a.dY, a.lddy, t, c) - sums.x - h * sums.y, d);
    return d;
  }
};

// (sh[0] and sh[1] take turns, so that the barrier of one sum keeps the other's place until every wave has read it)
struct Sums {
  float2* sh;
  int turn = 0;
  __device__ __forceinline__ float2 operator()(float2 v) {
    turn ^= 1;
    return row_sum<16>(v, sh + 16 * turn);
  }
};

template <class E>
__global__ void __launch_bounds__(1024) fwd_wide_kernel(Args a) {
  __shared__ float2 sh[32];
  Sums total{sh};
  const float n = (float)a.n;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const int64_t group = (unsigned)t / a.group_rows;
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    auto over = [&](auto&& f) {
      float s = 0.f;
      for (int c = threadIdx.x; c < a.n; c += 1024) s += f(c);
      return total(make_float2(s, 0.f)).x / n;
    };
    auto square = [](float v) { return v * v; };
    if (a.post) {
      if (a.post == kLayer) st.x = over([&](int c) { return Column<E>::get(a.B, a.ldb, t, c); });
      st.y = 1.f / sqrtf(over([&](int c) { return square(Column<E>::get(a.B, a.ldb, t, c) - st.x); }) + a.post_eps);
    }
    auto x = [&](const Column<E>& q, int c) { return q.x(a, t, c, q.p(a, q.hp(a, t, c, st))); };
    if (a.norm) {
      if (a.norm == kLayer) st.z = over([&](int c) { return x(Column<E>(a, group, c), c); });
      st.w = 1.f / sqrtf(over([&](int c) { return square(x(Column<E>(a, group, c), c) - st.z); }) + a.eps);
    }
    for (int c = threadIdx.x; c < a.n; c += 1024) {
      const Column<E> q(a, group, c);
      const float v = x(q, c);
      static_cast<E*>(a.X)[t * a.ldx + c] = (E)v;
      if (a.norm) static_cast<E*>(a.Y)[t * a.ldy + c] = (E)fmaf((v - st.z) * st.w, q.w, q.b);
    }
    if (threadIdx.x == 0 && a.stats) a.stats[t] = st;
  }
}

// The four means of each row, ...
template <class E>
__global__ void __launch_bounds__(1024) bwd_wide_sums_kernel(Args a) {
  __shared__ float2 sh[32];
  Sums total{sh};
  const float n = (float)a.n;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const int64_t group = (unsigned)t / a.group_rows;
    const float4 st = a.stats[t];
    float4 sums = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.norm) {
      float2 s = make_float2(0.f, 0.f);
      for (int c = threadIdx.x; c < a.n; c += 1024) {
        const Column<E> q(a, group, c);
        const float h = (q.x(a, t, c, q.p(a, q.hp(a, t, c, st))) - st.z) * st.w;
        const float f = q.w * Column<E>::get(a.dY, a.lddy, t, c);
        s.x += f;
        s.y = fmaf(f, h, s.y);
      }
      s = total(s);
      sums.x = a.norm == kLayer ? s.x / n : 0.f;
      sums.y = s.y / n;
    }
    if (a.post) {
      float2 s = make_float2(0.f, 0.f);
      for (int c = threadIdx.x; c < a.n; c += 1024) {
        const Column<E> q(a, group, c);
        const float hp = q.hp(a, t, c, st), h = (q.x(a, t, c, q.p(a, hp)) - st.z) * st.w;
        const float f = q.gt * q.D(a, t, c, h, st, sums) * q.pw;
        s.x += f;
        s.y = fmaf(f, hp, s.y);
      }
      s = total(s);
      sums.z = a.post == kLayer ? s.x / n : 0.f;
      sums.w = s.y / n;
    }
    if (threadIdx.x == 0) a.sums[t] = sums;
  }
}
// ... the vectors' gradients, a workgroup taking 256 columns at a time of a slice of the rows, ...
template <class E>
__global__ void __launch_bounds__(256) bwd_wide_vectors_kernel(Args a) {
  const unsigned per_group = a.slices / a.groups;
  for (int c = blockIdx.y * 256 + threadIdx.x; c < a.n; c += gridDim.y * 256) {
    float dpw = 0.f, dpb = 0.f, dw = 0.f, db = 0.f;
    for (unsigned slice = blockIdx.x; slice < a.slices; slice += gridDim.x) {
      const unsigned group = slice / per_group;
      const Column<E> q(a, group, c);
      float dg = 0.f;
      const int64_t first = (int64_t)group * a.group_rows, end = first + a.group_rows;
      for (int64_t t = first + (slice - group * per_group); t < end; t += per_group) {
        const float4 st = a.stats[t], sums = a.sums[t];
        const float hp = q.hp(a, t, c, st), p = q.p(a, hp), h = (q.x(a, t, c, p) - st.z) * st.w;
        const float D = q.D(a, t, c, h, st, sums), e = q.gt * D;
        dg = fmaf(a.block * D, p, dg);
        dpw = fmaf(e, hp, dpw);
        dpb += e;
        if (a.norm) {
          const float dy = Column<E>::get(a.dY, a.lddy, t, c);
          dw = fmaf(dy, h, dw);
          db += dy;
        }
      }
      if (a.gate_out) {
        float* o = a.gate_out + (int64_t)group * a.n + c;
        *o = a.gate_add ? *o + dg : dg;
      } else if (a.gate_part) {
        a.gate_part[(int64_t)slice * a.n + c] = dg;
      }
    }
    if (!a.part) continue;
    float* part = a.part + (int64_t)blockIdx.x * 4 * a.n;
    part[c] = dpw;
    part[a.n + (int64_t)c] = dpb;
    part[2 * (int64_t)a.n + c] = dw;
    part[3 * (int64_t)a.n + c] = db;
  }
}
// ... and then the rows (dr may be dx, db may be dy)
template <class E>
__global__ void __launch_bounds__(1024) bwd_wide_kernel(Args a) {
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const int64_t group = (unsigned)t / a.group_rows;
    const float4 st = a.stats[t], sums = a.sums[t];
    for (int c = threadIdx.x; c < a.n; c += 1024) {
      const Column<E> q(a, group, c);
      const float hp = q.hp(a, t, c, st), h = (q.x(a, t, c, q.p(a, hp)) - st.z) * st.w;
      const float D = q.D(a, t, c, h, st, sums), e = q.gt * D;
      if (a.X) static_cast<E*>(a.X)[t * a.ldx + c] = (E)(a.res * D);
      if (a.Y) static_cast<E*>(a.Y)[t * a.ldy + c] = (E)(a.post ? st.y * (e * q.pw - sums.z - hp * sums.w) : e);
    }
  }
}

// ------------------------------------------------------------------------------------------- sums

struct SumArgs {
  const float* part;       // [rows][4][n]
  int rows;
  float* out[4];
  const float* gate_part;  // [groups][gate_rows][n] (NULL: none)
  int gate_rows;
  float* gate;             // [groups][n]
  int n, add;
};

// out = [out +] sum over the partial rows, in a fixed order: 32 columns x 32 shares of the rows per workgroup.  blockIdx.y: the
// vectors that are wanted, then the gate's rows.
__global__ void __launch_bounds__(kSumThreads) sum_kernel(SumArgs a, int vectors) {
  __shared__ float sh[32][33];
  const int k = threadIdx.x & 31, q = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + k;
  const float* p;
  int64_t stride;
  int rows;
  float* out = nullptr;
  if ((int)blockIdx.y < vectors) {
    int v = 0;
    for (int seen = -1; v < 4; ++v)
      if (a.out[v] && ++seen == (int)blockIdx.y) break;
    out = a.out[v < 4 ? v : 0];
    p = a.part + (int64_t)v * a.n;
    stride = 4 * (int64_t)a.n;
    rows = a.rows;
  } else {
    const int64_t group = blockIdx.y - vectors;
    p = a.gate_part + group * a.gate_rows * a.n;
    stride = a.n;
    rows = a.gate_rows;
    out = a.gate + group * a.n;
  }
  float s = 0.f;
  if (c < a.n) {
#pragma unroll 8
    for (int r = q; r < rows; r += 32) s += p[r * stride + c];
  }
  sh[q][k] = s;
  __syncthreads();
  if (q || c >= a.n) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) s += sh[i][k];
  out[c] = a.add ? out[c] + s : s;
}

// ------------------------------------------------------------------------------------------- dispatch

// 0: both norms RMS without bias, 1: both, 2: norm alone, RMS without bias, 3: norm alone, 4: post alone, 5: none
#define RESNORM_INST(c) \
  hipError_t launch_bwd_##c##_0(const Args&, const Shape&, unsigned, hipStream_t); \
  hipError_t launch_bwd_##c##_1(const Args&, const Shape&, unsigned, hipStream_t);
RESNORM_INST(0) RESNORM_INST(1) RESNORM_INST(2) RESNORM_INST(3) RESNORM_INST(4) RESNORM_INST(5)

namespace {

template <class E, int NV, int WV>
void launch_fwd(const Args& a, const Shape& sh, unsigned groups, hipStream_t s) {
  const dim3 grid(groups), block(threads_of(WV));
  if (sh.part) hipLaunchKernelGGL((fwd_kernel<E, NV, WV, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((fwd_kernel<E, NV, WV, false>), grid, block, 0, s, a);
}

template <class E>
hipError_t run_fwd(const Args& a, hipStream_t s) {
  const Shape sh = shape_of(a.n, (int)sizeof(E), a.T, false);
  constexpr int k = 16 / Pack<E>::kN;
  const unsigned groups = (unsigned)fwd_groups(a.T, sh);
  if (sh.wv == 0) {
    hipLaunchKernelGGL(fwd_wide_kernel<E>, dim3((unsigned)(a.T < (1 << 20) ? a.T : (1 << 20))), dim3(1024), 0, s, a);
  } else if (sh.wv == 1 && sh.nv < k) {
    launch_fwd<E, k / 2, 1>(a, sh, groups, s);
  } else if (sh.wv == 1) {
    launch_fwd<E, k, 1>(a, sh, groups, s);
  } else if (sh.wv == 4 && sh.nv < k) {
    launch_fwd<E, 1, 4>(a, sh, groups, s);
  } else if (sh.wv == 4) {
    launch_fwd<E, k, 4>(a, sh, groups, s);
  } else {
    launch_fwd<E, k, 8>(a, sh, groups, s);
  }
  return hipGetLastError();
}

hipError_t run_bwd(const Args& a, const Shape& sh, bool bias, unsigned groups, bool bf16, hipStream_t s) {
  if (sh.wv == 0) {
    // a launch has fewer than 2^32 threads
    const dim3 rows((unsigned)(a.T < (1 << 20) ? a.T : (1 << 20)));
    const dim3 columns(groups, (unsigned)(a.n < (1 << 20) ? (a.n + 255) / 256 : 4096));
    if (bf16) {
      hipLaunchKernelGGL(bwd_wide_sums_kernel<__bf16>, rows, dim3(1024), 0, s, a);
      if (a.part || a.gate_part || a.gate_out) hipLaunchKernelGGL(bwd_wide_vectors_kernel<__bf16>, columns, dim3(256), 0, s, a);
      hipLaunchKernelGGL(bwd_wide_kernel<__bf16>, rows, dim3(1024), 0, s, a);
    } else {
      hipLaunchKernelGGL(bwd_wide_sums_kernel<float>, rows, dim3(1024), 0, s, a);
      if (a.part || a.gate_part || a.gate_out) hipLaunchKernelGGL(bwd_wide_vectors_kernel<float>, columns, dim3(256), 0, s, a);
      hipLaunchKernelGGL(bwd_wide_kernel<float>, rows, dim3(1024), 0, s, a);
    }
    return hipGetLastError();
  }
  typedef hipError_t (*Launch)(const Args&, const Shape&, unsigned, hipStream_t);
  static const Launch launches[2][6] = {
      {launch_bwd_0_0, launch_bwd_1_0, launch_bwd_2_0, launch_bwd_3_0, launch_bwd_4_0, launch_bwd_5_0},
      {launch_bwd_0_1, launch_bwd_1_1, launch_bwd_2_1, launch_bwd_3_1, launch_bwd_4_1, launch_bwd_5_1}};
  const int combo = a.norm ? (a.post ? 0 : 2) + bias : (a.post ? 4 : 5);
  return launches[bf16][combo](a, sh, groups, s);
}

ff_status check_rows(const char* name, const void* p, int64_t ld, int64_t n, int esz) {
  if (!p) return fail(FF_EINVAL, "%s is NULL", name);
  if (ld < n) return fail(FF_EINVAL, "leading dimension of %s (%lld) < %lld", name, (long long)ld, (long long)n);
  if ((uintptr_t)p % esz) return fail(FF_EINVAL, "%s is misaligned", name);
  return FF_OK;
}

ff_status check_sizes(int64_t T, int64_t n, int64_t groups) {
  if (T < 0 || T > ((int64_t)1 << 30) || n < 1 || n > ((int64_t)1 << 24))
    return fail(FF_EINVAL, "T=%lld or n=%lld out of range", (long long)T, (long long)n);
  if (groups < 1 || groups > ((int64_t)1 << 30) || T % groups)
    return fail(FF_EINVAL, "groups=%lld must divide T=%lld", (long long)groups, (long long)T);
  return FF_OK;
}

// Outputs of rows of n fp32 each, NULL for none: two that share memory would have two writers.
struct Out {
  const float* p;
  int64_t rows;
};
ff_status check_apart(int64_t n, std::initializer_list<Out> outs) {
  for (const Out* a = outs.begin(); a != outs.end(); ++a)
    for (const Out* b = outs.begin(); b != a; ++b)
      if (a->p && b->p && (uintptr_t)a->p < (uintptr_t)b->p + (uintptr_t)(4 * n * b->rows) &&
          (uintptr_t)b->p < (uintptr_t)a->p + (uintptr_t)(4 * n * a->rows))
        return fail(FF_EINVAL, "two vectors' gradients share memory");
  return FF_OK;
}

ff_status fill_args(const ff_resnorm* d, Args* a) {
  if (!d) return fail(FF_EINVAL, "the description is NULL");
  if (d->act != FF_F32 && d->act != FF_BF16) return fail(FF_EINVAL, "unknown activation dtype %d", d->act);
  if (d->w_dtype != FF_F32 && d->w_dtype != FF_BF16) return fail(FF_EINVAL, "unknown weight dtype %d", d->w_dtype);
  if (d->gate_dtype != FF_F32 && d->gate_dtype != FF_BF16) return fail(FF_EINVAL, "unknown gate dtype %d", d->gate_dtype);
  if (d->post < FF_NORM_NONE || d->post > FF_NORM_LAYER || d->norm < FF_NORM_NONE || d->norm > FF_NORM_LAYER)
    return fail(FF_EINVAL, "unknown norms %d, %d", d->post, d->norm);
  const int64_t groups = d->gate ? d->groups : 1;
  const ff_status st = check_sizes(d->T, d->n, groups);
  if (st != FF_OK) return st;
  if (!(d->post_eps >= 0.f) || !std::isfinite(d->post_eps) || !(d->eps >= 0.f) || !std::isfinite(d->eps))
    return fail(FF_EINVAL, "post_eps and eps must be finite and >= 0");
  if (!std::isfinite(d->res_scale) || !std::isfinite(d->block_scale)) return fail(FF_EINVAL, "the scales must be finite");
  const int wsz = d->w_dtype == FF_BF16 ? 2 : 4, gsz = d->gate_dtype == FF_BF16 ? 2 : 4;
  if ((uintptr_t)d->post_weight % wsz || (uintptr_t)d->post_bias % wsz || (uintptr_t)d->weight % wsz ||
      (uintptr_t)d->bias % wsz || (uintptr_t)d->gate % gsz)
    return fail(FF_EINVAL, "a vector or the gate is misaligned");
  if (d->gate && groups > 1 && d->ldgate < d->n)
    return fail(FF_EINVAL, "leading dimension of gate (%lld) < %lld", (long long)d->ldgate, (long long)d->n);
  a->T = d->T, a->n = (int)d->n, a->post = d->post, a->norm = d->norm, a->w_bf16 = d->w_dtype == FF_BF16;
  if (d->post) a->pw = d->post_weight, a->pb = d->post_bias;
  if (d->norm) a->w = d->weight, a->b = d->bias;
  a->gate = d->gate, a->ldgate = d->ldgate, a->gate_bf16 = d->gate_dtype == FF_BF16;
  a->groups = (unsigned)groups, a->group_rows = (unsigned)(d->T / groups);
  a->res = d->res_scale, a->block = d->block_scale, a->post_eps = d->post_eps, a->eps = d->eps;
  return FF_OK;
}

}  // namespace
}  // namespace resnorm
}  // namespace ff

#define RESNORM_CHECK(call)              \
  do {                                   \
    const ff_status st_ = (call);        \
    if (st_ != FF_OK) return st_;        \
  } while (0)

extern "C" {

ff_status ff_resnorm_fwd(const ff_resnorm* d, const void* R, int64_t ldr, const void* B, int64_t ldb, void* X, int64_t ldx,
                         void* Y, int64_t ldy, float* stats, void* stream) {
  using namespace ff::resnorm;
  ff::clear_error();
  Args a{};
  RESNORM_CHECK(fill_args(d, &a));
  if (a.T == 0) return FF_OK;
  const int esz = d->act == FF_BF16 ? 2 : 4;
  RESNORM_CHECK(check_rows("R", R, ldr, d->n, esz));
  RESNORM_CHECK(check_rows("B", B, ldb, d->n, esz));
  RESNORM_CHECK(check_rows("X", X, ldx, d->n, esz));
  if (d->norm) RESNORM_CHECK(check_rows("Y", Y, ldy, d->n, esz));
  if (X == R && a.T > 1 && ldx != ldr) return ff::fail(FF_EINVAL, "X over R needs the same leading dimension");
  if (d->norm && X == Y) return ff::fail(FF_EINVAL, "X and Y are the same memory");
  if ((uintptr_t)stats % 16) return ff::fail(FF_EINVAL, "stats is not 16-byte aligned");
  a.R = R, a.ldr = ldr, a.B = B, a.ldb = ldb, a.X = X, a.ldx = ldx, a.Y = Y, a.ldy = ldy;
  a.stats = reinterpret_cast<float4*>(stats);
  const hipError_t e = d->act == FF_BF16 ? run_fwd<__bf16>(a, (hipStream_t)stream) : run_fwd<float>(a, (hipStream_t)stream);
  return e == hipSuccess ? FF_OK : ff::fail(FF_EDEVICE, "join forward: %s", hipGetErrorString(e));
}

ff_status ff_resnorm_workspace(int64_t T, int64_t n, int64_t groups, int64_t* bytes) {
  using namespace ff::resnorm;
  ff::clear_error();
  RESNORM_CHECK(check_sizes(T, n, groups));
  if (!bytes) return ff::fail(FF_EINVAL, "bytes is NULL");
  *bytes = space_of(T, n, groups, shape_of(n, 2, T, true).wv == 0 || shape_of(n, 4, T, true).wv == 0).bytes;
  return FF_OK;
}

ff_status ff_resnorm_bwd(const ff_resnorm* d, const void* R, int64_t ldr, const void* B, int64_t ldb, const void* dX,
                         int64_t lddx, const void* dY, int64_t lddy, const float* stats, void* dR, int64_t lddr, void* dB,
                         int64_t lddb, int accumulate, float* dgate, float* dpost_weight, float* dpost_bias, float* dweight,
                         float* dbias, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace ff::resnorm;
  ff::clear_error();
  Args a{};
  RESNORM_CHECK(fill_args(d, &a));
  if (!d->gate && dgate) return ff::fail(FF_EINVAL, "dgate without a gate");
  if ((!d->post && (dpost_weight || dpost_bias)) || (!d->norm && (dweight || dbias)))
    return ff::fail(FF_EINVAL, "gradients of a norm that is not there");
  if ((uintptr_t)dgate % 4 || (uintptr_t)dpost_weight % 4 || (uintptr_t)dpost_bias % 4 || (uintptr_t)dweight % 4 ||
      (uintptr_t)dbias % 4)
    return ff::fail(FF_EINVAL, "a vector's gradient is misaligned");
  RESNORM_CHECK(check_apart(d->n, {{dgate, a.groups}, {dpost_weight, 1}, {dpost_bias, 1}, {dweight, 1}, {dbias, 1}}));
  const bool vectors = dpost_weight || dpost_bias || dweight || dbias;
  const bool bf16 = d->act == FF_BF16;
  const Shape sh = shape_of(d->n, bf16 ? 2 : 4, d->T, true);
  unsigned groups = 0, per_group = 0;
  const hipStream_t s = (hipStream_t)stream;
  if (a.T > 0) {
    const int esz = bf16 ? 2 : 4;
    RESNORM_CHECK(check_rows("R", R, ldr, d->n, esz));
    RESNORM_CHECK(check_rows("B", B, ldb, d->n, esz));
    if (dX) RESNORM_CHECK(check_rows("dX", dX, lddx, d->n, esz));
    if (d->norm) RESNORM_CHECK(check_rows("dY", dY, lddy, d->n, esz));
    if (dR) RESNORM_CHECK(check_rows("dR", dR, lddr, d->n, esz));
    if (dB) RESNORM_CHECK(check_rows("dB", dB, lddb, d->n, esz));
    for (const auto& [p, ld] : {std::make_pair(dR, lddr), std::make_pair(dB, lddb)})
      if (p && a.T > 1 && ((p == R && ld != ldr) || (p == B && ld != ldb) || (p == dX && ld != lddx) || (d->norm && p == dY && ld != lddy)))
        return ff::fail(FF_EINVAL, "dR or dB over R, B, dX or dY needs the same leading dimension");
    if (dR && dR == dB) return ff::fail(FF_EINVAL, "dR and dB are the same memory");
    if (!stats || (uintptr_t)stats % 16) return ff::fail(FF_EINVAL, "stats is NULL or not 16-byte aligned");
    const Space at = space_of(a.T, d->n, a.groups, sh.wv == 0);
    if (vectors || dgate || sh.wv == 0) {
      if (!workspace || (uintptr_t)workspace % 256) return ff::fail(FF_EINVAL, "the workspace is NULL or not 256-byte aligned");
      if (workspace_bytes < at.bytes)
        return ff::fail(FF_EINVAL, "the workspace holds %lld bytes, the call needs %lld", (long long)workspace_bytes,
                        (long long)at.bytes);
    }
    char* ws = static_cast<char*>(workspace);
    const int64_t per = slices_of(a.group_rows, a.groups, d->n, sh.wv == 1 ? 4 : 1), slices = per * a.groups;
    per_group = (unsigned)per;
    a.slices = (unsigned)slices;
    groups = (unsigned)(slices < most_groups(d->n) ? slices : most_groups(d->n));
    a.R = R, a.ldr = ldr, a.B = B, a.ldb = ldb, a.dX = dX, a.lddx = lddx, a.dY = dY, a.lddy = lddy;
    a.X = dR, a.ldx = lddr, a.Y = dB, a.ldy = lddb;
    a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
    if (vectors) a.part = reinterpret_cast<float*>(ws);
    if (dgate && per_group == 1) a.gate_out = dgate, a.gate_add = accumulate;
    else if (dgate) a.gate_part = reinterpret_cast<float*>(ws + at.gate);
    if (sh.wv == 0) a.sums = reinterpret_cast<float4*>(ws + at.sums);
    const bool bias = d->post == FF_NORM_LAYER || d->norm == FF_NORM_LAYER || a.pb || dpost_bias || dbias;
    const hipError_t e = run_bwd(a, sh, bias, groups, bf16, s);
    if (e != hipSuccess) return ff::fail(FF_EDEVICE, "join backward: %s", hipGetErrorString(e));
  }
  const int nv = !!dpost_weight + !!dpost_bias + !!dweight + !!dbias;
  // (with T = 0 there are no partial rows: the sums are zero)
  const bool gate_sum = dgate && per_group != 1;
  for (int64_t g0 = 0, ng = 0;; g0 += ng) {
    const int v = g0 == 0 ? nv : 0;
    ng = gate_sum ? sum_rows(d->n, v, a.groups - g0) : 0;
    if (v + ng == 0) break;
    SumArgs q{a.part, (int)groups, {dpost_weight, dpost_bias, dweight, dbias},
              a.gate_part ? a.gate_part + g0 * per_group * d->n : nullptr, (int)per_group, dgate ? dgate + g0 * d->n : nullptr,
              a.n, accumulate};
    hipLaunchKernelGGL(sum_kernel, dim3((unsigned)sum_blocks(d->n), (unsigned)(v + ng)), dim3(kSumThreads), 0, s, q, v);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return ff::fail(FF_EDEVICE, "join backward: %s", hipGetErrorString(e));
    if (!gate_sum) break;
  }
  return FF_OK;
}

}  // extern "C"
