// Gated feed-forward, forward and backward: the calls (glu_gemm.h has the kernels and their formulas, glu_plan.h the choice of
// tiles).
//
// A forward is one kernel.  A backward makes dG and dU first, element by element from the kept G and U or, without them, in the
// forward's kernel with another end; then dX as one sum over both halves of 2 F, and dWg and dWu in one launch.  dG and dU are
// rounded to the activations' type once, as the results that they are, and the products read them so.  Products accumulate in fp32;
// where a sum is split, its parts are added up in a fixed order.
#include <cmath>

#include "glu_gemm.h"
#include "glu_plan.h"

namespace ff {
namespace glu {

#define GLU_PROJ(p)                                                                       \
  hipError_t launch_projection_##p##_0(int, int, int, const ProjArgs&, hipStream_t);      \
  hipError_t launch_projection_##p##_1(int, int, int, const ProjArgs&, hipStream_t);      \
  hipError_t launch_point_##p##_0(const PointArgs&, hipStream_t);                         \
  hipError_t launch_point_##p##_1(const PointArgs&, hipStream_t);
GLU_PROJ(0) GLU_PROJ(1) GLU_PROJ(2)
#define GLU_GRAD(p)                                                       \
  hipError_t launch_gradient_##p##_0(int, const GradArgs&, hipStream_t);  \
  hipError_t launch_gradient_##p##_1(int, const GradArgs&, hipStream_t);
GLU_GRAD(3) GLU_GRAD(4)

hipError_t launch_projection(int bf16, int fn, int mode, int tile, int ks, const ProjArgs& a, hipStream_t s) {
  typedef hipError_t (*Launch)(int, int, int, const ProjArgs&, hipStream_t);
  static const Launch launches[3][2] = {{launch_projection_0_0, launch_projection_0_1},
                                        {launch_projection_1_0, launch_projection_1_1},
                                        {launch_projection_2_0, launch_projection_2_1}};
  return launches[fn][bf16](mode, tile, ks, a, s);
}
hipError_t launch_point(int bf16, int fn, const PointArgs& a, hipStream_t s) {
  typedef hipError_t (*Launch)(const PointArgs&, hipStream_t);
  static const Launch launches[3][2] = {{launch_point_0_0, launch_point_0_1}, {launch_point_1_0, launch_point_1_1},
                                        {launch_point_2_0, launch_point_2_1}};
  return launches[fn][bf16](a, s);
}
hipError_t launch_gradient(int bf16, int trb, int tile, const GradArgs& a, hipStream_t s) {
  if (trb) return bf16 ? launch_gradient_4_1(tile, a, s) : launch_gradient_4_0(tile, a, s);
  return bf16 ? launch_gradient_3_1(tile, a, s) : launch_gradient_3_0(tile, a, s);
}

namespace {

constexpr int64_t kLaunchItems = (int64_t)1 << 31;   // threads of a launch, at most (it has fewer than 2^32)

// out = beta out + sum over the splits of part[split][rows][M], four elements a thread; rows from `half` on are the second
// result's.
template <class E>
__global__ void __launch_bounds__(256) sum_kernel(const float* part, int splits, int64_t rows, int64_t half, int M, float beta,
                                                  E* out0, E* out1, int64_t ldo, int64_t first, int64_t items) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= items) return;
  const int64_t item = first + at;
  const unsigned m4 = (unsigned)M / 4;
  const int64_t row = item <= 0xffffffffll ? (int64_t)((unsigned)item / m4) : item / m4;
  const int c = (int)(item - row * m4) * 4;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  const float* p = part + row * M + c;
#pragma unroll 8
  for (int s = 0; s < splits; ++s) v += load4(p + (int64_t)s * rows * M);
  E* o = (row < half ? out0 + row * ldo : out1 + (row - half) * ldo) + c;
  if (beta != 0.f) v += beta * load4(o);
  store4(o, v);
}

hipError_t run_sum(bool bf16, const float* part, int splits, int64_t rows, int64_t half, int64_t M, float beta, void* out0,
                   void* out1, int64_t ldo, hipStream_t s) {
  const int64_t items = rows * (M / 4);
  for (int64_t first = 0; first < items; first += kLaunchItems) {
    const int64_t n = items - first < kLaunchItems ? items - first : kLaunchItems;
    const dim3 grid((unsigned)((n + 255) / 256));
    if (bf16)
      hipLaunchKernelGGL(sum_kernel<__bf16>, grid, dim3(256), 0, s, part, splits, rows, half, (int)M, beta, (__bf16*)out0,
                         (__bf16*)out1, ldo, first, n);
    else
      hipLaunchKernelGGL(sum_kernel<float>, grid, dim3(256), 0, s, part, splits, rows, half, (int)M, beta, (float*)out0,
                         (float*)out1, ldo, first, n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

struct Call {
  int64_t T, n, F;
  bool bf16;
  int fn;
};

hipError_t run_projection(const Call& c, int mode, const ProjArgs& call, hipStream_t s) {
  const Parts p = projection(c.T, c.n, c.F, c.bf16);
  const int esz = c.bf16 ? 2 : 4, kk = kk_of(esz);
  for (int i = 0; i < p.count; ++i) {
    const Part& q = p.part[i];
    const int bm = tile_m(q.tile) / 2, bn = tile_n(q.tile);
    auto in = [&](const void* x, int64_t ld) { return x ? static_cast<const char*>(x) + q.t0 * ld * esz : nullptr; };
    auto out = [&](void* x, int64_t ld) { return x ? static_cast<char*>(x) + q.t0 * ld * esz : nullptr; };
    ProjArgs a = call;
    a.X = in(a.X, a.ldx), a.Ag = in(a.Ag, a.lda), a.Au = in(a.Au, a.lda), a.dH = in(a.dH, a.lddh);
    a.H = out(a.H, a.ldh), a.G = out(a.G, a.ldg), a.U = out(a.U, a.ldg);
    a.F = (int)c.F, a.T = (int)q.T, a.n = (int)c.n;
    a.tm = (int)(up(c.F, bm) / bm), a.tn = (int)(up(q.T, bn) / bn), a.kt = (int)(up(c.n, kk) / kk);
    a.rest = q.ks ? 0 : rest_of(q.tile, (int64_t)a.tm * a.tn);
    const hipError_t e = launch_projection(c.bf16, c.fn, mode, q.tile, q.ks, a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t run_point(const Call& c, PointArgs a, hipStream_t s) {
  a.pieces = (int)(c.F / (c.bf16 ? 8 : 4));
  const int64_t all = c.T * a.pieces;
  for (int64_t first = 0; first < all; first += kLaunchItems) {
    a.first = first, a.items = all - first < kLaunchItems ? all - first : kLaunchItems;
    const hipError_t e = launch_point(c.bf16, c.fn, a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// trb: dW; otherwise dX
hipError_t run_gradient(const Call& c, bool trb, const Parts& p, const GradArgs& call, float* ws, hipStream_t s) {
  const int esz = c.bf16 ? 2 : 4, kk = kk_of(esz);
  for (int i = 0; i < p.count; ++i) {
    const Part& q = p.part[i];
    const int bm = tile_m(q.tile), bn = tile_n(q.tile);
    const int64_t K = trb ? c.T : c.F;
    GradArgs a = call;
    for (int h = 0; h < 2; ++h) {
      // a part's rows: tokens of dG and dU, or their columns
      a.B[h] = static_cast<const char*>(a.B[h]) + q.t0 * (trb ? 1 : a.ldb) * esz;
      a.out[h] = static_cast<char*>(a.out[h]) + q.t0 * a.ldo * esz;
    }
    a.M = (int)c.n, a.N = (int)q.T, a.K = (int)K;
    a.tm = (int)(up(c.n, bm) / bm), a.tn = (int)(up(q.T, bn) / bn);
    a.kt = (int)(up(K, kk) / kk), a.kt_split = q.kt_split, a.splits = q.splits;
    a.rest = rest_of(q.tile, (int64_t)a.tm * a.tn * (trb ? 2 : 1) * a.splits);
    a.part = ws;
    hipError_t e = launch_gradient(c.bf16, trb, q.tile, a, s);
    if (e == hipSuccess && q.splits > 1)
      e = run_sum(c.bf16, ws, q.splits, trb ? 2 * q.T : q.T, q.T, c.n, a.beta, a.out[0], a.out[1], a.ldo, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------- argument checks

ff_status check_sizes(int64_t T, int64_t n, int64_t F, int act, int fn) {
  if (act != FF_F32 && act != FF_BF16) return fail(FF_EINVAL, "unknown activation dtype %d", act);
  if (fn < FF_GLU_SILU || fn > FF_GLU_GELU_TANH) return fail(FF_EINVAL, "unknown function %d", fn);
  const int64_t mult = act == FF_BF16 ? 8 : 4, most = (int64_t)1 << 18;
  if (T < 0 || T > ((int64_t)1 << 28)) return fail(FF_EINVAL, "T=%lld out of range", (long long)T);
  if (n < mult || n > most || n % mult || F < mult || F > most || F % mult)
    return fail(FF_EINVAL, "n=%lld and F=%lld must be multiples of %lld, at most 262144", (long long)n, (long long)F,
                (long long)mult);
  return FF_OK;
}

ff_status check_rows(const char* name, const void* p, int64_t ld, int64_t n, int act) {
  const int64_t mult = act == FF_BF16 ? 8 : 4;
  if (!p) return fail(FF_EINVAL, "%s is NULL", name);
  if (ld < n || ld > xent::kMaxLd || ld % mult)
    return fail(FF_EINVAL, "leading dimension of %s (%lld) must be a multiple of %lld, from %lld to 1048576", name,
                (long long)ld, (long long)mult, (long long)n);
  if ((uintptr_t)p % 16) return fail(FF_EINVAL, "%s is not 16-byte aligned", name);
  return FF_OK;
}

#define GLU_CHECK(call)                  \
  do {                                   \
    const ff_status st_ = (call);        \
    if (st_ != FF_OK) return st_;        \
  } while (0)

ff_status check_inputs(const Call& c, int act, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw,
                       const void* Ag, const void* Au, int64_t lda) {
  GLU_CHECK(check_rows("X", X, ldx, c.n, act));
  GLU_CHECK(check_rows("Wg", Wg, ldw, c.n, act));
  GLU_CHECK(check_rows("Wu", Wu, ldw, c.n, act));
  if (Ag) GLU_CHECK(check_rows("Ag", Ag, lda, c.F, act));
  if (Au) GLU_CHECK(check_rows("Au", Au, lda, c.F, act));
  return FF_OK;
}

ff_status done(hipError_t e, const char* what) {
  return e == hipSuccess ? FF_OK : fail(FF_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace
}  // namespace glu
}  // namespace ff

extern "C" {

ff_status ff_glu_fwd(int64_t T, int64_t n, int64_t F, int act, int fn, const void* X, int64_t ldx, const void* Wg,
                     const void* Wu, int64_t ldw, const void* Ag, const void* Au, int64_t lda, void* H, int64_t ldh, void* G,
                     void* U, int64_t ldg, void* stream) {
  using namespace ff::glu;
  ff::clear_error();
  GLU_CHECK(check_sizes(T, n, F, act, fn));
  if (T == 0) return FF_OK;
  const Call c{T, n, F, act == FF_BF16, fn};
  GLU_CHECK(check_inputs(c, act, X, ldx, Wg, Wu, ldw, Ag, Au, lda));
  GLU_CHECK(check_rows("H", H, ldh, F, act));
  if (!G != !U) return ff::fail(FF_EINVAL, "G and U are kept together");
  if (G) {
    GLU_CHECK(check_rows("G", G, ldg, F, act));
    GLU_CHECK(check_rows("U", U, ldg, F, act));
    if (G == U || G == H || U == H) return ff::fail(FF_EINVAL, "two of H, G and U are the same memory");
  }
  ProjArgs a{};
  a.Wg = Wg, a.Wu = Wu, a.X = X, a.ldw = ldw, a.ldx = ldx, a.Ag = Ag, a.Au = Au, a.lda = lda;
  a.H = H, a.ldh = ldh, a.G = G, a.U = U, a.ldg = ldg;
  return done(run_projection(c, kForward, a, (hipStream_t)stream), "gated feed-forward");
}

ff_status ff_glu_workspace(int64_t T, int64_t n, int64_t F, int act, int want, int64_t* bytes) {
  using namespace ff::glu;
  ff::clear_error();
  GLU_CHECK(check_sizes(T, n, F, act, FF_GLU_SILU));
  if (want < 0 || want > (FF_GLU_DX | FF_GLU_DW)) return ff::fail(FF_EINVAL, "unknown outputs %d", want);
  if (!bytes) return ff::fail(FF_EINVAL, "bytes is NULL");
  Parts dx{}, dw{};
  if (T && (want & FF_GLU_DX)) dx = dx_product(T, n, F, act == FF_BF16);
  if (T && (want & FF_GLU_DW)) dw = dw_product(T, n, F, act == FF_BF16);
  *bytes = workspace(n, &dx, &dw);
  return FF_OK;
}

ff_status ff_glu_bwd(int64_t T, int64_t n, int64_t F, int act, int fn, const void* dH, int64_t lddh, const void* X, int64_t ldx,
                     const void* Wg, const void* Wu, int64_t ldw, const void* Ag, const void* Au, int64_t lda, const void* G,
                     const void* U, int64_t ldg, void* dG, void* dU, int64_t lddg, float beta_dx, void* dX, int64_t lddx,
                     float beta_dw, void* dWg, void* dWu, int64_t lddw, void* ws, int64_t workspace_bytes, void* stream) {
  using namespace ff::glu;
  ff::clear_error();
  GLU_CHECK(check_sizes(T, n, F, act, fn));
  if (!G != !U) return ff::fail(FF_EINVAL, "G and U are kept together");
  if (!dWg != !dWu) return ff::fail(FF_EINVAL, "dWg and dWu are made together");
  if (dWg && dWg == dWu) return ff::fail(FF_EINVAL, "dWg and dWu are the same memory");
  const Call c{T, n, F, act == FF_BF16, fn};
  const hipStream_t s = (hipStream_t)stream;
  if (dWg) {
    GLU_CHECK(check_rows("dWg", dWg, lddw, n, act));
    GLU_CHECK(check_rows("dWu", dWu, lddw, n, act));
  }
  if (T == 0) {
    if (!dWg) return FF_OK;
    hipError_t e = run_sum(c.bf16, nullptr, 0, 2 * F, F, n, beta_dw, dWg, dWu, lddw, s);
    return done(e, "gated feed-forward backward");
  }
  GLU_CHECK(check_rows("dH", dH, lddh, F, act));
  if (G) {
    GLU_CHECK(check_rows("G", G, ldg, F, act));
    GLU_CHECK(check_rows("U", U, ldg, F, act));
    // X for the weights' gradients alone, the weights for dX
    if (dWg) GLU_CHECK(check_rows("X", X, ldx, n, act));
    if (dX) {
      GLU_CHECK(check_rows("Wg", Wg, ldw, n, act));
      GLU_CHECK(check_rows("Wu", Wu, ldw, n, act));
    }
  } else {
    GLU_CHECK(check_inputs(c, act, X, ldx, Wg, Wu, ldw, Ag, Au, lda));
  }
  GLU_CHECK(check_rows("dG", dG, lddg, F, act));
  GLU_CHECK(check_rows("dU", dU, lddg, F, act));
  if (dG == dU) return ff::fail(FF_EINVAL, "dG and dU are the same memory");
  for (const void* p : {(const void*)dG, (const void*)dU})
    if (T > 1 && ((p == dH && lddg != lddh) || (G && (p == G || p == U) && lddg != ldg)))
      return ff::fail(FF_EINVAL, "dG or dU over dH, G or U needs the same leading dimension");
  if (dX) GLU_CHECK(check_rows("dX", dX, lddx, n, act));
  Parts dx{}, dw{};
  if (dX) dx = dx_product(T, n, F, c.bf16);
  if (dWg) dw = dw_product(T, n, F, c.bf16);
  const int64_t need = workspace(n, &dx, &dw);
  if ((dX || dWg) && (!ws || (uintptr_t)ws % 256)) return ff::fail(FF_EINVAL, "the workspace is NULL or not 256-byte aligned");
  if ((dX || dWg) && workspace_bytes < need)
    return ff::fail(FF_EINVAL, "the workspace holds %lld bytes, the call needs %lld", (long long)workspace_bytes, (long long)need);
  hipError_t e;
  if (G) {
    PointArgs a{};
    a.dH = dH, a.G = G, a.U = U, a.dG = dG, a.dU = dU, a.lddh = lddh, a.ldg = ldg, a.lddg = lddg;
    e = run_point(c, a, s);
  } else {
    ProjArgs a{};
    a.Wg = Wg, a.Wu = Wu, a.X = X, a.ldw = ldw, a.ldx = ldx, a.Ag = Ag, a.Au = Au, a.lda = lda;
    a.dH = dH, a.lddh = lddh, a.G = dG, a.U = dU, a.ldg = lddg;
    e = run_projection(c, kBackward, a, s);
  }
  GLU_CHECK(done(e, "gated feed-forward backward"));
  if (dX) {
    GradArgs a{};
    a.A[0] = Wg, a.A[1] = Wu, a.lda = ldw, a.B[0] = dG, a.B[1] = dU, a.ldb = lddg;
    a.out[0] = a.out[1] = dX, a.ldo = lddx, a.beta = beta_dx;
    GLU_CHECK(done(run_gradient(c, false, dx, a, static_cast<float*>(ws), s), "gated feed-forward backward"));
  }
  if (dWg) {
    GradArgs a{};
    a.A[0] = a.A[1] = X, a.lda = ldx, a.B[0] = dG, a.B[1] = dU, a.ldb = lddg;
    a.out[0] = dWg, a.out[1] = dWu, a.ldo = lddw, a.beta = beta_dw;
    GLU_CHECK(done(run_gradient(c, true, dw, a, static_cast<float*>(ws), s), "gated feed-forward backward"));
  }
  return FF_OK;
}

}  // extern "C"
