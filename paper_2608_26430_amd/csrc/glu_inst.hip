// Instances of the gated feed-forward's kernels (glu_gemm.h), compiled in parts: -DGLU_BF16=0/1 and -DGLU_PART=0..2 (the
// projections with that function) or 3, 4 (dX, dW).
#include "glu_gemm.h"
#include "glu_plan.h"

#if !defined(GLU_BF16) || !defined(GLU_PART)
#error "GLU_BF16 and GLU_PART select the instances"
#endif

namespace ff {
namespace glu {

#if GLU_BF16
typedef __bf16 E;
#else
typedef float E;
#endif

#define GLU_NAME3(n, p, b) n##_##p##_##b
#define GLU_NAME2(n, p, b) GLU_NAME3(n, p, b)
#define GLU_NAME(n) GLU_NAME2(n, GLU_PART, GLU_BF16)

// Buffers of small tiles: in fp32, bound by the matrix units, two, so that four workgroups share a CU (500 tokens, 768 -> 2048 dW 35.5 ->
// 33.4 us, 2048 tokens, 1024 -> 552 projections 58 -> 55, 1658 tokens, 1024 -> 4096 231 -> 225, dW 221 -> 208); dX starts with two tiles
// and needs three at least.
constexpr int kSmallNB = sizeof(E) == 4 && GLU_PART != 3 ? 2 : 4;

#if GLU_PART < 3

template <int MODE>
static void project(int tile, int ks, const ProjArgs& a, hipStream_t s) {
  constexpr int FN = GLU_PART;
  if (ks) {
    const int rows = a.T > 16 ? 32 : 16;
    const dim3 grid((unsigned)((a.F + 15) / 16) * (unsigned)((a.T + rows - 1) / rows));
#define GLU_NARROW(NT, KS) hipLaunchKernelGGL((narrow_kernel<E, NT, KS, FN, MODE>), grid, dim3(KS * 64), 0, s, a)
    if (a.T > 16 && ks == 4) GLU_NARROW(2, 4);
    else if (a.T > 16) GLU_NARROW(2, 8);
    else if (ks == 4) GLU_NARROW(1, 4);
    else GLU_NARROW(1, 8);
    return;
  }
  const int total = a.tm * a.tn;
  // large tiles: one workgroup per CU walks all of its tiles, each tile's first loads under the last one's results
  const dim3 grid((unsigned)tile_groups(tile, total, a.rest));
#if GLU_BF16
  if (tile == xent::kLarge) {
    hipLaunchKernelGGL((projection_kernel<E, 256, 256, 2, 4, 2, 2, FN, MODE>), grid, dim3(512), 0, s, a);
    return;
  }
#endif
  if (tile == xent::kMedium) hipLaunchKernelGGL((projection_kernel<E, 128, 128, 2, 2, 2, 2, FN, MODE>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((projection_kernel<E, 128, 32, 4, 1, kSmallNB, 2, FN, MODE>), grid, dim3(256), 0, s, a);
}

hipError_t GLU_NAME(launch_projection)(int mode, int tile, int ks, const ProjArgs& a, hipStream_t s) {
  if (mode == kForward) project<kForward>(tile, ks, a, s);
  else project<kBackward>(tile, ks, a, s);
  return hipGetLastError();
}

hipError_t GLU_NAME(launch_point)(const PointArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((point_kernel<E, GLU_PART>), dim3((unsigned)((a.items + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

#else

hipError_t GLU_NAME(launch_gradient)(int tile, const GradArgs& a, hipStream_t s) {
  constexpr bool TRB = GLU_PART == 4;
  const int total = a.tm * a.tn * (TRB ? 2 : 1) * a.splits;
  const dim3 grid((unsigned)tile_groups(tile, total, a.rest));
#if GLU_BF16
  if (tile == xent::kLarge) {
    hipLaunchKernelGGL((gradient_kernel<E, 256, 256, 2, 4, 2, TRB, 2>), grid, dim3(512), 0, s, a);
    return hipGetLastError();
  }
#endif
#if GLU_BF16 && GLU_PART == 3
  if (tile == xent::kMedium && dx_deep(true, total, 2 * a.kt_split)) {
    hipLaunchKernelGGL((gradient_kernel<E, 128, 128, 2, 2, 4, TRB, 1>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
#endif
  if (tile == xent::kMedium) hipLaunchKernelGGL((gradient_kernel<E, 128, 128, 2, 2, 2, TRB, 2>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((gradient_kernel<E, 128, 32, 4, 1, kSmallNB, TRB, 2>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

#endif

}  // namespace glu
}  // namespace ff
