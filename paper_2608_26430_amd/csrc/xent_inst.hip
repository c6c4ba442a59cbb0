// Instances of the head's matrix products (xent_gemm.h), compiled once per element type and operand layout:
// -DXENT_BF16=0/1, -DXENT_LAYOUT=0/1/2 (logits, dH, dW).
#include "xent_gemm.h"

#ifndef XENT_BF16
#error "XENT_BF16 and XENT_LAYOUT select the instances"
#endif

namespace ff {
namespace xent {

#define XENT_NAME2(l, b) launch_gemm_##l##_##b
#define XENT_NAME(l, b) XENT_NAME2(l, b)

hipError_t XENT_NAME(XENT_LAYOUT, XENT_BF16)(int tile, const GemmArgs& a, hipStream_t s) {
#if XENT_BF16
  typedef __bf16 E;
#else
  typedef float E;
#endif
  constexpr bool TRA = XENT_LAYOUT != 0, TRB = XENT_LAYOUT == 2;
  // large tiles: one workgroup per CU walks all of its tiles, each tile's first loads under the last one's results;
  // medium tiles hide them under the other workgroup of the CU, and walking cost them 7 to 24%
  const int total = a.tm * a.tn * a.splits;
  const dim3 grid((unsigned)(total > kCUs && tile == kLarge ? kCUs : total));
#if XENT_BF16
  if (tile == kLarge) {
    hipLaunchKernelGGL((gemm_kernel<E, 256, 256, 2, 4, 2, TRA, TRB, 2>), grid, dim3(512), 0, s, a);
    return hipGetLastError();
  }
#endif
#if XENT_LAYOUT == 0
  if (tile == kTiny) {
    hipLaunchKernelGGL((gemm_kernel<E, 32, 32, 2, 2, 4, TRA, TRB, 2>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
#endif
  if (tile == kMedium) {
    hipLaunchKernelGGL((gemm_kernel<E, 128, 128, 2, 2, 2, TRA, TRB, 2>), grid, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((gemm_kernel<E, 128, 32, 4, 1, 4, TRA, TRB, 2>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace xent
}  // namespace ff
