// Instances of the backward of the join of two blocks (resnorm.h), compiled once per element type and kind of norms:
// -DRESNORM_BF16=0/1, -DRESNORM_COMBO=0..5; with and without a gate.
#include "resnorm.h"

#if !defined(RESNORM_BF16) || !defined(RESNORM_COMBO)
#error "RESNORM_BF16 and RESNORM_COMBO select the instances"
#endif

namespace ff {
namespace resnorm {

#if RESNORM_BF16
typedef __bf16 E;
#else
typedef float E;
#endif

template <int NV, int WV>
static void go(const Args& a, const Shape& sh, unsigned groups, hipStream_t s) {
  constexpr bool P = RESNORM_COMBO < 2 || RESNORM_COMBO == 4, N = RESNORM_COMBO < 4, B = RESNORM_COMBO % 2 == 1 || RESNORM_COMBO == 4;
  const dim3 grid(groups), block(threads_of(WV));
  if (a.gate) {
    if (sh.part) hipLaunchKernelGGL((bwd_kernel<E, NV, WV, true, P, N, B, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((bwd_kernel<E, NV, WV, false, P, N, B, true>), grid, block, 0, s, a);
  } else {
    if (sh.part) hipLaunchKernelGGL((bwd_kernel<E, NV, WV, true, P, N, B, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((bwd_kernel<E, NV, WV, false, P, N, B, false>), grid, block, 0, s, a);
  }
}

#define RESNORM_NAME2(c, b) launch_bwd_##c##_##b
#define RESNORM_NAME(c, b) RESNORM_NAME2(c, b)

hipError_t RESNORM_NAME(RESNORM_COMBO, RESNORM_BF16)(const Args& a, const Shape& sh, unsigned groups, hipStream_t s) {
  constexpr int k = 16 / Pack<E>::kN;      // pieces of 16 elements
  // (shape_of: in fp32 16 elements a thread are left to the widest rows)
  constexpr bool kF32 = sizeof(E) == 4;
  if (sh.wv == 1 && sh.nv == k / 2) go<k / 2, 1>(a, sh, groups, s);
  else if (sh.wv == 1) go<2, 1>(a, sh, groups, s);
  else if (sh.wv == 4 && sh.nv == 1) go<1, 4>(a, sh, groups, s);
  else if (sh.wv == 4) go<2, 4>(a, sh, groups, s);
  else if (kF32 && sh.nv == 2) go<2, 8>(a, sh, groups, s);
  else go<k, 8>(a, sh, groups, s);
  return hipGetLastError();
}

}  // namespace resnorm
}  // namespace ff
