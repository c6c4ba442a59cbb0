// The plan of a gated feed-forward's call (csrc/glu_plan.h), asked from a test: lines of "T n F bf16" in, tiles and splits out.
#include <cstdio>

#include "glu_plan.h"

using namespace ff::glu;

int main() {
  long T, n, F;
  int bf16;
  while (std::scanf("%ld %ld %ld %d", &T, &n, &F, &bf16) == 4) {
    const Projection p = projection(T, n, F, bf16);
    const Product x = dx_product(T, n, F, bf16), w = dw_product(T, n, F, bf16);
    const long pt = (long)ff::xent::tiles_of(2 * F, T, p.tile), xt = (long)ff::xent::tiles_of(n, T, x.tile) * x.splits;
    const long wt = 2 * (long)ff::xent::tiles_of(n, F, w.tile) * w.splits;
    std::printf("%d %d %ld  %d %d %d %ld  %d %d %d %ld  %ld\n", p.tile, p.ks, pt, x.tile, x.splits, x.kt_split, xt, w.tile, w.splits,
                w.kt_split, wt, (long)workspace(T, n, F, bf16, true, true));
  }
  return 0;
}
