// The plan of a gated feed-forward's call (csrc/glu_plan.h), asked from a test: lines of "T n F bf16" in; for the projections, dX and
// dW: number of parts, and for each rows, tile, waves (few tokens), splits of k, tiles, halved tiles.
#include <cstdio>

#include "glu_plan.h"

using namespace ff::glu;

static void print(const Parts& p, int64_t M, int outs) {
  std::printf("%d ", p.count);
  int64_t at = 0;
  for (int i = 0; i < p.count; ++i) {
    const Part& q = p.part[i];
    const int64_t tiles = outs * tiles_of(M, q.T, q.tile) * q.splits;
    std::printf(" %lld %d %d %d %lld %d ", (long long)q.T, q.tile, q.ks, q.splits, (long long)tiles, rest_of(q.tile, tiles));
    if (q.t0 != at) std::printf(" gap ");
    at += q.T;
  }
}

int main() {
  long long T, n, F;
  int bf16;
  while (std::scanf("%lld %lld %lld %d", &T, &n, &F, &bf16) == 4) {
    print(projection(T, n, F, bf16), 2 * F, 1);
    const Parts dx = dx_product(T, n, F, bf16), dw = dw_product(T, n, F, bf16);
    print(dx, n, 1);
    print(dw, n, 2);
    std::printf(" %lld\n", (long long)workspace(n, &dx, &dw));
  }
  return 0;
}
