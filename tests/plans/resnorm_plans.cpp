// The plan of a join's call (csrc/resnorm_plan.h), asked from a test: lines "shape T n esz backward" give pieces, waves and whether the last
// piece overlaps; "sums n vectors groups" gives, for each launch of the sums, its threads and the gate rows it takes.
#include <cstdio>
#include <cstring>

#include "resnorm_plan.h"

using namespace ff::resnorm;

int main() {
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    long long a, b, c;
    int d;
    if (!std::strcmp(what, "shape") && std::scanf("%lld %lld %lld %d", &a, &b, &c, &d) == 4) {
      const Shape s = shape_of(b, (int)c, a, d != 0);
      std::printf("%d %d %d\n", s.nv, s.wv, (int)s.part);
    } else if (!std::strcmp(what, "sums") && std::scanf("%lld %lld %lld", &a, &b, &c) == 3) {
      for (int64_t g = 0, ng = 0; g < c; g += ng) {
        const int v = g == 0 ? (int)b : 0;
        ng = sum_rows(a, v, c - g);
        std::printf("%lld %lld ", (long long)(sum_blocks(a) * kSumThreads * (v + ng)), (long long)ng);
        if (ng < 1) break;
      }
      std::printf("\n");
    }
  }
  return 0;
}
