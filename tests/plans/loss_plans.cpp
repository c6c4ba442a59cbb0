// Prints what a call of the head's loss runs: for each line "T n V bf16 dh dw" of the input the tile, split of k and number
// of tiles of its products (of the first piece), and its pieces.
#include <cstdio>

#include "xent_plan.h"

using namespace ff::xent;

static void product(const char* name, const Product& p, int64_t M, int64_t N) {
  std::printf(" %s %d %d %lld", name, p.tile, p.splits, (long long)(tiles_of(M, N, p.tile) * p.splits));
}

int main() {
  long long T, n, V;
  int bf16, dh, dw;
  while (std::scanf("%lld %lld %lld %d %d %d", &T, &n, &V, &bf16, &dh, &dw) == 6) {
    const Call c = plan(T, n, V, bf16 ? FF_BF16 : FF_F32, dh, dw);
    const bool grad = dh || dw;
    const int64_t N = grad ? c.Tp : c.Tf;
    std::printf("terms %d by_vocab %d Tp %lld Vp %lld Tf %lld", c.terms, (int)c.by_vocab, (long long)c.Tp, (long long)c.Vp,
                (long long)c.Tf);
    product("logits", logits_product(c, N, grad ? c.Vp : V), grad ? c.Vp : V, N);
    if (dh) product("dh", dh_product(c, c.terms * N, c.Vp), n, c.terms * N);
    if (dw) {
      Product p = dw_product(c, c.Vp, c.terms * T);
      if (c.by_vocab) p.splits = 1;
      product("dw", p, n, c.Vp);
    }
    std::printf("\n");
  }
  return 0;
}
