// Plan of a call of the gated feed-forward (glu.hip): kernels, tiles and splits of its products, size of its workspace.  Plain
// arithmetic, shared by the host code and by a test that asks which instances a size runs.
#pragma once

#include "xent_plan.h"

namespace ff {
namespace glu {

using xent::Product;
using xent::up;

constexpr int kk_of(int esz) { return 128 / esz; }   // k of a tile

constexpr int64_t kNarrowTokens = 32;   // tokens up to which the few-token kernel makes the projections

struct Projection {
  int tile;    // xent::Tile
  int ks;      // waves of a few-token workgroup, 0: tiles
};

// Waves that share k in the few-token kernel: enough of them on the card to read at its rate, each with a chunk of 256 bytes at
// least.
inline int narrow_waves(int64_t T, int64_t n, int64_t F, int esz) {
  const int64_t groups = up(F, 16) / 16, chunks = up(n * esz, 256) / 256;
  for (int ks : {4, 8})
    if (groups * ks >= 2048 || chunks <= ks) return ks;
  return T > 16 ? 8 : 16;    // sixteen waves of two groups of tokens spill
}

inline Projection projection(int64_t T, int64_t n, int64_t F, bool bf16) {
  const int esz = bf16 ? 2 : 4, kk = kk_of(esz);
  if (T <= kNarrowTokens) return {xent::kSmall, narrow_waves(T, n, F, esz)};
  return {xent::choose(2 * F, T, up(n, kk) / kk, false, bf16).tile, 0};
}

// Of `tiles` tiles those of a last round of large ones that are halved, where their halves fit one round.
inline int rest_of(int tile, int64_t tiles) {
  const int rest = (int)(tiles % xent::kCUs);
  return tile == xent::kLarge && tiles > xent::kCUs && rest <= xent::kCUs / 2 ? rest : 0;
}

// Both halves of the sum over F are split alike: kt_split counts k tiles of one half.
inline Product dx_product(int64_t T, int64_t n, int64_t F, bool bf16) {
  const int kk = kk_of(bf16 ? 2 : 4);
  const int64_t kt = up(F, kk) / kk;
  Product p = xent::choose(n, T, 2 * kt, true, bf16);
  const int64_t per = (kt + p.splits - 1) / p.splits;
  p.splits = (int)((kt + per - 1) / per), p.kt_split = (int)per;
  return p;
}

inline Product dw_product(int64_t T, int64_t n, int64_t F, bool bf16) {
  const int kk = kk_of(bf16 ? 2 : 4);
  // partial sums of large weights are not worth a pass through memory
  return xent::choose(n, 2 * F, up(T, kk) / kk, 2 * F <= 4096, bf16);
}

inline int64_t workspace(int64_t T, int64_t n, int64_t F, bool bf16, bool dx, bool dw) {
  int64_t bytes = 256;
  if (T == 0) return bytes;
  auto more = [&](int64_t b) { bytes = b > bytes ? up(b, 256) : bytes; };
  if (dx) {
    const Product p = dx_product(T, n, F, bf16);
    if (p.splits > 1) more((int64_t)p.splits * T * n * 4);
  }
  if (dw) {
    const Product p = dw_product(T, n, F, bf16);
    if (p.splits > 1) more((int64_t)p.splits * 2 * F * n * 4);
  }
  return bytes;
}

}  // namespace glu
}  // namespace ff
