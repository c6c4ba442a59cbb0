// Plan of a call of the gated feed-forward (glu.hip): kernels, tiles, splits and parts of its products, size of its workspace.
// Plain arithmetic, shared by the host code and by a test that asks which instances a size runs.
#pragma once

#include "xent_plan.h"

namespace ff {
namespace glu {

using xent::kCUs;
using xent::kLarge;
using xent::kMedium;
using xent::kSmall;
using xent::tile_m;
using xent::tile_n;
using xent::up;

constexpr int kk_of(int esz) { return 128 / esz; }   // k of a tile

// Microseconds of a k tile (128 bytes of k) with few workgroups on the card, with one on every CU, and with all `slots` taken; and
// the k tiles that a tile's start and end cost.  Measured, projections of T tokens, n -> F, bf16:
//   large   4096 x 4096 -> 8192 (1024 tiles) 386 us, 2981 x 3712 -> 1408 (132) 77, 256 x 4096 -> 11008 (86) 81
//   medium  2048 x 4096 -> 4096 (1024) 120 (large 108), 2981 x 3712 -> 1408 (528) 87, 64 x 4096 -> 11008 (172) 46, 800 x 3968 -> 128
//           (14) 29
//   small   64 x 4096 -> 11008 (344) 37, 100 x 1024 -> 4096 (256) 8, 800 x 3968 -> 128 (50) 19, 700 x 4096 -> 1024 (352) 30
// fp32:
//   medium  500 x 768 -> 2048 (128 tiles) 56, 1658 x 1024 -> 4096 (832) 250;  small  31 (512), 231 (3328); 64 x 1024 -> 4096 (128) 23
struct TileCost {
  int slots;
  double few, one, full, ends;
};
constexpr TileCost kTileCosts[2][3] = {{{0, 0, 0, 0, 0}, {512, 2.0, 2.2, 3.84, 2}, {512, 0.60, 0.72, 1.08, 2}},
                                       {{256, 1.15, 1.53, 1.53, 5}, {512, 0.45, 0.80, 0.92, 3}, {512, 0.26, 0.28, 0.45, 4}}};
constexpr double kLaunch = 2.0;

// Of `tiles` tiles those of a last (or only) round of large ones that are halved, where their halves fit one round.  256 tokens, 4096 ->
// 11008 (86 tiles) 80 us whole, 54 as halves; dX of 1700 tokens, 2304 <- 2 x 6000 (63 tiles x 2 splits) 134 and 94.
inline int rest_of(int tile, int64_t tiles) {
  const int rest = (int)(tiles % kCUs);
  return tile == kLarge && rest <= kCUs / 2 ? rest : 0;
}
// What a round of halves takes of one of whole tiles.  Over 210 products (70 each of the projections, dX and dW, 64 to 4096 tokens) whose
// plan the number decides, the chosen plans take over the fastest of those timed 3.8% more with 0.50, 2.5 with 0.54, 2.0 with 0.56, 1.8 with
// 0.58, 1.6 with 0.60, 1.8 with 0.62, 2.0 with 0.68 and above (never halved there).
constexpr double kHalved = 0.60;
// Medium tiles of dX that have a CU each, and k tiles enough, take four buffers instead of two (of its steps, `kt`): 1003 tokens, 768 <-
// 2 x 2304 51 us -> 38 (48 tiles), 32 -> 28 (96), 22 -> 22 (192); 256 tokens, 4096 <- 2 x 11008 71 -> 55 (256); 4 k tiles 7.8 -> 8.8.
// The projections and dW gained nothing (500 x 768 -> 2304 10.2 -> 11.7, 512 x 2048 -> 4096 23.6 -> 21.7; dW 19 -> 17 to 12 -> 12).
inline bool dx_deep(bool bf16, int64_t tiles, int64_t kt) { return bf16 && tiles <= kCUs && kt >= 12; }
constexpr double kDeepFew = 0.40, kDeepOne = 0.55, kDeepEnds = 6;
// Workgroups of a launch of `tiles` tiles: large ones are walked by one workgroup a CU.
inline int tile_groups(int tile, int tiles, int rest) {
  if (tile != kLarge) return tiles;
  return tiles > kCUs ? kCUs : (rest ? 2 * rest : tiles);
}

inline double tiles_time(bool bf16, int tile, int64_t tiles, int64_t kt) {
  const TileCost& c = kTileCosts[bf16][tile];
  const int64_t rounds = tiles / c.slots, left = tiles % c.slots;
  double last = 0;
  // (two fp32 tiles on a CU take as long as when every CU has two: the matrix units bound them)
  if (left > kCUs) last = bf16 ? c.one + (c.full - c.one) * (double)(left - kCUs) / kCUs : c.full;
  else if (left) last = c.few + (c.one - c.few) * (double)left / kCUs;
  if (rest_of(tile, tiles)) last *= kHalved;
  return kLaunch + ((double)rounds * c.full + last) * ((double)kt + c.ends);
}

inline int64_t tiles_of(int64_t M, int64_t N, int tile) { return xent::tiles_of(M, N, tile); }
// A launch has fewer than 2^32 threads; large tiles are walked by one workgroup a CU.
inline bool fits(int64_t groups, int threads) { return groups * threads < (int64_t)1 << 32; }
inline bool tiles_fit(int tile, int64_t tiles) { return tile == kLarge || fits(tiles, 256); }

// ------------------------------------------------------------------------------------------- projections

// The few-token kernel: workgroups of 16 columns and 16 or 32 tokens, bound by what they read through the L2 (bf16, 256 tokens 1024 ->
// 4096: 31 us where tiles take 10; 100 tokens 1024 -> 1024: 6.7 and 7.5; one token 512 -> 640: 3.6 and 5.1; fp32, 100 tokens 1024 ->
// 1024: 11.7 and 22.9; at 4096 -> 11008 tiles are faster from the first token on, 27 and 30).
inline int64_t narrow_groups(int64_t T, int64_t F) { return up(F, 16) / 16 * (up(T, T > 16 ? 32 : 16) / (T > 16 ? 32 : 16)); }
inline double narrow_time(int64_t T, int64_t n, int64_t F, bool bf16) {
  const int64_t rows = 32 + (T > 16 ? 32 : T);
  return kLaunch + 1.0 + (double)(narrow_groups(T, F) * rows * n) * (bf16 ? 2 : 4) / (bf16 ? 8.0e6 : 6.5e6);
}
// Waves that share k: eight where four would leave the card empty and each has a chunk of 256 bytes (sixteen spill, and are slower).
inline int narrow_waves(int64_t T, int64_t n, int64_t F, int esz) {
  const int64_t groups = narrow_groups(T, F), chunks = up(n * esz, 256) / 256;
  return groups >= 256 || chunks <= 4 ? 4 : 8;
}

// Some of the tokens of a call; a call has one or two of them, one after the other.
struct Part {
  int64_t t0, T;
  int tile;        // xent::Tile
  int ks;          // waves of a few-token workgroup; 0: tiles
  int splits;      // gradients: of k
  int kt_split;    // k tiles of a split
};
struct Parts {
  int count;
  Part part[2];
  double time;
};

// One part for all rows, or two: as many rows as fill whole rounds of workgroups, and the others in what suits them.  one(T) is the best
// single part of T rows, columns(tile) the tiles along the other side.
template <class One, class Columns, class Time>
inline Parts parts_of(int64_t T, bool bf16, const One& one, const Columns& columns, const Time& time) {
  Parts best = one(T);
  for (int tile = bf16 ? kLarge : kMedium; tile <= kMedium; ++tile) {
    const int64_t tm = columns(tile), tn = up(T, tile_n(tile)) / tile_n(tile), slots = kTileCosts[bf16][tile].slots;
    for (int64_t rounds = tm * tn / slots, tries = 0; rounds > 0 && tries < 3; --rounds, ++tries) {
      const int64_t rows = rounds * slots / tm;
      if (rows < 1 || rows >= tn) continue;
      const int64_t t1 = rows * tile_n(tile);
      const Parts other = one(T - t1);
      const double t = time(tile, tm * rows) + other.time;
      if (t >= 0.97 * best.time || !tiles_fit(tile, tm * rows)) continue;
      best.count = 2, best.time = t;
      best.part[0] = {0, t1, tile, 0, 1, 0};
      best.part[1] = other.part[0];
      best.part[1].t0 = t1;
    }
  }
  return best;
}

inline Parts projection(int64_t T, int64_t n, int64_t F, bool bf16) {
  const int esz = bf16 ? 2 : 4;
  const int64_t kt = up(n, kk_of(esz)) / kk_of(esz);
  auto one = [&](int64_t rows) {
    const int ks = narrow_waves(rows, n, F, esz);
    Parts p{1, {{0, rows, kSmall, ks, 1, 0}}, fits(narrow_groups(rows, F), ks * 64) ? narrow_time(rows, n, F, bf16) : 1e30};
    for (int tile = bf16 ? kLarge : kMedium; tile <= kSmall; ++tile) {
      const int64_t tiles = tiles_of(2 * F, rows, tile);
      const double t = tiles_time(bf16, tile, tiles, kt);
      if (t < p.time && tiles_fit(tile, tiles)) p = Parts{1, {{0, rows, tile, 0, 1, 0}}, t};
    }
    return p;
  };
  return parts_of(T, bf16, one, [&](int tile) { return up(2 * F, tile_m(tile)) / tile_m(tile); },
                  [&](int tile, int64_t tiles) { return tiles_time(bf16, tile, tiles, kt); });
}

// ------------------------------------------------------------------------------------------- gradients

// M columns and `rows` rows of `outs` results, kt k tiles in each of `halves` parts of the sum, which are split alike.  Partial sums are
// written and read at about 7 TB/s (small ones through the caches) by a launch more; those of large results are not worth the pass through memory.
inline Parts gradient(int64_t rows, int64_t M, int64_t kt, int halves, int outs, bool bf16) {
  auto one = [&](int64_t N) {
    Parts p{1, {{0, N, kSmall, 0, 1, (int)kt}}, 1e30};
    for (int tile = bf16 ? kLarge : kMedium; tile <= kSmall; ++tile) {
      const int64_t tiles = outs * tiles_of(M, N, tile);
      for (int s : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64}) {
        if (s > 1 && (halves * kt < 4 * s || (outs == 2 && 2 * rows > 4096))) break;
        const int64_t per = (kt + s - 1) / s, splits = (kt + per - 1) / per;
        double t = tiles_time(bf16, tile, tiles * splits, halves * per);
        if (tile == kMedium && halves == 2 && dx_deep(bf16, tiles * splits, halves * per))
          t = kLaunch + (kDeepFew + (kDeepOne - kDeepFew) * (double)(tiles * splits) / kCUs) * ((double)(halves * per) + kDeepEnds);
        if (splits > 1) t += 4.5 + (double)(splits * outs * N * M) * 8.0 / 7e6;
        if (t < p.time && tiles_fit(tile, tiles * splits)) p = Parts{1, {{0, N, tile, 0, (int)splits, (int)per}}, t};
        if (tiles * splits >= 4 * kCUs) break;
      }
    }
    return p;
  };
  Parts p = parts_of(rows, bf16, one, [&](int tile) { return outs * (up(M, tile_m(tile)) / tile_m(tile)); },
                     [&](int tile, int64_t tiles) { return tiles_time(bf16, tile, tiles, halves * kt); });
  if (p.count == 2) p.part[0].kt_split = (int)kt;
  return p;
}
inline Parts dx_product(int64_t T, int64_t n, int64_t F, bool bf16) {
  const int kk = kk_of(bf16 ? 2 : 4);
  return gradient(T, n, up(F, kk) / kk, 2, 1, bf16);
}
inline Parts dw_product(int64_t T, int64_t n, int64_t F, bool bf16) {
  const int kk = kk_of(bf16 ? 2 : 4);
  return gradient(F, n, up(T, kk) / kk, 1, 2, bf16);
}

// Bytes of partial sums of `outs` results of n columns.
inline int64_t part_bytes(const Parts& p, int64_t n, int outs) {
  int64_t bytes = 0;
  for (int i = 0; i < p.count; ++i)
    if (p.part[i].splits > 1) {
      const int64_t b = (int64_t)p.part[i].splits * outs * p.part[i].T * n * 4;
      if (b > bytes) bytes = b;
    }
  return bytes;
}
inline int64_t workspace(int64_t n, const Parts* dx, const Parts* dw) {
  const int64_t x = dx ? part_bytes(*dx, n, 1) : 0, w = dw ? part_bytes(*dw, n, 2) : 0, most = x > w ? x : w;
  return most ? up(most, 256) : 256;
}

}  // namespace glu
}  // namespace ff
