// Plan of a call of the head's loss (xent.hip): tiles and splits of its products, its pieces, places in the workspace.  Plain
// arithmetic, shared by the host code and by a test that asks which instances a size runs.
#pragma once

#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "frameft.h"

namespace ff {
namespace xent {

// Tile sizes of the instances: large (256 x 256, wave 128 x 64; bf16 only), medium (128 x 128, wave 64 x 64), small (128 x
// 32, wave 32 x 32), and tiny (32 x 32, wave 16 x 16) for the logits of a few classes.
enum Tile { kLarge = 0, kMedium = 1, kSmall = 2, kTiny = 3 };
constexpr int tile_m(int t) { return t == kLarge ? 256 : (t == kTiny ? 32 : 128); }
constexpr int tile_n(int t) { return t == kLarge ? 256 : (t == kMedium ? 128 : 32); }
// columns of one entry of the logits' statistics
constexpr int stat_cols(int t) { return t == kLarge ? 128 : (t == kMedium ? 64 : (t == kSmall ? 32 : 16)); }

constexpr int kCUs = 256;

constexpr int64_t kPieceBytes = (int64_t)256 << 20;   // P of one piece
constexpr int64_t kPairTokens = 128;                  // tokens up to which bf16 P is kept in two terms
constexpr int64_t kFewTokens = 64;                    // tokens up to which a workgroup joins one token's statistics
constexpr int64_t kJoinReads = (int64_t)1 << 20;      // statistics up to which the rescaling workgroups join them
constexpr int64_t kStatBytes = (int64_t)64 << 20;     // statistics of one piece

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline int64_t tiles_of(int64_t M, int64_t N, int t) { return up(M, tile_m(t)) / tile_m(t) * (up(N, tile_n(t)) / tile_n(t)); }

struct Product {
  int tile;
  int splits;
  int kt_split;
};

// Microseconds of a k tile on one CU, from measured calls: with workgroups enough to fill the CU, and with one workgroup
// per CU at most; and the k tiles that a tile's start and end cost.
//   bf16 large  1.53 / 1.53    4096 tokens x 32,000 entries, 4096 wide: logits 840 us (medium 1040), dH 770 (1030)
//        medium 0.51 / 0.80    1003 x 30,001, 768 wide: dW 52 us (large 61); 128 x 32,000, 4096 wide: logits 60 (97, small 73)
//        small  0.30 / 0.60    16 x 32,000, 4096 wide: logits 41 us (medium 58); 64 tokens 48 (60)
//   fp32 medium 1.92 / 1.92    2048 x 33,000, 1024 wide: logits 1060 us (small 1120)
//        small  0.50 / 0.75    200 x 3000, 512 wide: logits 14 us (medium 39); 500 x 8001, 768 wide: dW 59 (68)
//   logits of few classes, tiny: bf16 0.14 / 0.16, fp32 0.20 / 0.28
//                              4000 x 100, 768 wide, bf16: 6.1 us (small 7.4); 190 x 44, 1024 wide, fp32: 10 us (small 23)
// The large tile has no fp32 instance: its registers spill.
struct TileCost {
  double full, single, ends;
};
constexpr TileCost kCosts[2][4] = {{{0, 0, 0}, {1.92, 1.92, 2}, {0.50, 0.75, 2}, {0.20, 0.28, 3}},
                                   {{1.53, 1.53, 5}, {0.51, 0.80, 3}, {0.30, 0.60, 4}, {0.14, 0.16, 6}}};
constexpr int64_t kTinyVocab = 4096;   // entries up to which the tiny tile is looked at

// Tile and split of k of a product with M columns, N rows and kt k tiles: the least estimated time, where partial sums are
// written and read at about 4.5 TB/s by a launch more.
inline Product choose(int64_t M, int64_t N, int64_t kt, bool may_split, bool bf16, bool tiny = false) {
  Product best{kSmall, 1, (int)kt};
  double least = 1e30;
  for (int tile = bf16 ? kLarge : kMedium; tile <= (tiny ? kTiny : kSmall); ++tile) {
    const TileCost& u = kCosts[bf16][tile];
    const int64_t tiles = tiles_of(M, N, tile);
    for (int s : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64}) {
      if (s > 1 && (!may_split || s > kt / 4)) break;
      const int64_t per = (kt + s - 1) / s, splits = (kt + per - 1) / per, wgs = tiles * splits;
      const int64_t rounds = (wgs + kCUs - 1) / kCUs;
      double t = (double)rounds * ((double)per + u.ends) * (rounds == 1 ? u.single : u.full);
      if (splits > 1) t += 3.0 + (double)splits * (double)N * (double)M * 8.0 / 4.5e6;
      if (t < least) least = t, best = Product{tile, (int)splits, (int)per};
      if (wgs >= 4 * kCUs) break;
    }
  }
  return best;
}

struct Call {
  int64_t T, n, V;
  int bf16, esz, kk;        // kk: k of a tile
  bool dh, dw;
  int64_t Tp, Vp;           // tokens and vocabulary entries of a piece of P
  int64_t Tf;               // tokens of a piece of the forward alone
  int terms;                // of P: 2 for few tokens in bf16
  bool by_vocab;            // pieces of the vocabulary (dW of a long call)
  size_t off_p, off_stats, off_zt, off_part, off_live, bytes;
};

inline Product logits_product(const Call& c, int64_t N, int64_t M) { return choose(M, N, up(c.n, c.kk) / c.kk, false, c.bf16, c.V <= kTinyVocab); }
inline Product dh_product(const Call& c, int64_t N, int64_t K) { return choose(c.n, N, up(K, c.kk) / c.kk, true, c.bf16); }
inline Product dw_product(const Call& c, int64_t M, int64_t K) {
  // sums of a whole head are not worth a pass through memory
  return choose(c.n, M, up(K, c.kk) / c.kk, M <= 4096, c.bf16);
}

inline Call plan(int64_t T, int64_t n, int64_t V, int act, bool dh, bool dw) {
  Call c{};
  c.T = T, c.n = n, c.V = V, c.bf16 = act == FF_BF16, c.esz = c.bf16 ? 2 : 4, c.kk = 128 / c.esz;
  c.dh = dh, c.dw = dw;
  c.bytes = 256;
  if (T == 0) return c;
  c.terms = c.bf16 && T <= kPairTokens ? 2 : 1;
  const int64_t ldp = up(V, 64);
  int64_t most = kPieceBytes / (ldp * c.esz) / 256 * 256;
  if (most < 256) most = 256;
  c.by_vocab = dw && T > most;
  c.Tp = c.by_vocab || T < most ? T : most;
  c.Vp = V;
  if (c.by_vocab) {
    c.Vp = kPieceBytes / (T * c.esz) / 256 * 256;
    if (c.Vp < 256) c.Vp = 256;
    if (c.Vp > V) c.Vp = V;
  }
  // at most, with the smallest tile's columns
  const int64_t cols = stat_cols(V <= kTinyVocab ? kTiny : kSmall), entries = up(V, cols) / cols;
  c.Tf = kStatBytes / (8 * entries) / 256 * 256;
  if (c.Tf < 256) c.Tf = 256;
  if (c.Tf > T) c.Tf = T;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t o = at;
    at += (size_t)up(bytes, 256);
    return o;
  };
  const bool grad = dh || dw;
  c.off_p = take(grad ? c.terms * c.Tp * up(c.Vp, 64) * c.esz : 0);
  const int64_t rows = c.by_vocab || !grad ? c.Tf : (c.Tp > c.Tf ? c.Tp : c.Tf);
  c.off_stats = take(rows * entries * 8);
  c.off_zt = take(rows * 4);
  int64_t part = 0;
  auto more = [&](int64_t b) { part = b > part ? b : part; };
  if (dh)
    for (int64_t N : {c.Tp, T % c.Tp ? T % c.Tp : c.Tp}) {
      const Product p = dh_product(c, c.terms * N, c.Vp);
      if (p.splits * c.terms > 1 || c.by_vocab) more((int64_t)p.splits * c.terms * N * n * 4);
    }
  if (dw && !c.by_vocab) {
    const Product p = dw_product(c, V, c.terms * T);
    if (p.splits > 1) more((int64_t)p.splits * V * n * 4);
  }
  c.off_part = take(part);
  c.off_live = take(dw ? c.terms * T * n * c.esz : 0);
  c.bytes = at < 256 ? 256 : at;
  return c;
}

}  // namespace xent
}  // namespace ff
