// Places in memory of the tiles of the head's matrix products (xent_gemm.h): plain integer arithmetic, shared by the
// kernels and by a test that walks it on the CPU.
#pragma once

#include <cstdint>

#ifdef __HIP__
#define FF_HD __host__ __device__ __forceinline__
#else
#define FF_HD inline
#endif

namespace ff {
namespace xent {

constexpr int kTileBytes = 128;   // of k in a tile of an operand stored along k

// A load's place within its tile's range has 32 bits, of which the highest is set for a place past every range.  The tallest
// tiles have 256 rows in bf16 and 128 in fp32: the longest rows that H, W, dH and dW may have, and those of P, which has a
// column per vocabulary entry.
constexpr int64_t kMaxLd = (int64_t)1 << 20, kMaxGradVocab = (int64_t)1 << 22;
static_assert(255 * kMaxGradVocab * 2 + kTileBytes < (int64_t)1 << 31 && 127 * kMaxGradVocab * 4 + kTileBytes < (int64_t)1 << 31 &&
                  kMaxLd <= kMaxGradVocab,
              "places within a tile fit 31 bits");

// An operand's tile of `bx` along i (or j) from x0 and one k tile: bytes from the operand's first element to the tile's, and
// the bytes from there on that may be read.  X: extent along i.  along_k: rows of memory run along k, X counts rows, and a
// row is read to the next whole 16-byte piece of k (H and W: their widths are whole pieces; P: zero padding).  Otherwise
// rows of memory run along i and are read to the next whole piece of X.
struct Span {
  int64_t first;
  uint32_t bytes;
};

FF_HD int64_t k_step(bool along_k, int esz, int64_t ld) { return along_k ? kTileBytes : (kTileBytes / esz) * ld * esz; }

// left: k of the tile that exist (at most kTileBytes / esz)
FF_HD Span span_of(bool along_k, int esz, int bx, int64_t ld, int64_t x0, int64_t X, int64_t kt, int left) {
  const int per = 16 / esz;
  Span s;
  if (along_k) {
    const int64_t rows = X - x0 < bx ? X - x0 : bx;
    s.first = x0 * ld * esz + kt * kTileBytes;
    s.bytes = (uint32_t)((rows - 1) * ld * esz + (left + per - 1) / per * 16);
  } else {
    s.first = x0 * esz + kt * k_step(false, esz, ld);
    s.bytes = (uint32_t)(((left - 1) * ld + (X + per - 1) / per * per - x0) * esz);
  }
  return s;
}

// Workgroups go round the eight XCDs; each XCD takes a contiguous run of the `total` tiles.
FF_HD int share_of(int wg, int total) {
  const int xcd = wg & 7, per = total >> 3, rem = total & 7;
  return xcd * per + (xcd < rem ? xcd : rem) + (wg >> 3);
}

// Tiles run in groups of eight along j and then along i, so that those that run at once on an XCD share their operands
// in its L2.
FF_HD void tile_of(int id, int tm, int tn, int* im, int* in) {
  const int group = 8 * tm;
  const int g = id / group, first = g * 8;
  const int w = tn - first < 8 ? tn - first : 8;
  const int in_group = id - g * group;
  *in = first + in_group % w;
  *im = in_group / w;
}

}  // namespace xent
}  // namespace ff
