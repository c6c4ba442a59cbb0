// The tiles of the head's matrix products, walked on the CPU as the kernels walk them: every tile of every call belongs to one
// workgroup, and no range that a load may read ends past its tensor.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "xent_span.h"

using namespace ff::xent;

static int failed = 0;
static long walked = 0;

static void check(bool ok, const char* what, long a, long b) {
  if (!ok && failed++ < 20) std::printf("%s: %ld %ld\n", what, a, b);
}

static int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct Side {
  bool along_k;
  int64_t ld, X, bytes;   // bytes of the tensor
};

static void walk(int esz, int bm, int bn, const Side& A, const Side& B, int64_t K, int splits) {
  const int kk = kTileBytes / esz;
  const int tm = (int)(up(A.X, bm) / bm), tn = (int)(up(B.X, bn) / bn), tiles = tm * tn;
  const int kt = (int)(up(K, kk) / kk), per = (kt + splits - 1) / splits, n = (kt + per - 1) / per, total = tiles * n;
  std::vector<char> seen(total, 0);
  for (int wg = 0; wg < total; ++wg) {
    const int id = share_of(wg, total);
    check(id >= 0 && id < total && !seen[id], "share", wg, id);
    if (id < 0 || id >= total) return;
    seen[id] = 1;
    const int split = id / tiles;
    int im, in;
    tile_of(id - split * tiles, tm, tn, &im, &in);
    check(im >= 0 && im < tm && in >= 0 && in < tn, "tile", im, in);
    for (int t = split * per; t < kt && t < (split + 1) * per; ++t) {
      const int left = (int)(K - (int64_t)t * kk < kk ? K - (int64_t)t * kk : kk);
      const Span a = span_of(A.along_k, esz, bm, A.ld, (int64_t)im * bm, A.X, t, left);
      const Span b = span_of(B.along_k, esz, bn, B.ld, (int64_t)in * bn, B.X, t, left);
      check(a.first >= 0 && a.first + a.bytes <= A.bytes, "A past its end", a.first + a.bytes, A.bytes);
      check(b.first >= 0 && b.first + b.bytes <= B.bytes, "B past its end", b.first + b.bytes, B.bytes);
      ++walked;
    }
  }
}

int main() {
  std::srand(3);
  const int tiles[4][2] = {{256, 256}, {128, 128}, {128, 32}, {32, 32}};
  for (int round = 0; round < 600; ++round) {
    const int esz = round % 2 ? 2 : 4, mult = 16 / esz;
    const int64_t T = round < 40 ? round / 2 + 1 : 1 + std::rand() % 700, n = mult * (1 + std::rand() % 90);
    const int64_t V = round < 40 ? 1 + std::rand() % 40 : 1 + std::rand() % 3000;
    const int64_t ldh = n + mult * (std::rand() % 3), ldw = n + mult * (std::rand() % 3), ldp = up(V, 64);
    // a tensor ends with the last element of its last row; P is padded to ldp
    const int64_t hb = ((T - 1) * ldh + n) * esz, wb = ((V - 1) * ldw + n) * esz, pb = T * ldp * esz;
    for (const auto& t : tiles)
      for (int splits : {1, 3, 16}) {
        walk(esz, t[0], t[1], {true, ldw, V, wb}, {true, ldh, T, hb}, n, 1);
        walk(esz, t[0], t[1], {false, ldw, n, wb}, {true, ldp, T, pb}, V, splits);
        walk(esz, t[0], t[1], {false, n, n, T * n * esz}, {false, ldp, V, pb}, T, splits);
      }
  }
  std::printf("spans: %ld tiles, %d failed checks\n", walked, failed);
  return failed != 0;
}
