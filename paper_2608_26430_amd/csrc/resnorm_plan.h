// Plan of a call of the join of two blocks (resnorm.hip): which instance takes a row, how many workgroups, what the workspace holds and
// the launches of the sums.  Plain arithmetic, shared by the host code and by a test that asks which instances a size runs.
#pragma once

#include <cstdint>
#include <initializer_list>

namespace ff {
namespace resnorm {

// The instance of a row of n: 16-byte pieces of a thread, waves of a row (0: rows are read several times), overlapping last
// piece.
struct Shape {
  int nv, wv;
  bool part;
};

// Rows of up to 4 KB: four waves of a piece a thread where one wave would hold a whole row in few workgroups (16 x 1000 fp32, both
// norms layer norms: backward 14.5 us, 7.6 with four waves; 300 x 768 bf16 forward 4.7 and 4.4, 1001 5.1 and 5.6, 12,608 19 and 32),
// and in the backward wherever the wave's threads would hold 16 elements in fp32, whose sums spill (12,608 x 1000 100 and 62 us).  Wider
// rows in fp32 take 8 elements a thread for the same reason (4000 x 2048 70 us with 16, 43 with 8; 4000 x 4096 123 and 96), but for the
// widest: sixteen waves have no more registers in all (4000 x 5000 247 and 237).  bf16 spills little (4000 x 4096 63 either way).
inline Shape shape_of(int64_t n, int esz, int64_t T, bool backward) {
  const int per = 16 / esz, whole = 16 / per;      // pieces of 16 elements a thread
  const int64_t p = (n + per - 1) / per;
  const bool part = n % per != 0;
  if (n < per) return {0, 0, part};
  if (p > 64 && p <= 256 && (T <= 512 || p > whole * 64 || (backward && p > 128))) return {1, 4, part};
  if (backward && esz == 4 && p > 256 && p <= 1024) return {2, p <= 512 ? 4 : 8, part};
  if (p <= whole / 2 * 64) return {whole / 2, 1, part};
  for (int wv : {1, 4, 8})
    if (p <= (int64_t)whole * wv * 64) return {whole, wv, part};
  return {0, 0, part};
}

inline int64_t fwd_groups(int64_t T, const Shape& s) {
  const int rows = s.wv == 1 ? 4 : 1;
  const int64_t g = (T + rows - 1) / rows;
  return g < 1024 ? g : 1024;
}

// Workgroups of a backward, at most: each leaves partial rows to be added up.
constexpr int kGroups = 512;
inline int64_t most_groups(int64_t n) { return n <= 4096 ? kGroups : kGroups / 2; }

// Slices of a group of `rows` rows: all groups' together fill the workgroups.
inline int64_t slices_of(int64_t rows, int64_t groups, int64_t n, int at_once) {
  const int64_t most = (rows + at_once - 1) / at_once, want = most_groups(n) / groups;
  return want < 1 ? 1 : (want < most ? want : most);
}

inline int64_t up(int64_t x) { return (x + 255) / 256 * 256; }

// Places in the workspace: partial rows of the four vectors, of the gate, the row sums of wide rows.
struct Space {
  int64_t gate, sums, bytes;
};
inline Space space_of(int64_t T, int64_t n, int64_t groups, bool wide) {
  const int64_t G = most_groups(n), rows = T < G ? (T ? T : 1) : G;
  Space s;
  s.gate = up(rows * 4 * n * 4);
  // a group of one slice needs none
  s.sums = s.gate + (groups < G ? up(rows * n * 4) : 0);
  s.bytes = s.sums + (wide ? up(T * 16) : 0);
  if (s.bytes < 256) s.bytes = 256;
  return s;
}

// Sums of the partial rows: workgroups of a row of n, and of `left` gate rows those that a launch takes beside `vectors` (at
// most four) rows of the vectors; three at least, n being 2^24 at most.
constexpr int kSumThreads = 1024;
inline int64_t sum_blocks(int64_t n) { return (n + 31) / 32; }
inline int64_t sum_rows(int64_t n, int vectors, int64_t left) {
  // (a launch has fewer than 2^32 threads)
  int64_t most = (((int64_t)1 << 32) - 1) / (sum_blocks(n) * kSumThreads) - vectors;
  most = most > 32768 ? 32768 : most;
  return left < most ? left : most;
}

}  // namespace resnorm
}  // namespace ff
