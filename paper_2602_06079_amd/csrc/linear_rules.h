// The rules by which a bf16 product takes its kernel (include/canz.h: canz_linear).  Host arithmetic only, so that a plain C++ program can ask them.
#pragma once
#include <cstdint>

namespace canz {

constexpr int LINEAR_CU = 256;
constexpr int64_t LINEAR_MAX_EXTENT = 65535 * 64;

constexpr int LINEAR_K = 32;        // k of a step of the tile kernels
constexpr int LINEAR_ROUND = 128;   // k of a round of their ring

// The kernel for few rows takes up to this many rows of A, where both operands are contiguous along k.
constexpr int LINEAR_FEW = 64;
constexpr bool linear_few(int64_t m, bool a_trans, bool b_trans) { return m <= LINEAR_FEW && !a_trans && !b_trans; }

// ns that a launch takes by the tiles it has, 256 x 256 in rounds of one to a CU or 128 x 128 in rounds of two, for `steps` of 32 k.
constexpr int64_t linear_large_ns(int64_t tiles, int64_t steps) { return (tiles + LINEAR_CU - 1) / LINEAR_CU * (680 * steps + 6000); }
constexpr int64_t linear_small_ns(int64_t tiles, int64_t steps) {
  const int64_t rest = tiles % (2 * LINEAR_CU);
  return tiles / (2 * LINEAR_CU) * (400 * steps + 3000) + (rest > LINEAR_CU ? 400 * steps + 3000 : rest > 0 ? 220 * steps + 3000 : 0);
}
constexpr bool linear_large_tiles(int64_t large, int64_t small, int64_t steps) { return linear_large_ns(large, steps) < linear_small_ns(small, steps); }

// Whole rounds of large tiles after which the others, less than a round, are done as quarters by small ones; 0: all are done by large ones.  An element's sum is the same in either.
constexpr int64_t linear_whole_rounds(int64_t large, int64_t steps) {
  const int64_t rounds = large / LINEAR_CU, rest = large % LINEAR_CU;
  return rounds > 0 && rest > 0 && linear_small_ns(4 * rest, steps) < linear_large_ns(rest, steps) ? rounds : 0;
}

// How many parts k is cut into, each with fp32 sums of its own in the workspace, which are added up in order: products whose tiles leave most of the chip idle for long.  A
// product alone decides, so that its sums do not depend on what shares the call.
constexpr int LINEAR_MAX_PARTS = 8;
constexpr int linear_parts(int64_t m, int64_t n, int64_t k) {
  if (m == 0 || n == 0 || k == 0) return 1;
  const int64_t tiles = ((m + 127) / 128) * ((n + 127) / 128), rounds = (k + LINEAR_ROUND - 1) / LINEAR_ROUND;
  int64_t parts = LINEAR_CU / tiles;
  if (parts > LINEAR_MAX_PARTS) parts = LINEAR_MAX_PARTS;
  if (parts > rounds / 4) parts = rounds / 4;
  return parts >= 2 && (rounds - rounds / parts) * 880 >= 8000 ? static_cast<int>(parts) : 1;
}

}  // namespace canz
