// The rules by which a bf16 product takes its kernel (include/canz.h: canz_linear).  Host arithmetic only, so that a plain C++ program can ask them.
#pragma once
#include <cstdint>

namespace canz {

constexpr int LINEAR_CU = 256;
constexpr int64_t LINEAR_MAX_EXTENT = 65535 * 64;

constexpr int LINEAR_K = 32;        // k of a step of the tile kernels
constexpr int LINEAR_ROUND = 128;   // k of a round of a ring of two stages

// The kernel for few rows takes up to this many rows of A, where both operands are contiguous along k.
constexpr int LINEAR_FEW = 64;
constexpr bool linear_few(int64_t m, bool a_trans, bool b_trans) { return m <= LINEAR_FEW && !a_trans && !b_trans; }
// Its blocks have 16, 32 or 64 rows of B (figures at the kernel); an image's block of 32 elements is one block's.
constexpr int linear_few_width(int64_t n, bool pre) { return n <= 4096 && !pre ? 0 : n < 12288 ? 1 : 2; }

// About how many ns a launch takes by the tiles it has, for `steps` of 32 k.  256 x 256 in rounds of one to a CU, of which beginning and end are not hidden; 128 x 128 one to a CU with a ring of four
// stages, or two to a CU with two.  us measured (large; small): 4096 x 4096 x 256 18; 19, x 1024 34; 39, x 4096 99; 117; 8192 x 4096 x 512 42; 48; 2048 x 4096 x 1024 35; 21, x 4096 88; 60; 1024 x 4096 x
// 4096 83; 34, x 1024 33; 13; 1024 x 1024 x 1024 32; 11; 128 x 1024 x 256 19; 8.
constexpr int64_t linear_large_ns(int64_t tiles, int64_t steps) { return (tiles + LINEAR_CU - 1) / LINEAR_CU * (700 * steps + 10500); }
constexpr int64_t linear_small_ns(int64_t tiles, int64_t steps) {
  if (tiles <= LINEAR_CU) return (146 + tiles / 4) * steps + 6000;
  const int64_t rest = tiles % (2 * LINEAR_CU);
  return tiles / (2 * LINEAR_CU) * (405 * steps + 7500) + (rest > LINEAR_CU ? 405 * steps + 7500 : rest > 0 ? 310 * steps + 6000 : 0);
}
// Whole rounds of large tiles after which the others, less than a round, are done as quarters by small ones, in a launch of their own; 0: all are done by large ones.  An element's sum is the
// same in either.  4352 x 4096 x 4096 takes 126 us like this and 150 with small tiles alone, 4096 x 25600 x 5120 835 and 985 with large ones alone.
constexpr int64_t linear_quarters_ns(int64_t large, int64_t steps) {
  return linear_large_ns(large / LINEAR_CU * LINEAR_CU, steps) + linear_small_ns(large % LINEAR_CU * 4, steps) + 2500;
}
constexpr int64_t linear_whole_rounds(int64_t large, int64_t steps) {
  return large > LINEAR_CU && large % LINEAR_CU > 0 && linear_quarters_ns(large, steps) < linear_large_ns(large, steps) ? large / LINEAR_CU : 0;
}
constexpr bool linear_large_tiles(int64_t large, int64_t small, int64_t steps) {
  return (linear_whole_rounds(large, steps) > 0 ? linear_quarters_ns(large, steps) : linear_large_ns(large, steps)) < linear_small_ns(small, steps);
}

// Whether small tiles are done one to a CU with a ring of four stages where there are more of them than CUs: where the longest takes as many steps as a CU's share of all.  Products of 400, 128 and
// 1000 rows by 1536 x 4096 take 54 us like this and 66 with two to a CU, four of 1000 rows 79 and 72.
constexpr bool linear_alone(int64_t longest, int64_t all_steps) { return longest * LINEAR_CU >= all_steps; }

// How many parts k is cut into, each with fp32 sums of its own in the workspace, which are added up in order: products whose small tiles leave CUs idle for long.  A product alone decides, so
// that its sums do not depend on what shares the call.  128 k take a tile 0.6 us, a second launch and the sums 4 to 10.
constexpr int LINEAR_MAX_PARTS = 8;
constexpr int linear_parts(int64_t m, int64_t n, int64_t k) {
  if (m == 0 || n == 0 || k == 0) return 1;
  const int64_t tiles = ((m + 127) / 128) * ((n + 127) / 128), rounds = (k + LINEAR_ROUND - 1) / LINEAR_ROUND;
  int64_t parts = LINEAR_CU / tiles;
  if (parts > LINEAR_MAX_PARTS) parts = LINEAR_MAX_PARTS;
  if (parts > rounds / 4) parts = rounds / 4;
  return parts >= 2 && (rounds - rounds / parts) * 600 >= 10000 ? static_cast<int>(parts) : 1;
}

}  // namespace canz
