// The rules by which a microscaled product takes its kernel (include/canz.h: canz_mx_product).  Host arithmetic only, so that a plain C++ program can ask them.
#pragma once
#include <cstdint>

#include "mx_layout.h"

namespace canz {

constexpr int N_CU = 256;

// ns that a launch takes by the tiles it has: 256 x 256 in rounds of one to a CU, 128 x 128 in rounds of two, or less than one at the end.  A k unit
// takes 780 ns of a round of large tiles and 460 of one of small ones (a quarter of the work, twice as often), 210 with one small tile to a CU; beginning
// and end of a tile 6000 and 2600.  us for bf16 results, 256 x 256 and 128 x 128: 8192^3 223, 252; 4096^3 35, 36; 8192 x 12288 x 4096 189, 213; 4096 x
// 25600 x 5120 246, 256; 6000 x 6000 x 2000 52, 42; 5000 x 4000 x 1000 28, 19; 4096 x 4096 x 1024 18.1, 16.8; 3000^3 25, 21; 2048 x 4096 x 8192 49, 35;
// 4096 x 2048 x 1024 15.7, 10.8; 1024^3 13.6, 6.3.
constexpr int64_t large_tiles_ns(int64_t tiles, int64_t ks) { return (tiles + N_CU - 1) / N_CU * (780 * ks + 6000); }
constexpr int64_t small_tiles_ns(int64_t tiles, int64_t ks) {
  const int64_t rest = tiles % (2 * N_CU);
  return tiles / (2 * N_CU) * (460 * ks + 2600) + (rest > N_CU ? 460 * ks + 2600 : rest > 0 ? 210 * ks + 2600 : 0);
}
// `ks`: k units of a small tile in the mean
constexpr bool mx_large_tiles(int64_t large, int64_t small, int64_t ks) { return large_tiles_ns(large, ks) < small_tiles_ns(small, ks); }

constexpr int FEW_ROWS = 64;   // the most rows of A that the kernel for few rows takes

// A product's A may be a matrix, which the kernel for few rows rounds on its way: with up to 16 rows, as long as every block rounding it again costs less than
// a launch that makes its image (4 us): 8 x 25600 x 5120 18.4 us and 16.9 + 4, 16 x 25600 x 5120 22.7 and 15.2 + 4.5, 8 x 5120 x 25600 24.8 and 20.8 + 4.5,
// 8 x 4096 x 4096 5.9 and 4.5 + 4.
constexpr bool mx_rounds_on_the_way(int64_t m, int64_t n, int64_t k) { return m <= 16 && m * n <= (int64_t(1) << 30) / (k > 0 ? k : 1); }

// How the kernel for few rows goes over B, by its rows (a product alone decides, so that its sums do not depend on what shares the launch):
// many of them are taken 64 to a block of four wavefronts, which halves what is read and rounded of A; with fewer the blocks are made smaller to fill the chip, and
// with very few a block takes more wavefronts, so that k is gone through faster.  us for one row of bf16, 64 rows / 32 rows / 32 rows with 16 wavefronts:
// 25600 x 5120 16.4 / 18.5 / 21.4, 12288 x 4096 6.9 / 7.5 / 8.2, 8192 x 5120 6.8 / 6.4 / 6.5, 5120 x 25600 24.1 / 19.2 / 20.1, 333 x 9000 9.2 / 8.0 / 6.8.
enum Width { NARROW, MIDDLE, WIDE, WIDTHS };
constexpr Width width_of(int64_t n) { return n >= 12288 ? WIDE : n >= 4096 ? MIDDLE : NARROW; }

// How many parts k is cut into, each a problem of its own with fp32 sums in the workspace, which launch_mx_join adds up: products of more than 64 rows whose
// tiles leave most of the chip idle for long.  A unit of k takes a tile 210 ns, a second launch and the sums through memory up to 8 us.  us, whole and in
// parts: 128 x 1024 x 65536 102 and 22.4, 100 x 1000 x 20000 35.5 and 14.4, 1024 x 1024 x 16384 29.5 and 24.2, 300 x 500 x 8000 17.9 and 13.2, 256 x 2048 x
// 8192 17.1 and 14.4, 1024 x 1024 x 8192 17.5 and 17.2; not cut: 2048 x 1024 x 4096 11.6, 128 x 128 x 4096 10.2.  A product alone decides, so that its
// sums do not depend on what shares the call.  Not cut either, whatever k: products of 65 and more tiles, which run on up to half of the chip (1024 x 2048 x
// 65536 138 us), and those of up to 64 rows, whose blocks have 32 or 64 columns each (64 x 1024 x 65536 35.7, 64 x 1000 x 20000 13.3).
constexpr int MX_MAX_PARTS = 8;
constexpr int mx_parts(int64_t m, int64_t n, int64_t k) {
  if (m <= 64 || n == 0 || k == 0) return 1;
  const int64_t tiles = ((m + 127) / 128) * ((n + 127) / 128), units = mx_k_units(k);
  int64_t parts = 128 / tiles;
  if (parts > MX_MAX_PARTS) parts = MX_MAX_PARTS;
  if (parts > units / 8) parts = units / 8;
  return parts >= 2 && (units - units / parts) * 210 >= 8000 ? static_cast<int>(parts) : 1;
}

}  // namespace canz
