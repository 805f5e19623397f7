// Storage layout of the microscaled 4-bit images (include/canz.h: canz_mx_image_bytes).
//
// An image holds R rows of K elements as an operand of v_mfma_scale_f32_16x16x128_f8f6f4: lane l supplies the 32 elements
// (16 bytes) of row l % 16 and block l / 16 of the 128 k of one instruction, and their scale byte in a register of four, of which
// the instruction picks one.  So the codes lie in units of 16 rows x 128 k, 1 KiB each and read or copied into LDS by a wavefront as
// one linear piece (conflict-free as it lies), and the scales in units of 64 rows x 128 k, 256 bytes, a dword per lane with the bytes of four
// units of codes.  Rows are padded to 64, k to 128; the padding holds zero codes and zero scale bytes (2^-127).
//
// Two units hold 32 rows, in pieces of four rows by turns: rows 0-3, 8-11, 16-19, 24-27 are slots 0 .. 15 of the first, the others those of the
// second.  The instruction leaves four consecutive slots of its first operand in a lane's four registers, so that a lane has 8 consecutive
// rows after two units: 16 bytes of a bf16 result, 64 bytes from the four lanes of a row of C, stored as they lie.
//   unit(row) = row / 32 * 2 + row / 4 % 2,  slot(row) = row / 8 % 4 * 4 + row % 4
//   codes   unit (unit(row), k / 128) at (unit(row) ks + k / 128) 1024; in it block (k / 32) % 4, slot(row), 16 bytes; element k in byte
//           (k % 32) / 2, even k in the low half
//   scales  behind the codes, unit (row / 64, k / 128) at ((row / 64) ks + k / 128) 256; in it block (k / 32) % 4, slot(row), unit(row) % 4
#pragma once
#include <cstddef>
#include <cstdint>

namespace canz {

constexpr int MX_BLOCK = 32;          // elements that share a scale
constexpr int MX_UNIT_ROWS = 16;
constexpr int MX_UNIT_K = 128;
constexpr int MX_UNIT_BYTES = MX_UNIT_ROWS * MX_UNIT_K / 2;
constexpr int MX_PAD_ROWS = 64;
constexpr int MX_SCALE_BYTES = MX_PAD_ROWS * MX_UNIT_K / MX_BLOCK;
constexpr int64_t MX_MAX_EXTENT = 65535 * 64;   // as for the matrices of the optimizer steps

// unit of codes and slot in it of a row, and the way back
template <typename I>
constexpr I mx_unit(I row) { return (row >> 5 << 1) + (row >> 2 & 1); }
template <typename I>
constexpr I mx_slot(I row) { return (row >> 3 & 3) * 4 + (row & 3); }
template <typename I>
constexpr I mx_row(I unit, I slot) { return (unit >> 1 << 5) + (slot >> 2) * 8 + (unit & 1) * 4 + (slot & 3); }

// units of 16 rows (a multiple of 4) and of 128 k
constexpr int64_t mx_row_tiles(int64_t rows) { return (rows + MX_PAD_ROWS - 1) / MX_PAD_ROWS * (MX_PAD_ROWS / MX_UNIT_ROWS); }
constexpr int64_t mx_k_units(int64_t k) { return (k + MX_UNIT_K - 1) / MX_UNIT_K; }
constexpr int64_t mx_code_bytes(int64_t rows, int64_t k) { return mx_row_tiles(rows) * mx_k_units(k) * MX_UNIT_BYTES; }
constexpr int64_t mx_image_bytes(int64_t rows, int64_t k) {
  return mx_code_bytes(rows, k) + mx_row_tiles(rows) / 4 * mx_k_units(k) * MX_SCALE_BYTES;
}

// Launches take a block of 256 threads per tile of 128 x 64 elements or more and stay below 2^32 threads for one matrix: refused are matrices of more than
// 2^37 padded elements (73 GB as an image, 275 GB in bf16).
constexpr bool mx_fits_grid(int64_t rows, int64_t cols) { return ((rows + 127) / 128) * ((cols + 127) / 128) <= (int64_t(1) << 37) / (128 * 128); }

}  // namespace canz
