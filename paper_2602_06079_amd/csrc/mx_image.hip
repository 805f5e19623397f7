// Microscaled 4-bit images of matrices: canz_mx_quantize and canz_mx_dequantize.
//
// A block of 32 consecutive elements along the contracted index shares a scale X = 2^e; an element is one of 0, .5, 1, 1.5, 2, 3, 4,
// 6 times X (mx_round.h).
#include "device_util.h"
#include "mx.h"
#include "mx_round.h"

namespace canz {
namespace {

constexpr int TILE = 128;      // rows and columns of a block's tile: whole units of codes and of scales for either image
constexpr int THREADS = 256;
#define CANZ_INLINE __attribute__((always_inline))

typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Code of one element with noise u in 0 .. 255: s floor((rint(256 a / s) + u) / 256) for a = |v| / X and the distance s of the values
// around it, s = 2^(e - 1) with e the exponent of a, at least 0.  Adding 1.5 2^23 (s / 256) rounds a to a multiple of s / 256, ties to even, and leaves
// that multiple in the low bits of the sum; with 2 e s added as well, bits 8 and up are the code after u is added to them.  The largest sums are those of e
// = 2, so that one limit keeps the code at 7.
// Returned with the code in bits 8 to 10, the sign of v in bit 11 and zeros up to bit 15.
__device__ __forceinline__ unsigned noisy_code(float v, unsigned byte, unsigned u) {
  const float a = __builtin_amdgcn_ldexpf(__builtin_fabsf(v), 127 - static_cast<int>(byte));
  const unsigned e = max(__builtin_bit_cast(unsigned, a) >> 23, 127u);   // + 127
  // bits of 1.5 2^(e + 14) + 2 e s: (e + 127 + 14) << 23 | 1 << 22 | e << 9
  constexpr unsigned STEP = (1u << 23) + (1u << 9), START = (14u << 23) + (1u << 22) - (127u << 9);
  constexpr unsigned LIMIT = ((2u + 127u + 14u) << 23) + (1u << 22) + 0x7FFu;
  const float magic = __builtin_bit_cast(float, __umul24(e, STEP) + START);
  const unsigned sum = min(__builtin_bit_cast(unsigned, a + magic) + u, LIMIT);
  constexpr unsigned SIGN = 1u << 11;
  return sum | (__builtin_bit_cast(unsigned, v) >> 20 & SIGN);   // LIMIT and what the sums reach leave bit 11 free
}
// The same for two bf16 elements at a time, whose eight digits fp16 holds: half the instructions.  `less`: their blocks' (byte - 16) << 7 (less_of); u: noise
// in the low bytes of the halves.  A difference of exponents makes 2 a in fp16 of |v| (what is below 2^-14 comes out as something below 2^-14 and is
// rounded to 0 like it).  a + 2^(e + 1) is rounded to a multiple of 2^(e - 9) = s / 256, and the bits of the sum count these multiples; 512 e more and bits 8 and up
// are the code.  Returned as by noisy_code, in either half.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
constexpr unsigned PAIRS_FROM = 16;   // the smallest scale byte; of zeros (padding, above all) any will do
__device__ __forceinline__ bool in_pairs(unsigned byte, unsigned top) { return byte >= PAIRS_FROM || top == 0; }
__device__ __forceinline__ unsigned short less_of(unsigned byte) { return static_cast<unsigned short>((max(byte, PAIRS_FROM) - PAIRS_FROM) << 7); }
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned noisy_pair(unsigned v, u16x2 less, unsigned u) {
  const u16x2 twice = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, v & 0x7FFF7FFFu), less) << 3;
  constexpr unsigned short TWO = 0x4000, LIMIT = 0x7FF;
  const unsigned top = __builtin_bit_cast(unsigned, __builtin_elementwise_max(twice, u16x2{TWO, TWO})) & 0x7C007C00u;   // 2^(e + 1): (e + 16) << 10
  const f16x2 sum = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, twice), f16x2{0.5f, 0.5f}, __builtin_bit_cast(f16x2, top));
  const unsigned count = __builtin_bit_cast(unsigned, sum) + u - (top >> 1) - 0x20002000u;   // 0 .. 2303 in either half, so nothing is borrowed
  const unsigned code = __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(u16x2, count), u16x2{LIMIT, LIMIT}));
  return code | (v >> 4 & 0x08000800u);
}

// eight codes of one block, element 0 in the lowest bits; u: noise bytes
template <bool NOISE>
__device__ __forceinline__ unsigned eight_codes(const float (&v)[8], unsigned byte, const unsigned (&u)[8]) {
  unsigned r = 0;
  if constexpr (NOISE) {
    unsigned c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = noisy_code(v[i], byte, u[i]);
    // bits 8 .. 15 of four of them to the bytes of a word
    auto gather = [](unsigned x, unsigned y, unsigned z, unsigned w) CANZ_INLINE {
      const unsigned xy = __builtin_amdgcn_perm(y, x, 0x0C0C0501u), zw = __builtin_amdgcn_perm(w, z, 0x05010C0Cu);
      return xy | zw;
    };
    r = gather(c[0], c[2], c[4], c[6]) | gather(c[1], c[3], c[5], c[7]) << 4;
  } else {
    const float s = mx_scale_value(byte);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], s, 3);
  }
  return byte == MX_SCALE_NAN ? 0u : r;
}

// Codes of four words of noisy_pair as bytes: those of the low halves, those of the high ones
__device__ __forceinline__ uint2 by_halves(unsigned p, unsigned q, unsigned r, unsigned s) {
  constexpr unsigned BYTES_1_3 = 0x07030501u, LOW = 0x05040100u, HIGH = 0x07060302u;
  const unsigned pq = __builtin_amdgcn_perm(q, p, BYTES_1_3), rs = __builtin_amdgcn_perm(s, r, BYTES_1_3);
  return {__builtin_amdgcn_perm(rs, pq, LOW), __builtin_amdgcn_perm(rs, pq, HIGH)};
}
constexpr unsigned NOISE_LOW = 0x0C010C00u, NOISE_HIGH = 0x0C030C02u;   // two of four noise bytes, a half each

// the largest of the four lanes that hold a block
__device__ __forceinline__ unsigned largest_of_four(unsigned v) {
  constexpr int SWAP_1 = 0xB1, SWAP_2 = 0x4E;   // quad permutes [1, 0, 3, 2] and [2, 3, 0, 1]
  v = max(v, static_cast<unsigned>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), SWAP_1, 0xF, 0xF, false)));
  return max(v, static_cast<unsigned>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), SWAP_2, 0xF, 0xF, false)));
}

// Bits of the largest magnitudes of two columns (or of the even and the odd elements), gathered pair by pair: of bf16 in one register.
template <typename E>
struct PairMax;
template <>
struct PairMax<float> {
  unsigned top[2] = {0, 0};
  typedef float pair __attribute__((ext_vector_type(2)));
  __device__ __forceinline__ void take(pair x) {
#pragma unroll
    for (int q = 0; q < 2; ++q) top[q] = max(top[q], mx_magnitude(x[q]));
  }
  __device__ __forceinline__ unsigned of(int q) const { return top[q]; }
};
template <>
struct PairMax<__bf16> {
  u16x2 top = {0, 0};
  __device__ __forceinline__ void take(mx_bf16x2 x) { top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, __builtin_bit_cast(unsigned, x) & 0x7FFF7FFFu)); }
  __device__ __forceinline__ unsigned of(int q) const { return static_cast<unsigned>(top[q]) << 16; }
};

// eight consecutive elements of a row, those behind its end as zeros
template <typename E>
using Eight = E __attribute__((ext_vector_type(8)));
template <typename E>
__device__ __forceinline__ Eight<E> load8(const E* p) {
  typedef E any __attribute__((ext_vector_type(8), aligned(sizeof(E))));
  return *reinterpret_cast<const any*>(p);
}
template <typename E>
__device__ __forceinline__ Eight<E> load8(const E* p, int64_t left) {
  if (left >= 8) return load8(p);
  Eight<E> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : static_cast<E>(0.f);
  return v;
}
__device__ __forceinline__ uint2 load_noise8(const uint8_t* p) {
  const u32x2_any w = *reinterpret_cast<const u32x2_any*>(p);
  return uint2{w[0], w[1]};
}
__device__ __forceinline__ uint2 load_noise8(const uint8_t* p, int64_t left) {
  if (left >= 8) return load_noise8(p);
  uint2 r = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) (i < 4 ? r.x : r.y) |= i < left ? static_cast<unsigned>(p[i]) << (8 * (i & 3)) : 0u;
  return r;
}
template <typename E>
__device__ __forceinline__ void store8(E* p, int64_t left, const float (&v)[8]) {
  if (left >= 8) {
    if constexpr (sizeof(E) == 4) {
      f32x4_any a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = v[i], b[i] = v[4 + i];
      *reinterpret_cast<f32x4_any*>(p) = a, *reinterpret_cast<f32x4_any*>(p + 4) = b;
    } else {
      bf16x8_any a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = static_cast<__bf16>(v[i]);
      *reinterpret_cast<bf16x8_any*>(p) = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = static_cast<E>(v[i]);
  }
}

// Tile (x, y) of a block.  Blocks go round the XCDs one by one; RUN tiles in a row go to the same one, since neighbours share lines: those of noise, of which a
// tile has 64 bytes a row, and all where rows do not begin on lines.  us without and with, both ways: bf16 8192 x 12288 66.6 and 59.0, 3 of 4097 x 1531 17.2 and 13.6,
// with noise 29.6 and 23.2, fp32 2 of 25600 x 5120 255 and 243.  (Here and below launches follow each other on three sets of buffers in turn; alone under a profiler a
// launch takes up to a quarter longer.)
constexpr int N_XCD = 8, RUN = 16;
__device__ __forceinline__ uint2 tile_of_block() {
  const unsigned n = gridDim.x * gridDim.y, id = blockIdx.x + gridDim.x * blockIdx.y, in = id % (N_XCD * RUN);
  const unsigned tile = id - in + N_XCD * RUN <= n ? id - in + in % N_XCD * RUN + in / N_XCD : id;   // the last ones are left as they are
  return {tile % gridDim.x, tile / gridDim.x};
}

// One block rounds a tile of 128 rows x 64 columns: first along its rows (8 lanes a row, 8 elements each, 4 lanes a block), keeping
// the elements in LDS, then along its columns (a thread two blocks).  Scale bytes are collected in LDS and leave in pieces of 128 bytes and more.
// Every element is read once and every image written once: fp32 25600 x 5120, two matrices, both ways 243 us (1.33 GB, 5.4 TB/s; a plain copy of 2 GiB, half of it
// writes, reaches 4.65 to 4.95), bf16 8192 x 12288 59 us (5.2 TB/s), 3 of 4097 x 1531 13.6 us (4.2).  The tile is as large as leaves room for four blocks and more on a CU
// (128 x 128 took 296 us for the first), and a thread's loads are all on their way before the first is used.  With noise
// arithmetic counts as much as memory: 7 instructions an element and side in pairs, 13 in fp32; both ways bf16 8192 x 12288 88 us (120 without pairs; 4.6 TB/s),
// fp32 123 us (5.0), two of fp32 25600 x 5120 321 us (5.0).
constexpr int ROWS = 128, COLS = 64;
template <typename E, bool ROW, bool COL, bool NOISE>
__global__ __launch_bounds__(THREADS) void k_mx_quantize(MxMats m) {
  constexpr bool PAIRS = NOISE && sizeof(E) == 2;   // two elements at a time where their scale allows it
  __shared__ __attribute__((aligned(32))) E tile[COL ? ROWS * COLS : 1];
  __shared__ __attribute__((aligned(8))) uint8_t tile_noise[COL && NOISE ? ROWS * COLS : 1];
  __shared__ unsigned row_scales[2][2][16], col_scales[4][16];   // 64 rows, block, slot; block, slot: dwords of the units' order
  const int t = threadIdx.x, which = blockIdx.z;
  const uint2 at = tile_of_block();
  const int64_t r0 = static_cast<int64_t>(at.y) * ROWS, c0 = static_cast<int64_t>(at.x) * COLS;
  const E* const src = static_cast<const E*>(m.mat[which]);
  const uint8_t* const noise = NOISE ? m.noise[which] : nullptr;
  const int ceil = m.scale_mode == CANZ_MX_SCALE_CEIL;
  const int64_t rows = m.rows[which], units_row = mx_k_units(m.cols), units_col = mx_k_units(rows);   // units along k of the two images
  if (r0 >= rows) return;   // a matrix of fewer rows than others of the launch
  const int kb0 = static_cast<int>(c0 / MX_BLOCK) & 3;                            // 0 or 2: the tile is one half of a k unit of by_row

  const int col = (t & 7) * 8;
  constexpr int EACH = ROWS / 32;   // rows of a thread
  Eight<E> x8[EACH];
  uint2 n8[EACH];
  const E* const from = src + (r0 + (t >> 3)) * m.ld + c0 + col;
  const uint8_t* const noise_from = NOISE ? noise + (r0 + (t >> 3)) * m.cols + c0 + col : nullptr;
  if (r0 + ROWS <= rows && c0 + COLS <= m.cols) {   // without a branch in between, so that all are on their way at once
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      x8[i] = load8(from + i * 32 * m.ld);
      n8[i] = {0, 0};
      if constexpr (NOISE) n8[i] = load_noise8(noise_from + i * 32 * m.cols);
    }
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t left = r0 + i * 32 + (t >> 3) < rows ? m.cols - (c0 + col) : 0;
      x8[i] = load8(from + i * 32 * m.ld, left);
      n8[i] = {0, 0};
      if constexpr (NOISE) n8[i] = load_noise8(noise_from + i * 32 * m.cols, left);
    }
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int row = i * 32 + (t >> 3);
    const uint2 noise8 = n8[i];
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x8[i][e]);
    if constexpr (COL) {
      *reinterpret_cast<Eight<E>*>(tile + row * COLS + col) = x8[i];
      if constexpr (NOISE) *reinterpret_cast<uint2*>(tile_noise + row * COLS + col) = noise8;
    }
    if constexpr (ROW) {
      PairMax<E> top;
#pragma unroll
      for (int e = 0; e < 8; e += 2) top.take({static_cast<E>(v[e]), static_cast<E>(v[e + 1])});
      const unsigned largest = largest_of_four(max(top.of(0), top.of(1))), byte = mx_scale_byte(largest, ceil);
      unsigned codes;
      if (PAIRS && in_pairs(byte, largest)) {
        const unsigned short less = less_of(byte);
        unsigned p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          p[e] = noisy_pair(__builtin_bit_cast(unsigned, mx_bf16x2{static_cast<__bf16>(v[2 * e]), static_cast<__bf16>(v[2 * e + 1])}), u16x2{less, less},
                            __builtin_amdgcn_perm(0u, e < 2 ? noise8.x : noise8.y, e & 1 ? NOISE_HIGH : NOISE_LOW));
        const uint2 even_odd = by_halves(p[0], p[1], p[2], p[3]);
        codes = byte == MX_SCALE_NAN ? 0u : even_odd.x | even_odd.y << 4;
      } else {
        unsigned u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = (e < 4 ? noise8.x : noise8.y) >> (8 * (e & 3)) & 255u;
        codes = eight_codes<NOISE>(v, byte, u);
      }
      const int kb = (t & 7) >> 2;
      const int64_t unit = mx_unit(r0 + row);
      if (unit < mx_row_tiles(rows))
        *reinterpret_cast<unsigned*>(m.by_row[which] + (unit * units_row + c0 / MX_UNIT_K) * MX_UNIT_BYTES + ((kb0 + kb) * 16 + mx_slot(row)) * 16 +
                                     (t & 3) * 4) = codes;
      if ((t & 3) == 0) reinterpret_cast<uint8_t*>(&row_scales[row >> 6][kb][mx_slot(row)])[mx_unit(row) % 4] = static_cast<uint8_t>(byte);
    }
  }
  __syncthreads();
  if constexpr (COL) {
    // two neighbouring columns of 32 rows per thread: one LDS access takes both
    typedef E pair __attribute__((ext_vector_type(2)));
    const int c = (t & 31) * 2, rb = t >> 5;
    if (rb < ROWS / MX_BLOCK && c0 < m.cols) {
      pair x[MX_BLOCK];
      PairMax<E> top;
#pragma unroll
      for (int e = 0; e < MX_BLOCK; ++e) {
        x[e] = *reinterpret_cast<const pair*>(tile + (rb * MX_BLOCK + e) * COLS + c);
        top.take(x[e]);
      }
      auto noise_of = [&](int e) CANZ_INLINE {   // of both
        unsigned n = 0;
        if constexpr (NOISE) n = *reinterpret_cast<const unsigned short*>(tile_noise + (rb * MX_BLOCK + e) * COLS + c);
        return n;
      };
      const unsigned byte[2] = {mx_scale_byte(top.of(0), ceil), mx_scale_byte(top.of(1), ceil)};
      u32x4 codes[2] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
      if (PAIRS && in_pairs(byte[0], top.of(0)) && in_pairs(byte[1], top.of(1))) {
        const u16x2 less = {less_of(byte[0]), less_of(byte[1])};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          unsigned p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            unsigned both = 0;
            if constexpr (sizeof(E) == 2) both = __builtin_bit_cast(unsigned, x[w * 8 + e]);
            p[e] = noisy_pair(both, less, __builtin_amdgcn_perm(0u, noise_of(w * 8 + e), NOISE_LOW));
          }
          const uint2 even = by_halves(p[0], p[2], p[4], p[6]), odd = by_halves(p[1], p[3], p[5], p[7]);
          codes[0][w] = byte[0] == MX_SCALE_NAN ? 0u : even.x | odd.x << 4;
          codes[1][w] = byte[1] == MX_SCALE_NAN ? 0u : even.y | odd.y << 4;
        }
      } else if constexpr (PAIRS) {   // rare: a rolled loop over what LDS holds, so that it takes no registers
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
          const u32x4 rest[2] = {codes[0], codes[1]};
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float v[8];
            unsigned u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = static_cast<float>(tile[(rb * MX_BLOCK + w * 8 + e) * COLS + c + q]);
              u[e] = noise_of(w * 8 + e) >> (8 * q) & 255u;
            }
            codes[q] = u32x4{rest[q][1], rest[q][2], rest[q][3], eight_codes<NOISE>(v, byte[q], u)};   // the vector turns instead of being indexed
          }
        }
      } else {
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            float v[8];
            unsigned u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x[w * 8 + e][q]), u[e] = noise_of(w * 8 + e) >> (8 * q) & 255u;
            codes[q][w] = eight_codes<NOISE>(v, byte[q], u);
          }
      }
      const int64_t unit = mx_unit(c0 + c);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        *reinterpret_cast<u32x4*>(m.by_col[which] + (unit * units_col + r0 / MX_UNIT_K) * MX_UNIT_BYTES + (rb * 16 + mx_slot(c + q)) * 16) = codes[q];
        reinterpret_cast<uint8_t*>(&col_scales[rb][mx_slot(c + q)])[mx_unit(c) % 4] = static_cast<uint8_t>(byte[q]);
      }
    }
    __syncthreads();
  }
  const int half = t >> 5 & 1, word = t & 31;
  if (ROW && t < 64 && r0 + half * MX_PAD_ROWS < rows)
    *reinterpret_cast<unsigned*>(m.by_row[which] + mx_code_bytes(rows, m.cols) +
                                 ((r0 / MX_PAD_ROWS + half) * units_row + c0 / MX_UNIT_K) * MX_SCALE_BYTES + (kb0 * 16 + word) * 4) = row_scales[half][word >> 4][word & 15];
  if (COL && t >= 64 && t < 128 && c0 < m.cols)
    *reinterpret_cast<unsigned*>(m.by_col[which] + mx_code_bytes(m.cols, rows) +
                                 (c0 / MX_PAD_ROWS * units_col + r0 / MX_UNIT_K) * MX_SCALE_BYTES + (t - 64) * 4) = col_scales[(t - 64) >> 4][t & 15];
}

__device__ __forceinline__ void eight_values(unsigned codes, unsigned byte, float (&v)[8]) {
  const float s = mx_scale_value(byte == MX_SCALE_NAN ? 127u : byte);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
  if (byte == MX_SCALE_NAN)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_nanf("");
}

// The values of a tile of 128 x 128 elements of the caller's matrix, from either image (the transposed one by way of LDS).  What is written bounds it: bf16 2 of
// 25600 x 5120 141 us from by_row and 127 from by_col (0.66 GB, 4.7 and 5.2 TB/s), 3 of 4097 x 1531, whose rows begin anywhere, 10.7 and 11.7 us (4.4 and 4.1).
// fp32: 337 and 255 us (3.5 and 4.65 TB/s), 17.7 and 21.6 us (4.8 and 4.0).
template <typename E, bool COL>
__global__ __launch_bounds__(THREADS) void k_mx_dequantize(MxMats m) {
  constexpr int LDT = TILE + 8 / sizeof(E);
  __shared__ E tile[COL ? TILE * LDT : 1];
  const int t = threadIdx.x, which = blockIdx.z;
  const uint2 at = tile_of_block();
  const int64_t r0 = static_cast<int64_t>(at.y) * TILE, c0 = static_cast<int64_t>(at.x) * TILE;
  E* const dst = static_cast<E*>(m.mat[which]);
  const int64_t rows = m.rows[which];
  if constexpr (COL) {
    const uint8_t* const img = m.by_col[which];
    const int64_t units = mx_k_units(rows), ks = r0 / MX_UNIT_K;
    const int c = t & (TILE - 1);
    const int64_t unit = mx_unit(c0 + c);
    if (c0 + c < m.cols) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int rb = (t >> 7) + 2 * i;
        const u32x4 codes = *reinterpret_cast<const u32x4*>(img + (unit * units + ks) * MX_UNIT_BYTES + (rb * 16 + mx_slot(c)) * 16);
        const unsigned byte = img[mx_code_bytes(m.cols, rows) + (unit / 4 * units + ks) * MX_SCALE_BYTES + (rb * 16 + mx_slot(c)) * 4 + unit % 4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[8];
          eight_values(codes[q], byte, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) tile[(rb * MX_BLOCK + q * 8 + e) * LDT + c] = static_cast<E>(v[e]);
        }
      }
    }
    __syncthreads();
  }
  const int col = (t & 15) * 8;
  const int64_t left = m.cols - (c0 + col);
  if (left <= 0) return;
#pragma unroll 4
  for (int i = 0; i < TILE / 16; ++i) {
    const int row = i * 16 + (t >> 4);
    if (r0 + row >= rows) break;
    float v[8];
    if constexpr (COL) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(tile[row * LDT + col + e]);
    } else {
      const uint8_t* const img = m.by_row[which];
      const int64_t units = mx_k_units(m.cols), ks = c0 / MX_UNIT_K, unit = mx_unit(r0 + row);
      const int slot = ((t & 15) >> 2) * 16 + mx_slot(row);
      const unsigned codes = *reinterpret_cast<const unsigned*>(img + (unit * units + ks) * MX_UNIT_BYTES + slot * 16 + (t & 3) * 4);
      const unsigned byte = img[mx_code_bytes(rows, m.cols) + (unit / 4 * units + ks) * MX_SCALE_BYTES + slot * 4 + unit % 4];
      eight_values(codes, byte, v);
    }
    store8(dst + (r0 + row) * m.ld + c0 + col, left, v);
  }
}

// tiles along the columns, along the rows (32768 at most), matrices
dim3 tiles_of(const MxMats& m, int64_t rows, int64_t cols) {
  return dim3(static_cast<unsigned>((m.cols + cols - 1) / cols), static_cast<unsigned>((m.most_rows + rows - 1) / rows), static_cast<unsigned>(m.n));
}

template <typename E, bool NOISE>
void quantize_sides(const MxMats& m, hipStream_t st) {
  // the images' padding along k is written too: by_row's last unit of 128 columns has two tiles
  MxMats padded = m;
  padded.cols = m.by_row[0] ? mx_k_units(m.cols) * MX_UNIT_K : m.cols;
  const dim3 grid = tiles_of(padded, ROWS, COLS);
  if (m.by_row[0] && m.by_col[0])
    k_mx_quantize<E, true, true, NOISE><<<grid, THREADS, 0, st>>>(m);
  else if (m.by_row[0])
    k_mx_quantize<E, true, false, NOISE><<<grid, THREADS, 0, st>>>(m);
  else
    k_mx_quantize<E, false, true, NOISE><<<grid, THREADS, 0, st>>>(m);
}

}  // namespace

hipError_t launch_mx_quantize(const MxMats& m, hipStream_t st) {
  if (m.dtype == CANZ_DT_F32)
    m.noise[0] ? quantize_sides<float, true>(m, st) : quantize_sides<float, false>(m, st);
  else
    m.noise[0] ? quantize_sides<__bf16, true>(m, st) : quantize_sides<__bf16, false>(m, st);
  return hipGetLastError();
}

hipError_t launch_mx_dequantize(const MxMats& m, hipStream_t st) {
  const bool col = m.by_col[0] != nullptr;
  if (m.dtype == CANZ_DT_F32)
    col ? k_mx_dequantize<float, true><<<tiles_of(m, TILE, TILE), THREADS, 0, st>>>(m) : k_mx_dequantize<float, false><<<tiles_of(m, TILE, TILE), THREADS, 0, st>>>(m);
  else
    col ? k_mx_dequantize<__bf16, true><<<tiles_of(m, TILE, TILE), THREADS, 0, st>>>(m) : k_mx_dequantize<__bf16, false><<<tiles_of(m, TILE, TILE), THREADS, 0, st>>>(m);
  return hipGetLastError();
}

}  // namespace canz
