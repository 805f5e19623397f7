// 8-bit images (include/canz.h: canz_mx_eight_store): layout, and rounding of a piece of a row, shared by every kernel that makes or reads them.
#pragma once
#include "device_util.h"
#include "mx.h"

namespace canz {

constexpr int MX8_BLOCK = 32;    // elements that share a scale
constexpr int MX8_PITCH = 128;   // rows of codes are padded to this many bytes, so that a piece of codes never crosses a row and a row's scales are whole dwords
constexpr int PIECE = 8;         // elements of a row that a thread takes at a time: 8 codes, 16 bytes of bf16; four threads hold a block

__host__ __device__ constexpr int64_t mx8_pitch(int64_t cols) { return (cols + MX8_PITCH - 1) / MX8_PITCH * MX8_PITCH; }
__host__ __device__ constexpr int64_t mx8_code_bytes(int64_t rows, int64_t cols) { return rows * mx8_pitch(cols); }
constexpr int64_t mx8_bytes(int64_t rows, int64_t cols) {
  return (mx8_code_bytes(rows, cols) / MX8_BLOCK * (MX8_BLOCK + 1) + 255) / 256 * 256;
}

// An image as the kernels see it.
struct Image8 {
  uint8_t* codes;
  uint8_t* scales;
  int64_t pitch;   // of codes; scales have a 32nd of it
};
inline Image8 image8(const void* at, int64_t rows, int64_t cols) {
  uint8_t* const p = static_cast<uint8_t*>(const_cast<void*>(at));
  return Image8{p, p ? p + mx8_code_bytes(rows, cols) : nullptr, mx8_pitch(cols)};
}

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// Eight consecutive elements of a row as they come from memory: converted where they are used, so that the loads of several pieces are in flight together.
template <typename E>
struct Raw {
  typedef E vec __attribute__((ext_vector_type(8)));
  vec v;
};
// From p on, of which `left` are there; zeros for the others.
template <typename E>
__device__ __forceinline__ Raw<E> load_raw(const E* p, int64_t left) {
  Raw<E> r;
  if (left >= PIECE) {
    typedef E any __attribute__((ext_vector_type(8), aligned(sizeof(E))));
    r.v = *reinterpret_cast<const any*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < PIECE; ++e) r.v[e] = static_cast<E>(0.f);
#pragma unroll
    for (int e = 0; e < PIECE - 1; ++e)
      if (e < left) r.v[e] = p[e];
  }
  return r;
}
template <typename E>
__device__ __forceinline__ f32x8 widen(const Raw<E>& r) {
  f32x8 v;
#pragma unroll
  for (int e = 0; e < PIECE; ++e) v[e] = static_cast<float>(r.v[e]);
  return v;
}
template <typename E>
__device__ __forceinline__ void store_piece8(E* p, int64_t left, f32x8 v) {
  if (left >= PIECE) {
    if constexpr (sizeof(E) == 4) {
      *reinterpret_cast<f32x4_any*>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4_any*>(p + 4) = f32x4_any{v[4], v[5], v[6], v[7]};
    } else {
      bf16x8_any x;
#pragma unroll
      for (int e = 0; e < PIECE; ++e) x[e] = static_cast<__bf16>(v[e]);
      *reinterpret_cast<bf16x8_any*>(p) = x;
    }
  } else {
#pragma unroll
    for (int e = 0; e < PIECE - 1; ++e)
      if (e < left) p[e] = static_cast<E>(v[e]);
  }
}

// Scale byte of a block whose largest magnitude has the bits `amax`.  448 = 1.75 2^8: with E the biased exponent, X = 2^(E - 127 - 8), twice that where the
// mantissa is above 1.75, at least 2^-124 (byte 3) and at most 2^119 (byte 246), so that every value is finite: 448 2^119 is 1.75 2^127.
constexpr unsigned MX8_LARGEST = 0x7F600000u;   // the bits of that
__device__ __forceinline__ unsigned mx8_scale_byte(unsigned amax) {
  constexpr unsigned NONFINITE = 0x7F800000u;
  const int e = static_cast<int>(amax >> 23) - 8 + static_cast<int>((amax & 0x7FFFFFu) > 0x600000u);
  return amax >= NONFINITE ? 255u : static_cast<unsigned>(min(max(e, 3), 246));
}

// By value: __builtin_bit_cast of an element of a vector takes the vector's first.
__device__ __forceinline__ unsigned magnitude(float v) { return __builtin_bit_cast(unsigned, v) & 0x7FFFFFFFu; }

// The largest of four neighbouring lanes' values (quad permutes).
__device__ __forceinline__ unsigned quad_max(unsigned v) {
  v = max(v, static_cast<unsigned>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xF, 0xF, false)));
  return max(v, static_cast<unsigned>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xF, 0xF, false)));
}

// Rounds a lane's eight elements of a block that it shares with the other three lanes of its quad, which all have to be active.  1 / X is a power of two
// within fp32's normal range (bytes 3 .. 246), so that the quotients are exact (below 2^-126 they round, far below half of the smallest code), and they are at most 448: the
// conversion rounds to the nearest code, ties to even.
struct Codes8 {
  u32x2 codes;
  unsigned scale;
};
__device__ __forceinline__ Codes8 round8(f32x8 v) {
  unsigned top = 0;
#pragma unroll
  for (int e = 0; e < PIECE; ++e) top = max(top, magnitude(v[e]));
  Codes8 r;
  top = quad_max(top);
  r.scale = mx8_scale_byte(top);
  if (top > MX8_LARGEST) {
    const float most = __builtin_bit_cast(float, MX8_LARGEST);
#pragma unroll
    for (int e = 0; e < PIECE; ++e) v[e] = __builtin_fminf(__builtin_fmaxf(v[e], -most), most);
  }
  const float inverse = __builtin_bit_cast(float, (254u - r.scale) << 23);
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inverse, v[5] * inverse, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inverse, v[7] * inverse, hi, true);
  const bool nan = r.scale == 255u;
  r.codes = u32x2{nan ? 0u : static_cast<unsigned>(lo), nan ? 0u : static_cast<unsigned>(hi)};
  return r;
}
// Stores the piece that begins at column `col` (below the pitch) of a row, and the block's scale byte.
__device__ __forceinline__ void store_codes(const Image8& im, int64_t row, int64_t col, int64_t cols, const Codes8& c) {
  *reinterpret_cast<u32x2*>(im.codes + row * im.pitch + col) = c.codes;
  if ((col & (MX8_BLOCK - 1)) == 0) im.scales[row * (im.pitch / MX8_BLOCK) + col / MX8_BLOCK] = col < cols ? static_cast<uint8_t>(c.scale) : 0;
}

// The values of eight codes, exact in fp32: X times a code of 4 significant bits, at least 2^-127 2^-9; from byte 247 on, which images made elsewhere may have, the largest are infinities.
__device__ __forceinline__ f32x8 values8(u32x2 codes, unsigned scale) {
  // byte 255 has the exponent field of an infinity; it stands for NaN.  Byte 0 has that of a subnormal number, 2^-127 with the mantissa 1/2
  const float x = __builtin_bit_cast(float, scale == 255u ? 0x7FC00000u : max(scale << 23, 0x00400000u));
  f32x8 v;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[h]), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[h]), true);
    v[4 * h] = a[0] * x, v[4 * h + 1] = a[1] * x, v[4 * h + 2] = b[0] * x, v[4 * h + 3] = b[1] * x;
  }
  return v;
}
// The piece that begins at column `col` of a row, as it comes from memory; padding is read as it lies there (zeros).
struct RawCodes {
  u32x2 codes;
  unsigned scale;
};
__device__ __forceinline__ RawCodes load_raw(const Image8& im, int64_t row, int64_t col) {
  return RawCodes{*reinterpret_cast<const u32x2*>(im.codes + row * im.pitch + col), im.scales[row * (im.pitch / MX8_BLOCK) + col / MX8_BLOCK]};
}
__device__ __forceinline__ f32x8 widen(const RawCodes& r) { return values8(r.codes, r.scale); }

// How the blocks of an elementwise kernel go over a matrix: a block of 256 threads has 2^log_tx pieces of a row side by side and 256 / 2^log_tx rows at a time; blocks
// that follow one another are neighbours along the row.
constexpr int EACH_THREADS = 256;
struct Cover {
  int log_tx;
  int across;        // blocks along a row
  int64_t blocks;
};
inline Cover cover(int64_t rows, int64_t cols) {
  const int64_t pieces = mx8_pitch(cols) / PIECE;   // a multiple of 16
  int log_tx = 8;
  while (pieces % (int64_t{1} << log_tx) != 0) --log_tx;
  const int64_t across = pieces >> log_tx, high = EACH_THREADS >> log_tx;
  return Cover{log_tx, static_cast<int>(across), across * ((rows + high - 1) / high)};
}
// This thread's row (there may be none) and its column.
struct Spot {
  int64_t row, col;
};
__device__ __forceinline__ Spot spot(unsigned block, int log_tx, int across) {
  const unsigned down = block / static_cast<unsigned>(across), along = block - down * across;
  const int ty = threadIdx.x >> log_tx, tx = threadIdx.x & ((1 << log_tx) - 1);
  return Spot{static_cast<int64_t>(down) * (EACH_THREADS >> log_tx) + ty, ((static_cast<int64_t>(along) << log_tx) + tx) * PIECE};
}

// Checks that the entry points share.
// Elements of a matrix, padded to 128 either way: a launch has fewer than 2^32 threads, and a thread at least 8 elements.
constexpr bool fits_launch(int64_t rows, int64_t cols) { return ((rows + 127) / 128) * ((cols + 127) / 128) <= (int64_t(1) << 34) / (128 * 128); }
constexpr int64_t MOST_BLOCKS = (int64_t(1) << 24) - 1;   // of EACH_THREADS in a launch
inline bool misaligned(const void* p, uintptr_t align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; }
constexpr bool float_dtype(int32_t t) { return t == CANZ_DT_F32 || t == CANZ_DT_BF16; }
constexpr uintptr_t element_bytes(int32_t t) { return t == CANZ_DT_F32 ? 4 : 2; }
// Extents of a matrix that the elementwise kernels go over.
int check_extents(const char* what, int idx, int64_t rows, int64_t cols);

}  // namespace canz
