// Products of microscaled 4-bit images: C[i][j] = alpha sum_k A[i][k] B[j][k] + beta C[i][j], fp32 sums.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows of either image over 128 k, scales included; a product of two elements is exact
// in fp32.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "device_util.h"
#include "mx.h"
#include "mx_round.h"

namespace canz {
namespace {

constexpr int THREADS = 256;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

#define CANZ_LDS(p) ((__attribute__((address_space(3))) void*)(p))
#define CANZ_GLB(p) ((const __attribute__((address_space(1))) void*)(p))
#define CANZ_INLINE __attribute__((always_inline))
#define CANZ_FENCE() __builtin_amdgcn_sched_barrier(0)

// A kernel's argument where it lies: scalar loads at any index, and no copy of it.
typedef const __attribute__((address_space(4))) MxProblems* KernArgs;

template <typename F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for(f, std::make_integer_sequence<int, N>{});
}

// SIZE bytes a lane from base + lane_off + off straight into LDS, lane after lane; zeros beyond the `room` bytes of the buffer.
template <int SIZE>
__device__ __forceinline__ void buffer_to_lds(const uint8_t* base, unsigned room, __attribute__((address_space(3))) void* lds, int lane_off, int off) {
#if defined(__HIP_DEVICE_COMPILE__)   // the descriptor's type is the device's only
  constexpr int RAW = 0x00027000;     // a raw buffer of dwords
  const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), static_cast<short>(0), static_cast<int>(room), RAW);
  if constexpr (SIZE == 16)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, lds, 16, lane_off, off, 0, 0);
  else
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, lds, 4, lane_off, off, 0, 0);
#endif
}

// Which of the launch's pieces of work this block has: the blocks of one XCD (blockIdx % 8) are neighbours, and share what they read in its L2.
constexpr int N_XCD = 8;
__device__ __forceinline__ int xcd_slot() {
  const int per = gridDim.x / N_XCD, rem = gridDim.x % N_XCD, xcd = blockIdx.x % N_XCD, q = blockIdx.x / N_XCD;
  return xcd < rem ? xcd * (per + 1) + q : rem * (per + 1) + (xcd - rem) * per + q;
}

// acc[16 slots of p][16 slots of q] += P Q^T over 128 k; SP, SQ: which byte of its scale register belongs to the unit
template <int SP, int SQ>
__device__ __forceinline__ f32x4 mfma(i32x4 p, i32x4 q, f32x4 acc, int scale_p, int scale_q) {
  constexpr int FP4 = 4;   // operand format E2M1: four registers of the eight other formats take
  const i32x8 a = {p[0], p[1], p[2], p[3], 0, 0, 0, 0}, b = {q[0], q[1], q[2], q[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, FP4, FP4, SP, scale_p, SQ, scale_q);
}

// Eight consecutive elements of a row of C, of which `left` are there.
template <typename E>
__device__ __forceinline__ f32x8 load_old(const E* c, int64_t left) {
  f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (left >= 8) {
    typedef E vec __attribute__((ext_vector_type(8), aligned(sizeof(E))));
    const vec x = *reinterpret_cast<const vec*>(c);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x[e]);
  } else {
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {   // a rolled loop: the vector turns instead of being indexed
      const float x = e < left ? static_cast<float>(c[e]) : 0.f;
      v = f32x8{v[1], v[2], v[3], v[4], v[5], v[6], v[7], x};
    }
  }
  return v;
}
// 16 bytes of a row of C, of which `left` elements are there.
template <typename E>
__device__ __forceinline__ void store_piece(E* c, int64_t left, i32x4 v) {
  constexpr int N = 16 / sizeof(E);
  if (left >= N) {
    typedef E any __attribute__((ext_vector_type(N), aligned(sizeof(E))));
    *reinterpret_cast<any*>(c) = __builtin_bit_cast(any, v);
  } else {
#pragma unroll 1
    for (int e = 0; e < left; ++e) {   // a rolled loop: the piece moves down instead of being indexed
      if constexpr (sizeof(E) == 4) {
        c[e] = __builtin_bit_cast(float, v[0]);
        v = i32x4{v[1], v[2], v[3], 0};
      } else {
        c[e] = __builtin_bit_cast(__bf16, static_cast<short>(v[0]));
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = static_cast<int>(static_cast<unsigned>(v[q]) >> 16 | (q < 3 ? static_cast<unsigned>(v[q < 3 ? q + 1 : 3]) << 16 : 0u));
      }
    }
  }
}

// ---- few rows: B goes by once -------------------------------------------------------------------------------------------------
// A block has UN units of 16 rows of B and all of k, which its wavefronts share unit by unit, so that together they read B in long pieces; A's
// units (UM of 16 rows) are multiplied with it from registers, and the wavefronts' sums are added in LDS in their order.  Memory is all
// that takes time, and each wavefront keeps AHEAD units in flight: 1 x 25600 x 5120 goes at 4.6 TB/s (15.1 us), 1 x 5120 x 25600, whose 160 blocks leave CUs
// without one, at 3.8 from bf16 and 4.6 from an image (18.2 and 15.2 us); a copy of 2 GiB reaches 4.65 TB/s here.
//
// The operand layout gives a lane 32 consecutive elements of one row, a block: a matrix A is rounded by the lane that needs it, without
// a word to another one, so that a call of few rows is one launch.

// the operand of one lane: 32 elements and their scale byte
struct Block {
  i32x4 codes;
  int scale;
};
template <typename A>
struct RawBlock;   // 32 elements on their way from memory
template <>
struct RawBlock<uint8_t> {
  i32x4 codes;
};
template <>
struct RawBlock<__bf16> {
  typedef bf16x8_any part;   // 16 bytes, anywhere
  part v[4];
};
template <>
struct RawBlock<float> {
  typedef f32x4_any part;
  part v[8];
};
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ Block round_block(const RawBlock<__bf16>& x, int ceil) {
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const i32x4 w = __builtin_bit_cast(i32x4, x.v[i]);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[e] & 0x7FFF7FFF));
  }
  const unsigned byte = mx_scale_byte(static_cast<unsigned>(max(top[0], top[1])) << 16, ceil);
  const float s = mx_scale_value(byte);
  Block r;
  r.scale = static_cast<int>(byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, mx_bf16x2{x.v[i][0], x.v[i][1]}, s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, mx_bf16x2{x.v[i][2], x.v[i][3]}, s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, mx_bf16x2{x.v[i][4], x.v[i][5]}, s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, mx_bf16x2{x.v[i][6], x.v[i][7]}, s, 3);
    r.codes[i] = static_cast<int>(c);
  }
  return r;
}
__device__ __forceinline__ Block round_block(const RawBlock<float>& x, int ceil) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, mx_magnitude(x.v[i][e]));
  const unsigned byte = mx_scale_byte(top, ceil);
  const float s = mx_scale_value(byte);
  Block r;
  r.scale = static_cast<int>(byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[2 * i][0], x.v[2 * i][1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[2 * i][2], x.v[2 * i][3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[2 * i + 1][0], x.v[2 * i + 1][1], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[2 * i + 1][2], x.v[2 * i + 1][3], s, 3);
    r.codes[i] = static_cast<int>(c);
  }
  return r;
}

// A: uint8_t for an image, or the type of the matrix
template <typename A, int UM, int UN, int WAVES, int AHEAD>
__global__ __launch_bounds__(64 * WAVES) void k_mx_product_few(MxProblems) {
  constexpr bool IMAGE = sizeof(A) == 1;
  const KernArgs ps = (KernArgs)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ f32x4 sums[WAVES][UM * UN][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slot = xcd_slot();
  int j = 0;
  while (slot >= ps->first_tile[j + 1]) ++j;
  const int64_t m = ps->pr[j].m, n = ps->pr[j].n, k = ps->pr[j].k, lda = ps->pr[j].lda;
  const int64_t part = slot - ps->first_tile[j];   // of B
  const int ks = static_cast<int>(mx_k_units(k));
  const uint8_t* const bc = ps->pr[j].b + part * UN * ks * MX_UNIT_BYTES + lane * 16;
  const uint8_t* const bs = ps->pr[j].b + mx_code_bytes(n, k) + part * UN / 4 * ks * MX_SCALE_BYTES + lane * 4;
  const int b_shift = UN == 4 ? 0 : static_cast<int>(part % (4 / UN)) * UN * 8;
  const uint8_t* const a = ps->pr[j].a;
  // this lane's row of every 16, at its block of unit 0, in the image or in the matrix; a row that is not there is read as the last
  const uint8_t *codes[UM], *scales[UM];
  int a_shift[UM];
  const A* row[UM];
#pragma unroll
  for (int i = 0; i < UM; ++i) {
    const int r = min(i * 16 + (lane & 15), static_cast<int>(m) - 1);
    if constexpr (IMAGE) {
      const int at = (lane >> 4) * 16 + mx_slot(r);
      codes[i] = a + static_cast<int64_t>(mx_unit(r)) * ks * MX_UNIT_BYTES + at * 16;
      scales[i] = a + mx_code_bytes(m, k) + at * 4;
      a_shift[i] = mx_unit(r) * 8;
    } else {
      row[i] = reinterpret_cast<const A*>(a) + r * lda + (lane >> 4) * MX_BLOCK;
    }
  }
  const int ceil = ps->pr[j].a_ceil;
  f32x4 acc[UM][UN] = {};
  RawBlock<A> ra[AHEAD][UM];
  i32x4 rb[AHEAD][UN];
  int rsa[AHEAD][UM], rsb[AHEAD];
  auto load_b = [&](int d, int64_t u) CANZ_INLINE {
#pragma unroll
    for (int q = 0; q < UN; ++q) rb[d][q] = *reinterpret_cast<const i32x4*>(bc + (static_cast<int64_t>(q) * ks + u) * MX_UNIT_BYTES);
    rsb[d] = *reinterpret_cast<const int*>(bs + u * MX_SCALE_BYTES);
  };
  auto load = [&](int d, int64_t u) CANZ_INLINE {
    load_b(d, u);
#pragma unroll
    for (int i = 0; i < UM; ++i) {
      if constexpr (IMAGE) {
        ra[d][i].codes = *reinterpret_cast<const i32x4*>(codes[i] + u * MX_UNIT_BYTES);
        rsa[d][i] = *reinterpret_cast<const int*>(scales[i] + u * MX_SCALE_BYTES);
      } else {
        constexpr int PARTS = sizeof(ra[d][i].v) / 16;
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
          ra[d][i].v[q] = *reinterpret_cast<const typename RawBlock<A>::part*>(row[i] + u * MX_UNIT_K + q * (MX_BLOCK / PARTS));
      }
    }
  };
  // `there`: a unit that is not there was read as another one and counts nothing
  auto multiply = [&](int d, bool there) CANZ_INLINE {
    const int vb = rsb[d] >> b_shift;
    static_for<UM>([&](auto x) CANZ_INLINE {
      constexpr int i = decltype(x)::value;
      Block b;
      if constexpr (IMAGE)
        b.codes = ra[d][i].codes, b.scale = rsa[d][i] >> a_shift[i];
      else
        b = round_block(ra[d][i], ceil);
#pragma unroll
      for (int e = 0; e < 4; ++e) b.codes[e] = there ? b.codes[e] : 0;
      static_for<UN>([&](auto y) CANZ_INLINE {
        constexpr int q = decltype(y)::value;
        acc[i][q] = mfma<q, 0>(rb[d][q], b.codes, acc[i][q], vb, b.scale);
      });
    });
  };
  // units that are there as a whole; the last one of a matrix may not be
  const int whole = IMAGE ? ks : static_cast<int>(k / MX_UNIT_K);
  if (wave < whole) {
    const int last = whole - 1;
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      load(d, min(wave + d * WAVES, last));
      CANZ_FENCE();   // in this order, or the compiler has no count of the younger loads to wait with
    }
    int u = wave;
#pragma clang loop unroll(disable)
    for (; u + AHEAD * WAVES < whole; u += AHEAD * WAVES) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) {
        multiply(d, true);
        CANZ_FENCE();
        load(d, min(u + (AHEAD + d) * WAVES, last));
        CANZ_FENCE();
      }
    }
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      multiply(d, u + d * WAVES < whole);
      CANZ_FENCE();
    }
  }
  if (!IMAGE && whole < ks && wave == whole % WAVES) {
    load_b(0, whole);
    const int64_t left = k - static_cast<int64_t>(whole) * MX_UNIT_K - (lane >> 4) * MX_BLOCK;   // of this lane's block
#pragma unroll
    for (int i = 0; i < UM; ++i) {
      if constexpr (!IMAGE) {
        constexpr int EACH = 16 / sizeof(A);
#pragma unroll
        for (int e = 0; e < MX_BLOCK; ++e)
          ra[0][i].v[e / EACH][e % EACH] = e < left ? row[i][static_cast<int64_t>(whole) * MX_UNIT_K + e] : static_cast<A>(0.f);
      }
    }
    multiply(0, true);
  }
#pragma unroll
  for (int i = 0; i < UM; ++i)
#pragma unroll
    for (int q = 0; q < UN; ++q) sums[wave][i * UN + q][lane] = acc[i][q];
  __syncthreads();
  // four columns of a row per thread
  for (int e = threadIdx.x; e < UM * UN * 64; e += 64 * WAVES) {
    const int tile = e >> 6, l = e & 63;
    f32x4 s = sums[0][tile][l];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += sums[w][tile][l];
    const int64_t r = tile / UN * 16 + (l & 15), col = mx_row(part * UN + tile % UN, static_cast<int64_t>(l >> 4) * 4);
    if (r >= m || col >= n) continue;
    const float alpha = ps->pr[j].alpha, beta = ps->pr[j].beta;
    const int64_t left = n - col, at = r * ps->pr[j].ldc + col;
    auto finish = [&](auto* c) CANZ_INLINE {
      using E = std::remove_pointer_t<decltype(c)>;
      typedef E vec __attribute__((ext_vector_type(4), aligned(sizeof(E))));
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[q] = alpha * s[q];
        if (beta != 0.f && q < left) v[q] = __builtin_fmaf(beta, static_cast<float>(c[q]), v[q]);
      }
      if (left >= 4) {
        *reinterpret_cast<vec*>(c) = vec{static_cast<E>(v[0]), static_cast<E>(v[1]), static_cast<E>(v[2]), static_cast<E>(v[3])};
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < left) c[q] = static_cast<E>(v[q]);
      }
    };
    void* const c = ps->pr[j].c;
    if (ps->pr[j].out_dtype == CANZ_DT_F32)
      finish(static_cast<float*>(c) + at);
    else
      finish(static_cast<__bf16*>(c) + at);
  }
}

// ---- sums of parts of k -------------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(THREADS) void k_mx_join(MxProblem p, const float* sums, int parts) {
  const int64_t total = p.m * p.n;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * THREADS) {
    float part[MX_MAX_PARTS];
#pragma unroll
    for (int q = 0; q < MX_MAX_PARTS; ++q) part[q] = q < parts ? sums[q * total + i] : 0.f;   // all on their way before the first is added
    float v = part[0];
#pragma unroll
    for (int q = 1; q < MX_MAX_PARTS; ++q) v += part[q];
    v *= p.alpha;
    const int64_t at = i / p.n * p.ldc + i % p.n;
    if (p.out_dtype == CANZ_DT_F32) {
      float* const c = static_cast<float*>(p.c) + at;
      *c = p.beta != 0.f ? __builtin_fmaf(p.beta, *c, v) : v;
    } else {
      __bf16* const c = static_cast<__bf16*>(p.c) + at;
      *c = static_cast<__bf16>(p.beta != 0.f ? __builtin_fmaf(p.beta, static_cast<float>(*c), v) : v);
    }
  }
}

// ---- nothing along k: C <- beta C ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(THREADS) void k_mx_scale(MxProblem p) {
  const int64_t total = p.m * p.n;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * THREADS) {
    const int64_t at = i / p.n * p.ldc + i % p.n;
    if (p.out_dtype == CANZ_DT_F32) {
      float* const c = static_cast<float*>(p.c) + at;
      *c = p.beta != 0.f ? p.beta * *c : 0.f;
    } else {
      __bf16* const c = static_cast<__bf16*>(p.c) + at;
      *c = static_cast<__bf16>(p.beta != 0.f ? p.beta * static_cast<float>(*c) : 0.f);
    }
  }
}

// ---- tiles through LDS ------------------------------------------------------------------------------------------------------
// A block of four wavefronts (2 x 2) owns a tile of C, 2 W units of A by 2 W of B (W = 8: 256 x 256, W = 4: 128 x 128); a wavefront has
// W x W MFMA tiles.  A stage is one k unit of the tile's units, codes as they lie in the images (a wavefront copies 1 KiB per instruction
// straight into LDS) and scales.  256 x 256 is what the accumulators allow (256 of a wavefront's 512 registers), and the larger the tile the fewer
// bytes go from L2 into LDS and from there into registers for an operation.
//
// Four stages form a ring over the k units of all tiles of the block, one tile after another without a gap: while unit t is multiplied from
// registers, the operands of t + 1 are read from LDS into a second set, t + 2 and t + 3 are in flight and t + 4 is requested into the stage of
// t, which every wavefront has read before the barrier at the start of the step.  So there is one barrier per k unit, W W MFMAs long.
//
// What bounds it is power.  8192^3 takes 233 us (4.7 PFLOP/s), at 1.75 GHz instead of 2.4 with the matrix cores busy half of the cycles, and just as long with 128
// idle cycles added to every k unit; with zeros as operands, which cost less energy, 180 us at 2.4 GHz.  The matrix instructions alone, from registers, would
// take 157 us (7.0 PFLOP/s, 1.83 GHz).  Left out one by one, requests from L2 into LDS make 48 us of it, reads from LDS 18, stores 15.  (32 x 32 x 64
// instructions reach 6.2 PFLOP/s from registers, 16 x 16 x 128 ones 7.0: that is why images are laid out for the latter.)
// So W instructions after one another keep their second operand and change the first: with the first one kept 8192 x 12288 x 4096 takes 215 us instead of 198.
// Old results cost their bytes and the waiting for them behind a tile: 8192 x 4096 x 12288 bf16 180 us without and 206 with, fp32 188 and 210.
constexpr int BAND = 4;   // tile rows that are walked column by column: 8192^3 233 us, with 2 or 16 of them 238; 4096 x 25600 x 5120 266, 267 and 261

template <int W>
struct Stage {
  static constexpr int codes = 2 * W * MX_UNIT_BYTES;       // of one operand
  static constexpr int scales = 2 * W / 4 * MX_SCALE_BYTES;
  static constexpr int bytes = 2 * (codes + scales);        // A codes, B codes, A scales, B scales
  static constexpr int code_loads = W, scale_loads = W / 4, loads = code_loads + scale_loads;   // of one wavefront
};

// What a block has to do and has to load next: of the launch's tiles those numbered blockIdx.x, blockIdx.x + gridDim.x, ... (tile_at)
struct Tile {
  int problem;   // -1: none
  int m0, n0;    // in units of 16 rows
};
// Number `logical` of the launch's tiles.  Every XCD (blockIdx % 8, and logical % 8, since a grid has a multiple of 8 blocks) has an
// eighth of each product, in one piece: what its blocks work on at a time is a patch of neighbours that share operands in its L2, and products of
// unequal length burden all XCDs alike.
template <int W>
__device__ __forceinline__ Tile tile_at(KernArgs ps, int logical) {
  const int xcd = logical % N_XCD;
  int q = logical / N_XCD;
  for (int j = 0; j < ps->n; ++j) {
    const int tiles = ps->first_tile[j + 1] - ps->first_tile[j];
    const int begin = tiles * xcd / N_XCD, count = tiles * (xcd + 1) / N_XCD - begin;
    if (q >= count) {
      q -= count;
      continue;
    }
    const int tix = begin + q;
    const int tiles_m = static_cast<int>((ps->pr[j].m + 32 * W - 1) / (32 * W)), tiles_n = static_cast<int>((ps->pr[j].n + 32 * W - 1) / (32 * W));
    const int band = tix / (BAND * tiles_n), in_band = tix - band * BAND * tiles_n, rows = min(BAND, tiles_m - band * BAND);
    const int tn = in_band / rows;
    return Tile{j, (band * BAND + in_band - tn * rows) * 2 * W, tn * 2 * W};
  }
  return Tile{-1, 0, 0};
}

// ONLY, ONLY_BETA: the type of the results and whether old ones are read; void: as each product says
template <int W, typename ONLY, bool ONLY_BETA>
__global__ __launch_bounds__(THREADS, W == 8 ? 1 : 2) void k_mx_product(MxProblems) {
  using S = Stage<W>;
  const KernArgs ps = (KernArgs)__builtin_amdgcn_kernarg_segment_ptr();
  // one array per stage: the compiler then knows that a fetch into one stage does not alias the reads of another
  __shared__ __attribute__((aligned(1024))) uint8_t st0[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st1[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st2[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st3[S::bytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  // ---- loading: this wavefront's pieces of the next four stages.  Every tile takes whole rounds of the ring, so its loop has no exit
  // inside and the accumulators stay where they are; units behind the last one are asked for in an empty buffer, which gives zeros.
  // Through buffer descriptors (of the tile's codes and scales of either operand) a load is one instruction beside its LDS address: the piece is the
  // lane's offset, the unit a scalar one.
  Tile next_tile;   // the one that is loaded: the next one, from the last round of a tile on
  int next_logical = blockIdx.x, load_u = 0, load_ks = 0;        // load_ks: the end of the product's part of k
  const uint8_t *code_base[2], *scale_base[2];   // of A and B, from the tile's first unit on
  unsigned code_room[2], scale_room[2];          // bytes there
  int code_off[W], scale_off[S::scale_loads];    // this lane's part of its pieces
  auto next_round = [&]() CANZ_INLINE {
    load_u += 4;
    if (load_u < load_ks) return;
    const Tile t = next_tile = tile_at<W>(ps, next_logical);
    load_ks = 0;
    if (t.problem < 0) return;   // nothing left: zeros
    next_logical += gridDim.x;
    load_u = ps->pr[t.problem].first_unit, load_ks = load_u + ps->pr[t.problem].units;
    const int ks = static_cast<int>(mx_k_units(ps->pr[t.problem].k));
    const int row_bytes = ks * MX_UNIT_BYTES, scale_bytes = ks * MX_SCALE_BYTES;   // 2^25 at most
    int there[2];   // units of the tile that the image has
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const uint8_t* const image = o == 0 ? ps->pr[t.problem].a : ps->pr[t.problem].b;
      const int units = static_cast<int>(mx_row_tiles(o == 0 ? ps->pr[t.problem].m : ps->pr[t.problem].n)), first = o == 0 ? t.m0 : t.n0;
      there[o] = min(units - first, 2 * W);
      code_base[o] = image + static_cast<int64_t>(first) * row_bytes, code_room[o] = static_cast<unsigned>(there[o]) * row_bytes;
      scale_base[o] = image + static_cast<int64_t>(units) * row_bytes + static_cast<int64_t>(first / 4) * scale_bytes;
      scale_room[o] = static_cast<unsigned>(there[o] / 4) * scale_bytes;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {   // A's 2 W pieces, then B's; a unit that is not there is read as the last
      const int o = i < W / 2 ? 0 : 1, piece = wave + 4 * i - o * 2 * W;
      code_off[i] = min(piece, there[o] - 1) * row_bytes + lane * 16;
    }
#pragma unroll
    for (int i = 0; i < S::scale_loads; ++i) {
      const int piece = wave + 4 * i, o = piece < W / 2 ? 0 : 1;
      scale_off[i] = min(piece - o * (W / 2), there[o] / 4 - 1) * scale_bytes + lane * 4;
    }
  };
  auto fetch_one = [&](uint8_t* st, int u, auto idx) CANZ_INLINE {
    constexpr int I = decltype(idx)::value;
    const bool there = u < load_ks;
    if constexpr (I < W) {
      constexpr int o = I < W / 2 ? 0 : 1;
      buffer_to_lds<16>(code_base[o], there ? code_room[o] : 0u, CANZ_LDS(st + (wave + 4 * I) * MX_UNIT_BYTES), code_off[I],
                        there ? u * MX_UNIT_BYTES : 0);
    } else {
      constexpr int i = I - W;
      const int o = S::scale_loads == 2 ? i : wave < W / 2 ? 0 : 1;
      buffer_to_lds<4>(o == 0 ? scale_base[0] : scale_base[1], there ? (o == 0 ? scale_room[0] : scale_room[1]) : 0u,
                       CANZ_LDS(st + 2 * S::codes + (wave + 4 * i) * MX_SCALE_BYTES), scale_off[i], there ? u * MX_SCALE_BYTES : 0);
    }
  };

  // ---- operands in registers, two sets: W units of A and of B, and their scales, four units to a register
  i32x4 fa[2][W], fb[2][W];
  int sa[2][W / 4], sb[2][W / 4];
  f32x4 acc[W][W];
  constexpr int READS = 2 * W + W / 2;
  auto read_one = [&](const uint8_t* st, int set, auto idx) CANZ_INLINE {
    constexpr int I = decltype(idx)::value;
    if constexpr (I < W / 4)
      sb[set][I] = *reinterpret_cast<const int*>(st + 2 * S::codes + S::scales + (wn * (W / 4) + I) * MX_SCALE_BYTES + lane * 4);
    else if constexpr (I < W / 2)
      sa[set][I - W / 4] = *reinterpret_cast<const int*>(st + 2 * S::codes + (wm * (W / 4) + I - W / 4) * MX_SCALE_BYTES + lane * 4);
    else if constexpr (I < W / 2 + W)
      fb[set][I - W / 2] = *reinterpret_cast<const i32x4*>(st + S::codes + (wn * W + I - W / 2) * MX_UNIT_BYTES + lane * 16);
    else
      fa[set][I - W / 2 - W] = *reinterpret_cast<const i32x4*>(st + (wm * W + I - W / 2 - W) * MX_UNIT_BYTES + lane * 16);
  };
  // vmcnt(n) lgkmcnt(0)
  constexpr auto wait_code = [](int vm) { return (vm & 15) | 0x70 | (vm >> 4) << 14; };

  // One k unit from register set `set`; `nxt` holds the next one, `cur` (read by everybody at the barrier) takes unit `u` of the next round.
  auto step = [&](auto set_c, uint8_t* cur, const uint8_t* nxt, int u) CANZ_INLINE {
    constexpr int set = decltype(set_c)::value;
    __builtin_amdgcn_s_waitcnt(wait_code(2 * S::loads));
    __builtin_amdgcn_s_barrier();
    CANZ_FENCE();
    static_for<W * W>([&](auto x) CANZ_INLINE {
      constexpr int idx = decltype(x)::value, i = idx / W, j = idx % W;
      acc[i][j] = mfma<j % 4, i % 4>(fb[set][j], fa[set][i], acc[i][j], sb[set][j / 4], sa[set][i / 4]);
      constexpr int PACE = W * W / READS;   // MFMAs per read
      if constexpr (idx % PACE == 0 && idx / PACE < READS) {
        CANZ_FENCE();
        read_one(nxt, set ^ 1, std::integral_constant<int, idx / PACE>{});
        CANZ_FENCE();
      }
      constexpr int LPACE = W * W / S::loads;
      if constexpr (idx % LPACE == LPACE / 2 && idx / LPACE < S::loads) {
        CANZ_FENCE();
        fetch_one(cur, u, std::integral_constant<int, idx / LPACE>{});
        CANZ_FENCE();
      }
    });
  };

  auto store_tile = [&](const Tile& t, auto type, auto reads) CANZ_INLINE {
    using E = std::remove_pointer_t<decltype(type)>;
    constexpr bool BETA = decltype(reads)::value;
    int lane = threadIdx.x & 63;   // opaque, or every address that depends on it is kept across the tiles
    asm volatile("" : "+v"(lane));
    const int64_t rows = ps->pr[t.problem].m, ldc = ps->pr[t.problem].ldc;
    const int64_t row0 = (t.m0 + wm * W) * MX_UNIT_ROWS, col0 = (t.n0 + wn * W) * MX_UNIT_ROWS + (lane >> 4) * 8;
    const int64_t left = ps->pr[t.problem].n - col0;   // columns from this lane's first one on
    const float alpha = ps->pr[t.problem].alpha, beta = ps->pr[t.problem].beta;
    E* const c = static_cast<E*>(ps->pr[t.problem].c);
    // Pieces of 16 bytes leave in pairs (the two halves of eight fp32 results, or two neighbouring pairs of units in bf16), which lanes 8 apart
    // exchange, so that a store instruction has 8 rows of 128 bytes instead of 16 of 64 or of every other 16.
    constexpr int APART = sizeof(E) == 4 ? 4 : 32;   // columns from one of a pair to the other
    constexpr int PAIRS = sizeof(E) == 4 ? W / 2 : W / 4, STEP = sizeof(E) == 4 ? 32 : 64;
    const int slot = lane & 15, out_col = slot < 8 ? 0 : APART;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      float v[W / 2][8];   // this lane's row, eight columns of every pair of units
#pragma unroll
      for (int e = 0; e < W * 4; ++e) v[e >> 3][e & 7] = alpha * acc[i][e >> 2][e & 3];
      if constexpr (BETA) {
        const int64_t row = row0 + mx_row(i, slot);
        f32x8 old[W / 2];
        if (row < rows) {
#pragma unroll
          for (int jp = 0; jp < W / 2; ++jp) old[jp] = load_old(c + row * ldc + col0 + jp * 32, left - jp * 32);
#pragma unroll
          for (int e = 0; e < W * 4; ++e) v[e >> 3][e & 7] = __builtin_fmaf(beta, old[e >> 3][e & 7], v[e >> 3][e & 7]);
        }
      }
      i32x4 low[PAIRS], high[PAIRS];   // rows of slots 0 .. 7 and 8 .. 15
#pragma unroll
      for (int q = 0; q < PAIRS; ++q) {
        i32x4 x, y;
        if constexpr (sizeof(E) == 4) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(int, v[q][e]), y[e] = __builtin_bit_cast(int, v[q][4 + e]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = __builtin_bit_cast(int, mx_bf16x2{static_cast<__bf16>(v[2 * q][2 * e]), static_cast<__bf16>(v[2 * q][2 * e + 1])});
            y[e] = __builtin_bit_cast(int, mx_bf16x2{static_cast<__bf16>(v[2 * q + 1][2 * e]), static_cast<__bf16>(v[2 * q + 1][2 * e + 1])});
          }
        }
        constexpr int ROTATE_8 = 0x128;   // within 16 lanes; the bank masks are their last and first eight
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          low[q][e] = __builtin_amdgcn_update_dpp(x[e], y[e], ROTATE_8, 0xF, 0xC, false);
          high[q][e] = __builtin_amdgcn_update_dpp(y[e], x[e], ROTATE_8, 0xF, 0x3, false);
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int64_t row = row0 + mx_row(i, half * 8 + (slot & 7));
        if (row < rows) {
          E* const at = c + row * ldc + col0 + out_col;
#pragma unroll
          for (int q = 0; q < PAIRS; ++q) store_piece(at + q * STEP, left - out_col - q * STEP, half == 0 ? low[q] : high[q]);
        }
      }
      CANZ_FENCE();
    }
  };
  using Set0 = std::integral_constant<int, 0>;
  using Set1 = std::integral_constant<int, 1>;
  next_round();
  if (next_tile.problem < 0) return;   // this XCD's share is one tile less than others'
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st0, load_u, idx); });
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st1, load_u + 1, idx); });
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st2, load_u + 2, idx); });
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st3, load_u + 3, idx); });
  __builtin_amdgcn_s_waitcnt(wait_code(3 * S::loads));
  __builtin_amdgcn_s_barrier();
  CANZ_FENCE();
  static_for<READS>([&](auto idx) CANZ_INLINE { read_one(st0, 0, idx); });

  for (;;) {
    const Tile t = next_tile;
    if (t.problem < 0) break;
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int rounds = (ps->pr[t.problem].units + 3) / 4; rounds > 0; --rounds) {
      next_round();
      step(Set0{}, st0, st1, load_u);
      step(Set1{}, st1, st2, load_u + 1);
      step(Set0{}, st2, st3, load_u + 2);
      step(Set1{}, st3, st0, load_u + 3);
    }
    if constexpr (!std::is_void_v<ONLY>) {
      store_tile(t, static_cast<ONLY*>(nullptr), std::bool_constant<ONLY_BETA>{});
    } else {
      const bool reads = ps->pr[t.problem].beta != 0.f;
      auto as = [&](auto type) CANZ_INLINE {
        if (reads)
          store_tile(t, type, std::true_type{});
        else
          store_tile(t, type, std::false_type{});
      };
      if (ps->pr[t.problem].out_dtype == CANZ_DT_F32)
        as(static_cast<float*>(nullptr));
      else
        as(static_cast<__bf16*>(nullptr));
    }
  }
  __builtin_amdgcn_s_waitcnt(wait_code(0));   // the requests behind the last tile have landed before the block leaves
}

// sets first_tile of every problem for tiles of rows x cols; the number of tiles
int64_t count_tiles(MxProblems& ps, int rows, int cols) {
  int64_t tiles = 0;
  for (int i = 0; i < ps.n; ++i) {
    ps.first_tile[i] = static_cast<int>(tiles);
    tiles += (ps.pr[i].m + rows - 1) / rows * ((ps.pr[i].n + cols - 1) / cols);
  }
  ps.first_tile[ps.n] = static_cast<int>(tiles);
  return tiles;
}

// blocks for these tiles, `most` (a multiple of 8) at a time: as many on each XCD as the one with most tiles has
dim3 tile_grid(const MxProblems& ps, int most) {
  int64_t longest = 0;   // an XCD has at most an eighth of each product, rounded up
  for (int i = 0; i < ps.n; ++i) longest += (ps.first_tile[i + 1] - ps.first_tile[i] + N_XCD - 1) / N_XCD;
  return dim3(static_cast<unsigned>(std::min<int64_t>(N_XCD * longest, most)));
}

template <typename E, bool BETA>
void launch_large_tiles(const MxProblems& all, hipStream_t st) {
  MxProblems ps;
  ps.n = 0;
  for (int i = 0; i < all.n; ++i)
    if ((all.pr[i].out_dtype == CANZ_DT_F32) == (sizeof(E) == 4) && (all.pr[i].beta != 0.f) == BETA) ps.pr[ps.n++] = all.pr[i];
  if (ps.n == 0) return;
  count_tiles(ps, 256, 256);
  k_mx_product<8, E, BETA><<<tile_grid(ps, N_CU), THREADS, 0, st>>>(ps);
}

// All products in one launch of small tiles, or in one of large tiles for each type of result (a large tile's epilogue is too much code
// to have it in a kernel four times).
hipError_t launch_tiles(MxProblems& ps, hipStream_t st) {
  std::sort(ps.pr, ps.pr + ps.n, [](const MxProblem& x, const MxProblem& y) { return x.units > y.units; });   // the longest begin
  const int64_t large = count_tiles(ps, 256, 256), small = count_tiles(ps, 128, 128);
  int64_t units = 0;   // of all small tiles along k
  for (int i = 0; i < ps.n; ++i) units += static_cast<int64_t>(ps.first_tile[i + 1] - ps.first_tile[i]) * ps.pr[i].units;
  const int64_t ks = (units + small - 1) / small;
  if (mx_large_tiles(large, small, ks)) {
    launch_large_tiles<float, false>(ps, st);
    launch_large_tiles<__bf16, false>(ps, st);
    launch_large_tiles<float, true>(ps, st);
    launch_large_tiles<__bf16, true>(ps, st);
  } else {
    k_mx_product<4, void, false><<<tile_grid(ps, 2 * N_CU), THREADS, 0, st>>>(ps);
  }
  return hipGetLastError();
}

template <typename A, int UM, int UN, int WAVES, int AHEAD>
hipError_t launch_few_as(MxProblems& ps, hipStream_t st) {
  const int64_t blocks = count_tiles(ps, FEW_ROWS, UN * MX_UNIT_ROWS);
  k_mx_product_few<A, UM, UN, WAVES, AHEAD><<<dim3(static_cast<unsigned>(blocks)), 64 * WAVES, 0, st>>>(ps);
  return hipGetLastError();
}

template <typename A, int UM, int AHEAD>
hipError_t launch_few(MxProblems& ps, Width width, hipStream_t st) {
  constexpr int MID = UM == 1 ? 4 : 8, SHORT = UM < 4 ? 16 : 8;   // wavefronts
  constexpr int LESS = AHEAD < 2 ? AHEAD : 2;                     // 16 wavefronts have little of k each
  switch (width) {
    case NARROW: return launch_few_as<A, UM, 2, SHORT, LESS>(ps, st);
    case MIDDLE: return launch_few_as<A, UM, 2, MID, AHEAD>(ps, st);
    default: return launch_few_as<A, UM, 4, 4, AHEAD>(ps, st);
  }
}

// The launches that a product may be part of.
enum Kind { SCALE, TILES, IMAGE_16, IMAGE_32 = IMAGE_16 + WIDTHS, IMAGE_64 = IMAGE_32 + WIDTHS, ROUND_BF16 = IMAGE_64 + WIDTHS,
            ROUND_F32 = ROUND_BF16 + WIDTHS, KINDS = ROUND_F32 + WIDTHS };
int kind_of(const MxProblem& p) {
  if (p.k == 0) return SCALE;
  const Width w = width_of(p.n);
  if (p.a_dtype != CANZ_DT_MX) return (p.a_dtype == CANZ_DT_BF16 ? ROUND_BF16 : ROUND_F32) + w;
  if (p.m <= FEW_ROWS) return (p.m <= 16 ? IMAGE_16 : p.m <= 32 ? IMAGE_32 : IMAGE_64) + w;
  return TILES;
}

hipError_t launch_kind(int kind, MxProblems& ps, hipStream_t st) {
  hipError_t err = hipSuccess;
  switch (kind) {
    case SCALE:
      for (int i = 0; i < ps.n && err == hipSuccess; ++i) {
        k_mx_scale<<<dim3(4 * N_CU), THREADS, 0, st>>>(ps.pr[i]);
        err = hipGetLastError();
      }
      return err;
    case TILES: return launch_tiles(ps, st);
    default: break;
  }
  const Width w = static_cast<Width>((kind - IMAGE_16) % WIDTHS);
  switch (kind - w) {
    case IMAGE_16: return launch_few<uint8_t, 1, 4>(ps, w, st);
    case IMAGE_32: return launch_few<uint8_t, 2, 3>(ps, w, st);
    case IMAGE_64: return launch_few<uint8_t, 4, 2>(ps, w, st);
    case ROUND_BF16: return launch_few<__bf16, 1, 4>(ps, w, st);
    default: return launch_few<float, 1, 2>(ps, w, st);
  }
}

}  // namespace

hipError_t launch_mx_join(const MxProblem& p, const float* sums, int parts, hipStream_t st) {
  k_mx_join<<<dim3(static_cast<unsigned>(std::min<int64_t>((p.m * p.n + THREADS - 1) / THREADS, 16 * N_CU))), THREADS, 0, st>>>(p, sums, parts);
  return hipGetLastError();
}

hipError_t launch_mx_product(const MxProblems& ps, hipStream_t st) {
  int kind[MX_MAX_PROBLEMS];
  for (int i = 0; i < ps.n; ++i) kind[i] = kind_of(ps.pr[i]);
  for (int i = 0; i < ps.n; ++i) {
    if (kind[i] < 0) continue;
    MxProblems part;
    part.n = 0;
    const int now = kind[i];
    for (int q = i; q < ps.n; ++q)
      if (kind[q] == now) part.pr[part.n++] = ps.pr[q], kind[q] = -1;
    if (const hipError_t err = launch_kind(now, part, st); err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace canz
