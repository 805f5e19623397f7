// Products of up to 64 rows of A (canz_linear): B goes by once.
//
// A block has 16 UN rows of B and all of k, which its wavefronts share in units of 128 k by turns, so that together they read long pieces of B's rows; A's rows (16 UM of them, bf16, or an
// 8-bit image whose elements the lane that needs them turns into bf16) come out of L2.  Memory is all that takes time: each wavefront keeps AHEAD units in flight.
//
// v_mfma_f32_16x16x32_bf16 with B first: lane l supplies 8 k (from 8 (l / 16) on) of row l % 16 of either, and holds columns 4 (l / 16) .. + 3 of row l % 16 of C.
#include <algorithm>
#include <type_traits>

#include "linear.h"

namespace canz {
namespace {

#define CANZ_INLINE __attribute__((always_inline))
#define CANZ_FENCE() __builtin_amdgcn_sched_barrier(0)

constexpr int UNIT = 128, PARTS = UNIT / 32;   // k of a unit, instructions for it
constexpr int WAVES = 4;                       // of a block

// Eight k of a row of A on their way from memory.
template <bool IMAGE>
struct RawA {
  bf16x8_any v;
};
template <>
struct RawA<true> {
  u32x2 codes;
};
__device__ __forceinline__ bf16x8 operand(const RawA<false>& r, unsigned) { return __builtin_bit_cast(bf16x8, r.v); }
__device__ __forceinline__ bf16x8 operand(const RawA<true>& r, unsigned scale) {
  const f32x8 v = values8(r.codes, scale);
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = static_cast<__bf16>(v[e]);   // exact but for blocks below 2^-124, which images made elsewhere may have
  return o;
}

template <bool IMAGE, int UM, int UN, int AHEAD>
__global__ __launch_bounds__(64 * WAVES) void k_linear_few(LinearProblems) {
  const LinearArgs ps = (LinearArgs)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ f32x4 sums[WAVES][UM * UN][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slot = blockIdx.x;
  int j = 0;
  while (slot >= ps->first_tile[j + 1]) ++j;
  const int64_t m = ps->pr[j].m, n = ps->pr[j].n, k = ps->pr[j].k, lda = ps->pr[j].lda, ldb = ps->pr[j].ldb;
  const int64_t col0 = static_cast<int64_t>(slot - ps->first_tile[j]) * (16 * UN);
  const int l = lane & 15, at = (lane >> 4) * 8;
  // this lane's rows, from its k of a unit on; a row that is not there is read as the last
  const __bf16* b[UN];
#pragma unroll
  for (int q = 0; q < UN; ++q) b[q] = static_cast<const __bf16*>(ps->pr[j].b) + min(col0 + q * 16 + l, n - 1) * ldb + at;
  const uint8_t *a[UM], *scales[UM];
#pragma unroll
  for (int i = 0; i < UM; ++i) {
    const int64_t row = min(static_cast<int64_t>(i * 16 + l), m - 1);
    a[i] = static_cast<const uint8_t*>(ps->pr[j].a) + (row * lda + at) * (IMAGE ? 1 : 2);
    scales[i] = IMAGE ? ps->pr[j].a_scales + row * (lda / MX8_BLOCK) : nullptr;
  }
  f32x4 acc[UM][UN] = {};
  bf16x8_any rb[AHEAD][UN][PARTS];
  RawA<IMAGE> ra[AHEAD][UM][PARTS];
  unsigned rs[AHEAD][UM];   // the four scale bytes of a unit
  auto load = [&](int d, int64_t u) CANZ_INLINE {
#pragma unroll
    for (int q = 0; q < UN; ++q)
#pragma unroll
      for (int p = 0; p < PARTS; ++p) rb[d][q][p] = *reinterpret_cast<const bf16x8_any*>(b[q] + u * UNIT + p * 32);
#pragma unroll
    for (int i = 0; i < UM; ++i) {
#pragma unroll
      for (int p = 0; p < PARTS; ++p) ra[d][i][p] = *reinterpret_cast<const RawA<IMAGE>*>(a[i] + (u * UNIT + p * 32) * (IMAGE ? 1 : 2));
      rs[d][i] = IMAGE ? *reinterpret_cast<const unsigned*>(scales[i] + u * PARTS) : 0u;
    }
  };
  // `there`: a unit that is not there was read as another one and counts nothing
  auto multiply = [&](int d, bool there) CANZ_INLINE {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      bf16x8 y[UN];
#pragma unroll
      for (int q = 0; q < UN; ++q) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        i32x4 v = __builtin_bit_cast(i32x4, rb[d][q][p]);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = there ? v[e] : 0;
        y[q] = __builtin_bit_cast(bf16x8, v);
      }
#pragma unroll
      for (int i = 0; i < UM; ++i) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        i32x4 x = __builtin_bit_cast(i32x4, operand(ra[d][i][p], rs[d][i] >> (8 * p) & 255u));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = there ? x[e] : 0;   // a NaN there would count, too
#pragma unroll
        for (int q = 0; q < UN; ++q) acc[i][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[q], __builtin_bit_cast(bf16x8, x), acc[i][q], 0, 0, 0);
      }
    }
  };
  const int whole = static_cast<int>(k / UNIT);
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
  if (whole * UNIT < k && wave == whole % WAVES) {   // the last unit, of which only a part is there
    const int64_t left = k - static_cast<int64_t>(whole) * UNIT - at;   // of this lane's row, from its first k on
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
#pragma unroll
      for (int q = 0; q < UN; ++q) rb[0][q][p] = load_raw(b[q] + static_cast<int64_t>(whole) * UNIT + p * 32, left - p * 32).v;
#pragma unroll
      for (int i = 0; i < UM; ++i) {
        if constexpr (IMAGE)   // an image's rows are padded with zeros to whole units
          ra[0][i][p] = *reinterpret_cast<const RawA<IMAGE>*>(a[i] + static_cast<int64_t>(whole) * UNIT + p * 32);
        else
          ra[0][i][p].v = load_raw(reinterpret_cast<const __bf16*>(a[i]) + static_cast<int64_t>(whole) * UNIT + p * 32, left - p * 32).v;
      }
    }
#pragma unroll
    for (int i = 0; i < UM; ++i) rs[0][i] = IMAGE ? *reinterpret_cast<const unsigned*>(scales[i] + static_cast<int64_t>(whole) * PARTS) : 0u;
    multiply(0, true);
  }
#pragma unroll
  for (int i = 0; i < UM; ++i)
#pragma unroll
    for (int q = 0; q < UN; ++q) sums[wave][i * UN + q][lane] = acc[i][q];
  __syncthreads();
  // eight columns of a row per thread: columns 8 c .. of the block's 16 UN lie in tile c / 2, lanes from 32 (c % 2) on
  const LinearEnd e = linear_end_of(ps->pr[j].end);
  constexpr int COLS = 2 * UN;
  for (int x = threadIdx.x; x < 16 * UM * COLS; x += 64 * WAVES) {
    const int c = x % COLS, row = x / COLS, tile = row / 16 * UN + c / 2, from = (c & 1) * 32 + (row & 15);
    f32x4 lo = sums[0][tile][from], hi = sums[0][tile][from + 16];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) lo += sums[w][tile][from], hi += sums[w][tile][from + 16];
    f32x8 z[1] = {f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}};
    linear_end<false, 1>(e, row, 0, col0 + c * 8, m, n, z);
  }
}

template <bool IMAGE, int UM, int UN, int AHEAD>
void launch(LinearProblems& ps, hipStream_t st) {
  int64_t blocks = 0;
  for (int i = 0; i < ps.n; ++i) {
    ps.first_tile[i] = static_cast<int>(blocks);
    const int64_t cols = ps.pr[i].end.pre.codes ? ps.pr[i].end.pre.pitch : ps.pr[i].n;   // an image's padding is written, too
    blocks += (cols + 16 * UN - 1) / (16 * UN);
  }
  ps.first_tile[ps.n] = static_cast<int>(blocks);
  k_linear_few<IMAGE, UM, UN, AHEAD><<<dim3(static_cast<unsigned>(blocks)), 64 * WAVES, 0, st>>>(ps);
}

// The wavefronts alone decide the order of a sum, so products of different numbers of rows may share a launch.  us, 64 rows of B to a block / 32 / 32 and eight wavefronts: 1 x 25600 x 5120
// 52 / 53 / 56 (262 MB, 5.0 TB/s), 17 x 25600 x 5120 60 / 69 / 78, 16 x 12288 x 4096 24 / 32 / 30, 64 x 12288 x 4096 35 / 49 / 50; 1 x 5120 x 25600 97 / 56 / 57, 8 x 4096 x 4096 20 / 14 / 13,
// 37 x 1536 x 4096 28 / 21 / 20, 1 x 1024 x 1024 7.3 / 5.1 / 7.7.  32 / 16: 1 x 1536 x 4096 10.9 / 7.5, 37 x 1536 x 4096 21.6 / 15.9, 8 x 4096 x 4096 13.1 / 9.4, 64 x 512 x 8192 44.6 / 37.4,
// 1 x 5120 x 25600 56.5 / 65.9, 64 x 8192 x 4096 28.0 / 38.8.
template <bool IMAGE>
void launch(LinearProblems& ps, hipStream_t st) {
  int64_t m = 0;
  for (int i = 0; i < ps.n; ++i) m = std::max(m, ps.pr[i].m);
  auto with = [&](auto un, auto ahead) {
    constexpr int UN = un(), AHEAD = ahead();
    if (m <= 16)
      launch<IMAGE, 1, UN, 2 * AHEAD>(ps, st);
    else if (m <= 32)
      launch<IMAGE, 2, UN, 2>(ps, st);
    else
      launch<IMAGE, 4, UN, AHEAD>(ps, st);
  };
  using std::integral_constant;
  switch (linear_few_width(ps.pr[0].n, ps.pr[0].end.pre.codes != nullptr)) {
    case 0: return with(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    case 1: return with(integral_constant<int, 2>{}, integral_constant<int, 1>{});
    default: return with(integral_constant<int, 4>{}, integral_constant<int, 1>{});
  }
}

}  // namespace

hipError_t launch_linear_few(LinearProblems& ps, hipStream_t st) {
  if (ps.pr[0].a_scales)
    launch<true>(ps, st);
  else
    launch<false>(ps, st);
  return hipGetLastError();
}

}  // namespace canz
