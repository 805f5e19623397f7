// Products of microscaled 4-bit images: C[i][j] = alpha sum_k A[i][k] B[j][k] + beta C[i][j], fp32 sums.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows of either image over 128 k, scales included; a product of two elements is exact
// in fp32.
#include "device_util.h"
#include "mx.h"

namespace canz {
namespace {

constexpr int THREADS = 256;
constexpr int BM = 64, BN = 64;   // tile of a block; a wavefront owns 32 x 32 of it

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// an operand of four registers (the instruction's other formats take up to eight)
__device__ __forceinline__ i32x8 operand(i32x4 v) { return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }
constexpr int FP4 = 4;   // operand format E2M1

__device__ __forceinline__ void store_c(const MxProblem& p, int64_t row, int64_t col, float v) {
  const int64_t at = row * p.ldc + col;
  v *= p.alpha;
  if (p.out_dtype == CANZ_DT_F32) {
    float* c = static_cast<float*>(p.c) + at;
    *c = p.beta != 0.f ? __builtin_fmaf(p.beta, *c, v) : v;
  } else {
    __bf16* c = static_cast<__bf16*>(p.c) + at;
    *c = static_cast<__bf16>(p.beta != 0.f ? __builtin_fmaf(p.beta, static_cast<float>(*c), v) : v);
  }
}

__global__ __launch_bounds__(THREADS) void k_mx_product(MxProblems ps) {
  int j = 0;
  while (j + 1 < ps.n && static_cast<int>(blockIdx.x) >= ps.pr[j + 1].first_tile) ++j;
  const MxProblem p = ps.pr[j];
  const int tile = blockIdx.x - p.first_tile, tiles_m = static_cast<int>((p.m + BM - 1) / BM);
  const int64_t m0 = static_cast<int64_t>(tile % tiles_m) * BM, n0 = static_cast<int64_t>(tile / tiles_m) * BN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row_w = m0 + (wave >> 1) * 32, col_w = n0 + (wave & 1) * 32;
  const int64_t ks = mx_k_units(p.k);
  // images are padded to 64 rows, so that every unit of the tile exists
  const uint8_t* const a = p.a + row_w / MX_UNIT_ROWS * ks * MX_UNIT_BYTES + lane * 16;
  const uint8_t* const b = p.b + col_w / MX_UNIT_ROWS * ks * MX_UNIT_BYTES + lane * 16;
  const uint8_t* const sa = p.a + mx_code_bytes(p.m, p.k) + m0 / MX_PAD_ROWS * ks * MX_SCALE_BYTES + lane * 4;
  const uint8_t* const sb = p.b + mx_code_bytes(p.n, p.k) + n0 / MX_PAD_ROWS * ks * MX_SCALE_BYTES + lane * 4;
  f32x4 acc[2][2] = {};
  for (int64_t u = 0; u < ks; ++u) {
    i32x8 fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = operand(*reinterpret_cast<const i32x4*>(a + (i * ks + u) * MX_UNIT_BYTES));
      fb[i] = operand(*reinterpret_cast<const i32x4*>(b + (i * ks + u) * MX_UNIT_BYTES));
    }
    // the wavefront's two row tiles are bytes 0 and 1 or 2 and 3 of the scale registers
    const int va = *reinterpret_cast<const int*>(sa + u * MX_SCALE_BYTES) >> (wave >> 1) * 16;
    const int vb = *reinterpret_cast<const int*>(sb + u * MX_SCALE_BYTES) >> (wave & 1) * 16;
    acc[0][0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[0], fb[0], acc[0][0], FP4, FP4, 0, va, 0, vb);
    acc[0][1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[0], fb[1], acc[0][1], FP4, FP4, 0, va, 1, vb);
    acc[1][0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[1], fb[0], acc[1][0], FP4, FP4, 1, va, 0, vb);
    acc[1][1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[1], fb[1], acc[1][1], FP4, FP4, 1, va, 1, vb);
  }
  // register r of lane l: row 4 (l / 16) + r, column l % 16
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int jn = 0; jn < 2; ++jn)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t row = row_w + i * 16 + 4 * (lane >> 4) + r, col = col_w + jn * 16 + (lane & 15);
        if (row < p.m && col < p.n) store_c(p, row, col, acc[i][jn][r]);
      }
}

}  // namespace

hipError_t launch_mx_product(MxProblems& ps, hipStream_t st) {
  int64_t tiles = 0;
  for (int i = 0; i < ps.n; ++i) {
    ps.pr[i].first_tile = static_cast<int>(tiles);
    tiles += (ps.pr[i].m + BM - 1) / BM * ((ps.pr[i].n + BN - 1) / BN);
  }
  if (tiles > 0) k_mx_product<<<dim3(static_cast<unsigned>(tiles)), THREADS, 0, st>>>(ps);
  return hipGetLastError();
}

}  // namespace canz
