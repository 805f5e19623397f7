// Launchers behind canz_linear (internal, not part of the ABI).
#pragma once
#include "act.h"
#include "linear_rules.h"
#include "mx8.h"

namespace canz {

// What is done to eight consecutive sums of a row of A B^T.
struct LinearEnd {
  void* c;
  const void* r;       // the residual, C itself or, where beta is 0, not looked at
  const void* bias;    // or null
  Image8 pre;          // codes null: not asked for
  int64_t ldc, ldr;
  float alpha, beta;
  int act, out_f32, bias_f32;
};

// One product as the kernels see it: bf16 operands.  The tile kernels want each of them 16-byte aligned, rows a multiple of 8 elements apart and at most 2^22, the extent that is
// contiguous in memory a multiple of 8 (`k_a`, `k_b`: k as each operand has it, zeros beyond k).
struct LinearProblem {
  const void *a, *b;
  int64_t lda, ldb;
  int64_t m, n, k;
  int k_a, k_b;
  int first_step, steps;   // the part of k that is multiplied, in steps of 32
  const uint8_t* a_scales; // few rows: A is an image; its codes are a
  LinearEnd end;
};

constexpr int LINEAR_PROBLEMS = 16;
struct LinearProblems {
  int n;
  int first_tile[LINEAR_PROBLEMS + 1];   // of every problem, then their number
  int from, to;                          // tiles: which of an XCD's tiles the launch has
  int quarters;                          // tiles of 128 x 128: the launch's tiles are those of 256 x 256, in quarters
  LinearProblem pr[LINEAR_PROBLEMS];
};

// tiles: all problems of one launch have the same orientations
hipError_t launch_linear_tiles(LinearProblems& ps, bool a_trans, bool b_trans, hipStream_t st);
// up to LINEAR_FEW rows, both operands contiguous along k, at any address; the same kind of A in all of them
hipError_t launch_linear_few(LinearProblems& ps, hipStream_t st);
// C from the sum of `parts` matrices of m x pitch fp32 sums, one behind the other (none: from zeros)
hipError_t launch_linear_join(const LinearProblem& p, const float* sums, int64_t pitch, int parts, hipStream_t st);

// A matrix as an operand of the tile kernels: bf16, rows `pitch` apart, zeros behind `cols`.
struct LinearCopy {
  const void* from;
  const uint8_t* scales;   // `from` are the codes of an image; null: a bf16 matrix
  __bf16* to;
  int64_t rows, cols, ld, pitch;
};
constexpr int LINEAR_COPIES = 32;
struct LinearCopies {
  int n;
  unsigned first_block[LINEAR_COPIES + 1];
  LinearCopy cp[LINEAR_COPIES];
};
hipError_t launch_linear_copies(LinearCopies& cs, hipStream_t st);

// sums[i] <- alpha (sum over k of A) + beta sums[i]: over the columns of a stored m x k matrix, or over the rows of a k x m one (`trans`).
struct LinearSums {
  const void* from;
  const uint8_t* scales;
  int64_t rows, cols, ld;   // as stored
  int trans;
  float alpha, beta;
  float* partial;           // trans: linear_sum_groups(rows) rows of mx8_pitch(cols) floats
  float* sums;
};
constexpr int64_t linear_sum_groups(int64_t rows) { return rows < 128 ? rows : 128; }
hipError_t launch_linear_sums(const LinearSums& s, hipStream_t st);

#if defined(__HIPCC__)
// A kernel's argument where it lies: scalar loads at any index, and no copy of it.
typedef const __attribute__((address_space(4))) LinearProblems* LinearArgs;
__device__ __forceinline__ LinearEnd linear_end_of(LinearArgs ps, int j) {
  const auto& e = ps->pr[j].end;
  return LinearEnd{e.c, e.r, e.bias, Image8{e.pre.codes, e.pre.scales, e.pre.pitch}, e.ldc, e.ldr, e.alpha, e.beta, e.act, e.out_f32, e.bias_f32};
}

// z = alpha sum + bias;  C = act(z) + beta R.  `col` is a multiple of 8, the lane's quad holds the 32 columns of a block and is active as a whole; what is not `there` (or behind n) is
// not read or written.
__device__ __forceinline__ void linear_end(const LinearEnd& e, int64_t row, int64_t col, int64_t n, bool there, f32x8 sum) {
  const int64_t left = there ? n - col : 0;
  f32x8 z;
  if (e.bias) {
    const f32x8 b = e.bias_f32 ? widen(load_raw(static_cast<const float*>(e.bias) + col, left)) : widen(load_raw(static_cast<const __bf16*>(e.bias) + col, left));
#pragma unroll
    for (int i = 0; i < PIECE; ++i) z[i] = __builtin_fmaf(e.alpha, sum[i], b[i]);
  } else {
#pragma unroll
    for (int i = 0; i < PIECE; ++i) z[i] = e.alpha * sum[i];
  }
  if (e.pre.codes) {
    f32x8 kept = z;
#pragma unroll
    for (int i = 0; i < PIECE; ++i) kept[i] = i < left ? z[i] : 0.f;
    const Codes8 c = round8(kept);
    const Image8 im{e.pre.codes, e.pre.scales, e.pre.pitch};
    if (there && col < im.pitch) store_codes(im, row, col, n, c);
  }
  if (left <= 0) return;
  if (e.act == CANZ_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < PIECE; ++i) z[i] = act_both<CANZ_ACT_SILU>(z[i]).value;
  } else if (e.act == CANZ_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < PIECE; ++i) z[i] = act_both<CANZ_ACT_GELU>(z[i]).value;
  } else if (e.act == CANZ_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < PIECE; ++i) z[i] = act_both<CANZ_ACT_RELU>(z[i]).value;
  }
  auto out = [&](auto* c, const auto* r) {
    if (e.beta != 0.f) {
      const f32x8 old = widen(load_raw(r + row * e.ldr + col, left));
#pragma unroll
      for (int i = 0; i < PIECE; ++i) z[i] = __builtin_fmaf(e.beta, old[i], z[i]);
    }
    store_piece8(c + row * e.ldc + col, left, z);
  };
  if (e.out_f32)
    out(static_cast<float*>(e.c), static_cast<const float*>(e.r));
  else
    out(static_cast<__bf16*>(e.c), static_cast<const __bf16*>(e.r));
}
#endif

}  // namespace canz
