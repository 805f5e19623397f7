// Launchers behind canz_linear (internal, not part of the ABI).
#pragma once
#include <type_traits>

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
// up to LINEAR_FEW rows, both operands contiguous along k, at any address; the same kind of A and the same linear_few_width in all of them
hipError_t launch_linear_few(LinearProblems& ps, hipStream_t st);
// C from the sum of `parts` matrices of m x pitch fp32 sums, one behind the other (none: from zeros).
struct LinearJoin {
  LinearEnd end;
  int64_t m, n, pitch;
  const float* sums;
  int parts, log_tx, across;
};
constexpr int LINEAR_JOINS = 16;
struct LinearJoins {
  int n;
  unsigned first_block[LINEAR_JOINS + 1];
  LinearJoin jn[LINEAR_JOINS];
};
hipError_t launch_linear_joins(LinearJoins& js, hipStream_t st);

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
template <typename E>   // a LinearEnd among a kernel's arguments
__device__ __forceinline__ LinearEnd linear_end_of(const E& e) {
  return LinearEnd{e.c, e.r, e.bias, Image8{e.pre.codes, e.pre.scales, e.pre.pitch}, e.ldc, e.ldr, e.alpha, e.beta, e.act, e.out_f32, e.bias_f32};
}

// z = alpha sum + bias;  C = act(z) + beta R, for eight columns (from `col` on, a multiple of 8) of the rows row, row + step, ... , R of them, m and n rows and columns of C.  The lane's quad
// holds the 32 columns of a block and is active as a whole; what is not there is not read or written (WHOLE: all of it is).  Rows go through every part together, so that their loads are in
// flight at once and a part's branch is taken once.
template <bool WHOLE, int R>
__device__ __forceinline__ void linear_end(const LinearEnd& e, int64_t row, int step, int64_t col, int64_t m, int64_t n, f32x8 (&z)[R]) {
  const int64_t there = WHOLE ? PIECE : n - col;
  auto left = [&](int r) { return WHOLE || row + r * step < m ? there : int64_t{0}; };
  if (e.bias) {
    const f32x8 b = e.bias_f32 ? widen(load_raw(static_cast<const float*>(e.bias) + col, there)) : widen(load_raw(static_cast<const __bf16*>(e.bias) + col, there));
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < PIECE; ++i) z[r][i] = __builtin_fmaf(e.alpha, z[r][i], b[i]);
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < PIECE; ++i) z[r][i] *= e.alpha;
  }
  if (e.pre.codes) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      f32x8 kept = z[r];
      if constexpr (!WHOLE) {
#pragma unroll
        for (int i = 0; i < PIECE; ++i) kept[i] = i < there ? kept[i] : 0.f;
      }
      const Codes8 c = round8(kept);
      if (WHOLE || (row + r * step < m && col < e.pre.pitch)) store_codes(e.pre, row + r * step, col, n, c);
    }
  }
  auto apply = [&](auto kind) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < PIECE; ++i) z[r][i] = act_both<decltype(kind)::value, false>(z[r][i]).value;
  };
  if (e.act == CANZ_ACT_SILU)
    apply(std::integral_constant<int, CANZ_ACT_SILU>{});
  else if (e.act == CANZ_ACT_GELU)
    apply(std::integral_constant<int, CANZ_ACT_GELU>{});
  else if (e.act == CANZ_ACT_RELU)
    apply(std::integral_constant<int, CANZ_ACT_RELU>{});
  auto out = [&](auto* c, const auto* old) {
    using E = std::remove_pointer_t<decltype(c)>;
    if (e.beta != 0.f) {
      Raw<E> x[R];
#pragma unroll
      for (int r = 0; r < R; ++r) x[r] = load_raw(old + (row + r * step) * e.ldr + col, left(r));
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const f32x8 v = widen(x[r]);
#pragma unroll
        for (int i = 0; i < PIECE; ++i) z[r][i] = __builtin_fmaf(e.beta, v[i], z[r][i]);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (WHOLE || left(r) > 0) store_piece8(c + (row + r * step) * e.ldc + col, left(r), z[r]);
  };
  if (e.out_f32)
    out(static_cast<float*>(e.c), static_cast<const float*>(e.r));
  else
    out(static_cast<__bf16*>(e.c), static_cast<const __bf16*>(e.r));
}
#endif

}  // namespace canz
