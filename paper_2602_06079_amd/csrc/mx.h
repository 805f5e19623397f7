// Launchers behind the canz_mx_* entry points (internal, not part of the ABI).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "canz.h"
#include "mx_layout.h"
#include "mx_rules.h"

namespace canz {

// The stream that a caller named.  The legacy default stream is the null stream by another name, and the runtime is only given that one: a call with the
// handle of the former ended the process inside it.
inline hipStream_t stream_of(void* named) { return named == hipStreamLegacy ? nullptr : static_cast<hipStream_t>(named); }

// Kernels are launched on the device the caller's stream belongs to, whatever the thread's current device is.
class StreamDevice {
 public:
  explicit StreamDevice(hipStream_t st) {
    hipDevice_t dev = 0;
    if (st == nullptr || st == hipStreamPerThread) return;   // these are the current device's
    if ((err_ = hipStreamGetDevice(st, &dev)) != hipSuccess || (err_ = hipGetDevice(&before_)) != hipSuccess) return;
    if (dev != before_) restore_ = (err_ = hipSetDevice(dev)) == hipSuccess;
  }
  ~StreamDevice() {
    if (restore_) (void)hipSetDevice(before_);
  }
  StreamDevice(const StreamDevice&) = delete;
  StreamDevice& operator=(const StreamDevice&) = delete;
  hipError_t error() const { return err_; }

 private:
  int before_ = 0;
  bool restore_ = false;
  hipError_t err_ = hipSuccess;
};

// Matrices of one type, width and row distance in one launch.
constexpr int MX_MAX_MATS = 32;
struct MxMats {
  int64_t cols, ld;
  int64_t most_rows;   // of all of them
  int n, dtype, scale_mode;
  int rows[MX_MAX_MATS];
  void* mat[MX_MAX_MATS];
  uint8_t* by_row[MX_MAX_MATS];       // all null or none
  uint8_t* by_col[MX_MAX_MATS];
  const uint8_t* noise[MX_MAX_MATS];
};
hipError_t launch_mx_quantize(const MxMats& m, hipStream_t st);
hipError_t launch_mx_dequantize(const MxMats& m, hipStream_t st);

// C = alpha A B^T + beta C of images A (m x k) and B (n x k), several products in one launch.  A may also be a matrix, which the kernel rounds on
// its way (mx_rounds_on_the_way).
struct MxProblem {
  const uint8_t* a;   // image, or the matrix's first element
  const uint8_t* b;
  void* c;
  int64_t m, n, k, lda, ldc;
  float alpha, beta;
  int a_dtype, a_ceil, out_dtype;
  int first_unit, units;   // the part of k that is multiplied (images of more than 64 rows), in units of 128
};
constexpr int MX_MAX_PROBLEMS = 32;

struct MxProblems {
  int n;
  int first_tile[MX_MAX_PROBLEMS + 1];   // of every problem, then their number: set by the launcher, side by side, since every block goes through them
  MxProblem pr[MX_MAX_PROBLEMS];
};
hipError_t launch_mx_product(const MxProblems& p, hipStream_t st);

// C = alpha (sum of `parts` matrices of m x n fp32 sums, one behind the other) + beta C
hipError_t launch_mx_join(const MxProblem& p, const float* sums, int parts, hipStream_t st);

// Validates one group of canz_mx_quantize (`back`: of canz_mx_dequantize).
int check_mx_group(const canz_mx_group& g, int idx, bool back);
// The images of a checked group, in launches of MX_MAX_MATS matrices.
int quantize_group(const canz_mx_group& g, int scale_mode, hipStream_t st);

}  // namespace canz
