// canz_norm_forward and canz_norm_backward: the root-mean-square norm with the residual's addition, and its gradients.
//
//   h = x + residual,  rstd = 1 / sqrt(mean(h^2) + eps),  y = w n  with  n = h rstd
//   dx = dsum + rstd (u - n mean(u n))  with  u = w dy,       dw = sum over rows of dy n
//
// A row is held in the registers of a wavefront or of a block between its reduction and its results, so that every operand is read once; rows
// longer than that (LONG_*) are read twice.  Memory is what bounds them: 8192 x 4096 in bf16 with a residual takes 47 us forward (268 MB, 5.7 TB/s) and 46 back (268 MB, 5.8 TB/s) and 5 for dweight's
// join; 4097 x 1531 with the stream in fp32 18 us (75 MB, 4.1 TB/s: rows begin anywhere) and 25 from the image of h (69 MB, 2.8 TB/s: four rows to a wavefront, each loaded behind the stores of the one before).
// With y as an image as well 8192 x 4096 takes 59 us (303 MB, 5.1 TB/s); 2048 x 25600 in bf16 100 us forward (419 MB, 4.2 TB/s) and 129 back (419 MB, 3.2 TB/s: dy and h go by three times, the cache behind L2 helps).
#include <algorithm>
#include <type_traits>

#include "canz_internal.h"
#include "mx8.h"

namespace canz {
namespace {

// ---- pieces ---------------------------------------------------------------------------------------------------------------------
// Eight weights from column `col` on, in fp32.
__device__ __forceinline__ f32x8 load_weight(const void* w, int f32, int64_t col, int64_t cols) {
  return f32 ? widen(load_raw(static_cast<const float*>(w) + col, cols - col)) : widen(load_raw(static_cast<const __bf16*>(w) + col, cols - col));
}
// Rounds to a type and back.
template <typename S>
__device__ __forceinline__ f32x8 as_held(f32x8 v) {
#pragma unroll
  for (int e = 0; e < PIECE; ++e) v[e] = static_cast<float>(static_cast<S>(v[e]));
  return v;
}
__device__ __forceinline__ float dot(f32x8 a, f32x8 b, float sum) {
#pragma unroll
  for (int e = 0; e < PIECE; ++e) sum = __builtin_fmaf(a[e], b[e], sum);
  return sum;
}
// Sum over the TX threads that share a row; every one receives it.  Rows alternate between two sets of LDS words (`parity`), so that one barrier a row is enough: a
// wavefront that writes the next but one has passed the barrier that every other one reached after reading this one.
template <int TX>
__device__ __forceinline__ float row_sum(float v, int parity) {
  v = wave_sum(v);
  if constexpr (TX > 64) {
    __shared__ float part[2][TX / 64];
    if ((threadIdx.x & 63) == 0) part[parity][threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < TX / 64; ++i) v += part[parity][i];
  }
  return v;
}
constexpr int block_threads(int tx) { return tx < 256 ? 256 : tx; }

// ---- forward --------------------------------------------------------------------------------------------------------------------
struct Forward {
  const void *x, *residual, *weight;
  void *sum, *y;
  Image8 y8;   // codes null: not asked for
  float* rstd;
  int64_t rows, cols, ldx, lds, ldy;
  float eps, one_of_cols;
  int weight_f32;
};

template <typename E, typename S>
__device__ __forceinline__ f32x8 add(const Raw<E>& x, const Raw<S>& r, bool residual) {
  f32x8 v = widen(x);
  if (residual) v += widen(r);
  return as_held<S>(v);
}
template <typename E>
__device__ __forceinline__ void finish(const Forward& a, int64_t row, int64_t col, f32x8 h, f32x8 w, float rstd) {
  f32x8 y;
#pragma unroll
  for (int e = 0; e < PIECE; ++e) y[e] = h[e] * rstd * w[e];
  if (a.y8.codes) store_codes(a.y8, row, col, a.cols, round8(y));
  if (a.y && col < a.cols) store_piece8(static_cast<E*>(a.y) + row * a.ldy + col, a.cols - col, y);
}

// TX threads hold a row, NV pieces each: up to 8 TX NV columns.  All loads of a row are on their way before the first is used.
template <typename E, typename S, int TX, int NV>
__global__ __launch_bounds__(block_threads(TX)) void k_norm(Forward a) {
  const int tx = threadIdx.x & (TX - 1);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (block_threads(TX) / TX) + threadIdx.x / TX;
  if (row >= a.rows) return;   // whole wavefronts, and no barrier where a block has several rows
  const int64_t pitch = mx8_pitch(a.cols);
  Raw<E> x[NV];
  Raw<S> r[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t col = (static_cast<int64_t>(j) * TX + tx) * PIECE;
    x[j] = load_raw(static_cast<const E*>(a.x) + row * a.ldx + col, a.cols - col);
    if (a.residual) r[j] = load_raw(static_cast<const S*>(a.residual) + row * a.lds + col, a.cols - col);
  }
  f32x8 h[NV];
  float squares = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    h[j] = add(x[j], r[j], a.residual != nullptr);
    squares = dot(h[j], h[j], squares);
  }
  const float rstd = 1.f / __builtin_sqrtf(__builtin_fmaf(row_sum<TX>(squares, 0), a.one_of_cols, a.eps));
  if (a.rstd && tx == 0) a.rstd[row] = rstd;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t col = (static_cast<int64_t>(j) * TX + tx) * PIECE;
    if (col >= pitch) continue;   // whole blocks of 32
    if (a.sum && col < a.cols) store_piece8(static_cast<S*>(a.sum) + row * a.lds + col, a.cols - col, h[j]);
    if (a.y || a.y8.codes) finish<E>(a, row, col, h[j], load_weight(a.weight, a.weight_f32, col, a.cols), rstd);
  }
}

// Long rows are read twice, once for the mean and once for the results; a row is some 100 KB, so that the second reading finds it in L2.
constexpr int LONG_THREADS = 1024;
template <typename E, typename S>
__global__ __launch_bounds__(LONG_THREADS) void k_norm_long(Forward a) {
  const int64_t row = blockIdx.x, pitch = mx8_pitch(a.cols);
  auto load = [&](int64_t col) {
    const Raw<E> x = load_raw(static_cast<const E*>(a.x) + row * a.ldx + col, a.cols - col);
    Raw<S> r{};
    if (a.residual) r = load_raw(static_cast<const S*>(a.residual) + row * a.lds + col, a.cols - col);
    return add(x, r, a.residual != nullptr);
  };
  float squares = 0.f;
  for (int64_t col = static_cast<int64_t>(threadIdx.x) * PIECE; col < a.cols; col += LONG_THREADS * PIECE) {
    const f32x8 h = load(col);
    squares = dot(h, h, squares);
  }
  const float rstd = 1.f / __builtin_sqrtf(__builtin_fmaf(row_sum<LONG_THREADS>(squares, 0), a.one_of_cols, a.eps));
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
  for (int64_t col = static_cast<int64_t>(threadIdx.x) * PIECE; col < pitch; col += LONG_THREADS * PIECE) {
    const f32x8 h = load(col);
    if (a.sum && col < a.cols) store_piece8(static_cast<S*>(a.sum) + row * a.lds + col, a.cols - col, h);   // sum may be residual: its piece has been read
    if (a.y || a.y8.codes) finish<E>(a, row, col, h, load_weight(a.weight, a.weight_f32, col, a.cols), rstd);
  }
}

// ---- backward -------------------------------------------------------------------------------------------------------------------
struct Backward {
  const void *dy, *h, *weight, *dsum;
  const float* rstd;
  void* dx;
  float* partial;   // [groups][pitch] sums over each group's rows, or null
  Image8 h8;        // where h is an image
  int64_t rows, cols, ldy, lds;
  int64_t groups;   // group g has the rows g, g + groups, ...
  float one_of_cols;
  int weight_f32;
};

template <typename H>
using HRaw = std::conditional_t<std::is_same_v<H, Image8>, RawCodes, Raw<std::conditional_t<std::is_same_v<H, Image8>, float, H>>>;
// the piece of h; nothing (zeros) behind the padded row
template <typename H>
__device__ __forceinline__ HRaw<H> load_h(const Backward& a, int64_t row, int64_t col) {
  if constexpr (std::is_same_v<H, Image8>)
    return col < a.h8.pitch ? load_raw(a.h8, row, col) : RawCodes{u32x2{0u, 0u}, 0u};
  else
    return load_raw(static_cast<const H*>(a.h) + row * a.lds + col, a.cols - col);
}

// A group of rows one after another; the weights and the sums for dw stay in registers.
template <typename E, typename S, typename H, int TX, int NV>
__global__ __launch_bounds__(block_threads(TX)) void k_norm_grad(Backward a) {
  const int tx = threadIdx.x & (TX - 1);
  const int64_t group = static_cast<int64_t>(blockIdx.x) * (block_threads(TX) / TX) + threadIdx.x / TX;
  if (group >= a.groups) return;   // as in k_norm
  f32x8 w[NV], dw[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t col = (static_cast<int64_t>(j) * TX + tx) * PIECE;
    w[j] = load_weight(a.weight, a.weight_f32, col, a.cols);
    dw[j] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  }
  int parity = 0;
  for (int64_t row = group; row < a.rows; row += a.groups, parity ^= 1) {
    Raw<E> dy[NV];
    HRaw<H> hr[NV];
    Raw<S> ds[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t col = (static_cast<int64_t>(j) * TX + tx) * PIECE;
      dy[j] = load_raw(static_cast<const E*>(a.dy) + row * a.ldy + col, a.cols - col);
      hr[j] = load_h<H>(a, row, col);
      if (a.dx && a.dsum) ds[j] = load_raw(static_cast<const S*>(a.dsum) + row * a.lds + col, a.cols - col);
    }
    const float rstd = a.rstd[row];
    f32x8 n[NV], u[NV];
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const f32x8 d = widen(dy[j]);
      n[j] = widen(hr[j]) * rstd;
      u[j] = w[j] * d;
#pragma unroll
      for (int e = 0; e < PIECE; ++e) dw[j][e] = __builtin_fmaf(d[e], n[j][e], dw[j][e]);
      s = dot(u[j], n[j], s);
    }
    if (!a.dx) continue;
    const float mean = row_sum<TX>(s, parity) * a.one_of_cols;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t col = (static_cast<int64_t>(j) * TX + tx) * PIECE;
      if (col >= a.cols) continue;
      f32x8 v, old;
      if (a.dsum) old = widen(ds[j]);
#pragma unroll
      for (int e = 0; e < PIECE; ++e) {
        v[e] = rstd * __builtin_fmaf(-mean, n[j][e], u[j][e]);
        if (a.dsum) v[e] += old[e];
      }
      store_piece8(static_cast<S*>(a.dx) + row * a.lds + col, a.cols - col, v);
    }
  }
  if (!a.partial) return;
  const int64_t pitch = mx8_pitch(a.cols);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t col = (static_cast<int64_t>(j) * TX + tx) * PIECE;
    if (col < a.cols) store_piece8(a.partial + group * pitch + col, PIECE, dw[j]);
  }
}

// A long row's dx: two readings of dy and h, the second one out of L2 or the cache behind it.
template <typename E, typename S, typename H>
__global__ __launch_bounds__(LONG_THREADS) void k_norm_grad_long(Backward a) {
  const int64_t row = blockIdx.x;
  const float rstd = a.rstd[row];
  auto terms = [&](int64_t col, f32x8& n, f32x8& u) {
    const Raw<E> dy = load_raw(static_cast<const E*>(a.dy) + row * a.ldy + col, a.cols - col);
    n = widen(load_h<H>(a, row, col)) * rstd;
    u = load_weight(a.weight, a.weight_f32, col, a.cols) * widen(dy);
  };
  f32x8 n, u;
  float s = 0.f;
  for (int64_t col = static_cast<int64_t>(threadIdx.x) * PIECE; col < a.cols; col += LONG_THREADS * PIECE) {
    terms(col, n, u);
    s = dot(u, n, s);
  }
  const float mean = row_sum<LONG_THREADS>(s, 0) * a.one_of_cols;
  for (int64_t col = static_cast<int64_t>(threadIdx.x) * PIECE; col < a.cols; col += LONG_THREADS * PIECE) {
    terms(col, n, u);
    f32x8 v;
#pragma unroll
    for (int e = 0; e < PIECE; ++e) v[e] = rstd * __builtin_fmaf(-mean, n[e], u[e]);
    if (a.dsum) v += widen(load_raw(static_cast<const S*>(a.dsum) + row * a.lds + col, a.cols - col));
    store_piece8(static_cast<S*>(a.dx) + row * a.lds + col, a.cols - col, v);
  }
}
// Long rows' sums for dw: a block has 2048 columns of a group of rows.
template <typename E, typename H>
__global__ __launch_bounds__(EACH_THREADS) void k_norm_dw_long(Backward a, int across) {
  const unsigned group = blockIdx.x / static_cast<unsigned>(across), along = blockIdx.x - group * across;
  const int64_t col = (static_cast<int64_t>(along) * EACH_THREADS + threadIdx.x) * PIECE;
  if (col >= a.cols) return;
  f32x8 dw = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int64_t row = group; row < a.rows; row += a.groups) {
    const f32x8 d = widen(load_raw(static_cast<const E*>(a.dy) + row * a.ldy + col, a.cols - col));
    const f32x8 n = widen(load_h<H>(a, row, col)) * a.rstd[row];
#pragma unroll
    for (int e = 0; e < PIECE; ++e) dw[e] = __builtin_fmaf(d[e], n[e], dw[e]);
  }
  store_piece8(a.partial + group * mx8_pitch(a.cols) + col, PIECE, dw);
}

// dweight <- beta dweight + the groups' sums: 32 columns to a block, whose 32 rows of threads add up a 32nd of the groups each.
constexpr int JOIN = 32;
__global__ __launch_bounds__(JOIN * JOIN) void k_norm_join(const float* partial, int64_t pitch, int64_t groups, int64_t cols, float beta, float* dweight) {
  __shared__ float part[JOIN][JOIN + 1];
  const int tx = threadIdx.x & (JOIN - 1), ty = threadIdx.x / JOIN;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * JOIN + tx;
  float s = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int64_t g = ty; g < groups; g += JOIN) s += partial[g * pitch + col];
  }
  part[ty][tx] = s;
  __syncthreads();
  if (ty != 0 || col >= cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < JOIN; ++i) s += part[i][tx];
  dweight[col] = beta != 0.f ? __builtin_fmaf(beta, dweight[col], s) : s;
}

// ---- host -----------------------------------------------------------------------------------------------------------------------
// Which threads hold a row: a wavefront up to 2048 columns, and as few more as its pieces need from there on.
template <typename F>
void for_width(int64_t cols, F&& f) {
  using std::integral_constant;
  auto go = [&](auto tx, auto nv) { f(tx, nv); };
  if (cols <= 64 * 8)
    go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (cols <= 64 * 8 * 4)
    go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  else if (cols <= 256 * 8 * 2)
    go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (cols <= 256 * 8 * 4)
    go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else
    go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
}
constexpr int64_t LONG_COLS = 512 * 8 * 4;   // rows longer than this are read twice

template <typename F>
void for_float(int dtype, F&& f) {
  if (dtype == CANZ_DT_F32)
    f(static_cast<float*>(nullptr));
  else
    f(static_cast<__bf16*>(nullptr));
}

void launch_forward(const canz_norm& x, const Forward& a, hipStream_t st) {
  for_float(x.dtype, [&](auto e) {
    for_float(x.sum_dtype, [&](auto s) {
      using E = std::remove_pointer_t<decltype(e)>;
      using S = std::remove_pointer_t<decltype(s)>;
      if (a.cols > LONG_COLS) {
        k_norm_long<E, S><<<dim3(static_cast<unsigned>(a.rows)), LONG_THREADS, 0, st>>>(a);
        return;
      }
      for_width(a.cols, [&](auto tx, auto nv) {
        constexpr int TX = tx(), THREADS = block_threads(TX), EACH = THREADS / TX;
        k_norm<E, S, TX, nv()><<<dim3(static_cast<unsigned>((a.rows + EACH - 1) / EACH)), THREADS, 0, st>>>(a);
      });
    });
  });
}

void launch_backward(const canz_norm_grad& x, const Backward& a, hipStream_t st) {
  for_float(x.dtype, [&](auto e) {
    for_float(x.sum_dtype, [&](auto s) {
      using E = std::remove_pointer_t<decltype(e)>;
      using S = std::remove_pointer_t<decltype(s)>;
      auto with = [&](auto h) {
        using H = std::remove_pointer_t<decltype(h)>;
        if (a.cols > LONG_COLS) {
          if (a.dx) k_norm_grad_long<E, S, H><<<dim3(static_cast<unsigned>(a.rows)), LONG_THREADS, 0, st>>>(a);
          const int across = static_cast<int>((a.cols + EACH_THREADS * PIECE - 1) / (EACH_THREADS * PIECE));
          if (a.partial) k_norm_dw_long<E, H><<<dim3(static_cast<unsigned>(a.groups * across)), EACH_THREADS, 0, st>>>(a, across);
          return;
        }
        for_width(a.cols, [&](auto tx, auto nv) {
          constexpr int TX = tx(), THREADS = block_threads(TX), EACH = THREADS / TX;
          k_norm_grad<E, S, H, TX, nv()><<<dim3(static_cast<unsigned>((a.groups + EACH - 1) / EACH)), THREADS, 0, st>>>(a);
        });
      };
      if (x.h_dtype == CANZ_DT_MX8)
        with(static_cast<Image8*>(nullptr));
      else
        for_float(x.h_dtype, with);
    });
  });
}

// Groups of rows that are summed up by themselves for dw: enough of them to fill the chip, few enough for the join.  us for backward and join: 8192 x 4096 with 256 groups 67 + 5, 512 46 + 5, 1024 48 + 5,
// 2048 54 + 8; 4097 x 1531 with 512 groups 36 + 5, 1024 25 + 5, 2048 22 + 6, 4096 26 + 10.
int64_t groups_of(const canz_norm_grad& x) {
  if (!x.dweight) return x.rows;
  int64_t most = 512;
  if (x.cols > LONG_COLS)
    most = 128;
  else
    for_width(x.cols, [&](auto tx, auto) { most = tx() == 64 ? 1024 : 512; });
  return std::min(x.rows, most);
}
size_t partial_bytes(const canz_norm_grad& x) { return x.dweight ? static_cast<size_t>(groups_of(x)) * mx8_pitch(x.cols) * sizeof(float) : 0; }

bool bad(const void* p, uintptr_t align, bool needed) { return p ? misaligned(p, align) : needed; }

int check_forward(const canz_norm& a, int idx) {
  if (int rc = check_extents("norm", idx, a.rows, a.cols)) return rc;
  if (!float_dtype(a.dtype) || !float_dtype(a.sum_dtype) || !float_dtype(a.weight_dtype)) return fail(CANZ_EUNSUPPORTED, "norm %d: unknown dtype", idx);
  if (!(a.eps >= 0.f)) return fail(CANZ_EINVAL, "norm %d: eps negative or NaN", idx);
  if (a.ldx < a.cols || a.lds < a.cols || a.ldy < a.cols) return fail(CANZ_EINVAL, "norm %d: a row distance below cols", idx);
  if (a.rows == 0 || a.cols == 0) return CANZ_OK;
  if (!a.sum && !a.y && !a.y8 && !a.rstd) return fail(CANZ_EINVAL, "norm %d: nothing is asked for", idx);
  const uintptr_t el = element_bytes(a.dtype), sel = element_bytes(a.sum_dtype);
  if (bad(a.x, el, true) || bad(a.residual, sel, false) || bad(a.weight, element_bytes(a.weight_dtype), a.y || a.y8) || bad(a.sum, sel, false) ||
      bad(a.y, el, false) || bad(a.rstd, 4, false))
    return fail(CANZ_EINVAL, "norm %d: a buffer is null or not aligned to its elements", idx);
  if (bad(a.y8, 256, false)) return fail(CANZ_EINVAL, "norm %d: y8 is not 256-byte aligned", idx);
  return CANZ_OK;
}

int check_backward(const canz_norm_grad& a, int idx, bool need_ptrs) {
  if (int rc = check_extents("norm", idx, a.rows, a.cols)) return rc;
  if (!float_dtype(a.dtype) || !float_dtype(a.sum_dtype) || !float_dtype(a.weight_dtype) || (!float_dtype(a.h_dtype) && a.h_dtype != CANZ_DT_MX8))
    return fail(CANZ_EUNSUPPORTED, "norm %d: unknown dtype", idx);
  if (a.ldy < a.cols || a.lds < a.cols) return fail(CANZ_EINVAL, "norm %d: a row distance below cols", idx);
  if (!need_ptrs || a.cols == 0) return CANZ_OK;
  if (!a.dx && !a.dweight) return fail(CANZ_EINVAL, "norm %d: neither dx nor dweight is asked for", idx);
  if (bad(a.dweight, 4, false)) return fail(CANZ_EINVAL, "norm %d: dweight is not aligned to its elements", idx);
  if (a.rows == 0) return CANZ_OK;
  const uintptr_t sel = element_bytes(a.sum_dtype), hel = a.h_dtype == CANZ_DT_MX8 ? 256 : element_bytes(a.h_dtype);
  if (bad(a.dy, element_bytes(a.dtype), true) || bad(a.weight, element_bytes(a.weight_dtype), true) || bad(a.rstd, 4, true) || bad(a.dsum, sel, false) ||
      bad(a.dx, sel, false))
    return fail(CANZ_EINVAL, "norm %d: a buffer is null or not aligned to its elements", idx);
  if (bad(a.h, hel, true)) return fail(CANZ_EINVAL, "norm %d: h null or not aligned to %s", idx, hel == 256 ? "256 bytes" : "its elements");
  return CANZ_OK;
}

size_t backward_workspace(const canz_norm_grad* a, int32_t n) {
  size_t need = 256;
  for (int i = 0; i < n; ++i) need = std::max(need, partial_bytes(a[i]));
  return need;
}

}  // namespace
}  // namespace canz

extern "C" int canz_norm_forward(const canz_norm* a, int32_t n, void* hip_stream) {
  using namespace canz;
  if (n < 0 || (n > 0 && !a)) return fail(CANZ_EINVAL, "bad array");
  for (int i = 0; i < n; ++i)
    if (int rc = check_forward(a[i], i)) return rc;
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  for (int i = 0; i < n; ++i) {
    const canz_norm& x = a[i];
    if (x.rows == 0 || x.cols == 0) continue;
    const Forward f{x.x, x.residual, x.weight, x.sum, x.y, image8(x.y8, x.rows, x.cols), x.rstd, x.rows, x.cols, x.ldx, x.lds, x.ldy, x.eps,
                    static_cast<float>(1.0 / static_cast<double>(x.cols)), x.weight_dtype == CANZ_DT_F32};
    launch_forward(x, f, st);
    if (const hipError_t err = hipGetLastError(); err != hipSuccess) return fail(CANZ_EHIP, "norm: %s", hipGetErrorString(err));
  }
  return CANZ_OK;
}

extern "C" int canz_norm_backward_workspace_bytes(const canz_norm_grad* a, int32_t n, size_t* bytes_out) {
  using namespace canz;
  if (!bytes_out) return fail(CANZ_EINVAL, "null output pointer");
  if (n < 0 || (n > 0 && !a)) return fail(CANZ_EINVAL, "bad array");
  for (int i = 0; i < n; ++i)
    if (int rc = check_backward(a[i], i, false)) return rc;
  *bytes_out = backward_workspace(a, n);
  return CANZ_OK;
}

extern "C" int canz_norm_backward(const canz_norm_grad* a, int32_t n, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace canz;
  if (n < 0 || (n > 0 && !a)) return fail(CANZ_EINVAL, "bad array");
  bool any = false, scratch = false;
  for (int i = 0; i < n; ++i) {
    if (int rc = check_backward(a[i], i, true)) return rc;
    any = any || a[i].cols > 0;
    scratch = scratch || (a[i].cols > 0 && a[i].dweight);
  }
  if (!any) return CANZ_OK;
  if (scratch) {
    if (!workspace || misaligned(workspace, 256)) return fail(CANZ_EWORKSPACE, "workspace null or not 256-byte aligned");
    const size_t need = backward_workspace(a, n);
    if (workspace_bytes < need) return fail(CANZ_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
  }
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  for (int i = 0; i < n; ++i) {
    const canz_norm_grad& x = a[i];
    if (x.cols == 0) continue;
    float* const partial = x.dweight ? static_cast<float*>(workspace) : nullptr;
    const Backward b{x.dy, x.h, x.weight, x.dsum, x.rstd, x.dx, partial, image8(x.h_dtype == CANZ_DT_MX8 ? x.h : nullptr, x.rows, x.cols), x.rows, x.cols, x.ldy,
                     x.lds, groups_of(x), static_cast<float>(1.0 / static_cast<double>(x.cols)), x.weight_dtype == CANZ_DT_F32};
    if (x.rows > 0) launch_backward(x, b, st);
    if (x.dweight)
      k_norm_join<<<dim3(static_cast<unsigned>((x.cols + JOIN - 1) / JOIN)), JOIN * JOIN, 0, st>>>(partial, mx8_pitch(x.cols), x.rows > 0 ? b.groups : 0, x.cols,
                                                                                                  x.beta, x.dweight);
    if (const hipError_t err = hipGetLastError(); err != hipSuccess) return fail(CANZ_EHIP, "norm: %s", hipGetErrorString(err));
  }
  return CANZ_OK;
}
