// canz_act_forward and canz_act_backward: out = act(gate) up and its gradients, gate and up kept in 8 bits in between.
//
// Both read every operand once and write every result once; memory is what bounds them.  A thread takes eight elements of a row, its quad a block of the images.  8192 x 12288 in bf16 with SiLU, gate
// and up: forward with both images 145 us (811 MB, 5.6 TB/s), backward from them with both gradients and the result once more 174 us (1013 MB, 5.8 TB/s).  With two rows to a thread 146 and 178 us
// (fp32 253 and 350 instead of 247 and 329).
#include "act.h"
#include "canz_internal.h"
#include "mx8.h"

namespace canz {
namespace {

struct Forward {
  const void *gate, *up;
  void* out;
  Image8 gate8, up8;   // codes null: not asked for
  int64_t rows, cols, ld_in, ld_out;
  int log_tx, across;
};

template <typename E, int ACT, bool UP>
__global__ __launch_bounds__(EACH_THREADS) void k_act_forward(Forward a) {
  const Spot s = spot(blockIdx.x, a.log_tx, a.across);
  if (s.row >= a.rows) return;   // a row's quads are whole
  const int64_t left = a.cols - s.col, at = s.row * a.ld_in + s.col;
  const Raw<E> gate = load_raw(static_cast<const E*>(a.gate) + at, left);
  Raw<E> up;
  if (UP) up = load_raw(static_cast<const E*>(a.up) + at, left);
  const f32x8 g = widen(gate);
  f32x8 u;
  if (UP) u = widen(up);
  if (a.gate8.codes) store_codes(a.gate8, s.row, s.col, a.cols, round8(g));
  if (UP && a.up8.codes) store_codes(a.up8, s.row, s.col, a.cols, round8(u));
  if (a.out && left > 0) {
    f32x8 v;
#pragma unroll
    for (int e = 0; e < PIECE; ++e) {
      const float t = act_both<ACT, std::is_same_v<E, float>>(g[e]).value;
      v[e] = UP ? t * u[e] : t;
    }
    store_piece8(static_cast<E*>(a.out) + s.row * a.ld_out + s.col, left, v);
  }
}

struct Backward {
  const void *dout, *gate, *up;
  void *dgate, *dup, *out;
  Image8 gate8, up8;   // where gate and up are images
  int64_t rows, cols, ld_in, ld_out;
  int log_tx, across;
};

// I: the type of gate and up, or Image8
template <typename E, typename I, int ACT, bool UP>
__global__ __launch_bounds__(EACH_THREADS) void k_act_backward(Backward a) {
  constexpr bool IMAGE = std::is_same_v<I, Image8>;
  const Spot s = spot(blockIdx.x, a.log_tx, a.across);
  const int64_t left = a.cols - s.col;
  if (s.row >= a.rows || left <= 0) return;
  std::conditional_t<IMAGE, RawCodes, Raw<std::conditional_t<IMAGE, float, I>>> gate, up;
  Raw<E> dout;
  if constexpr (IMAGE) {
    gate = load_raw(a.gate8, s.row, s.col);
    if (UP) up = load_raw(a.up8, s.row, s.col);
  } else {
    gate = load_raw(static_cast<const I*>(a.gate) + s.row * a.ld_in + s.col, left);
    if (UP) up = load_raw(static_cast<const I*>(a.up) + s.row * a.ld_in + s.col, left);
  }
  if (a.dout) dout = load_raw(static_cast<const E*>(a.dout) + s.row * a.ld_out + s.col, left);
  const f32x8 g = widen(gate);
  f32x8 u, d, value, slope;
  if (UP) u = widen(up);
  if (a.dout) d = widen(dout);
#pragma unroll
  for (int e = 0; e < PIECE; ++e) {
    const ActValue t = act_both<ACT, std::is_same_v<E, float>>(g[e]);
    value[e] = t.value, slope[e] = t.slope;
  }
  f32x8 v;
  if (a.dgate) {
#pragma unroll
    for (int e = 0; e < PIECE; ++e) v[e] = (UP ? d[e] * u[e] : d[e]) * slope[e];
    store_piece8(static_cast<E*>(a.dgate) + s.row * a.ld_in + s.col, left, v);
  }
  if (UP && a.dup) {
#pragma unroll
    for (int e = 0; e < PIECE; ++e) v[e] = d[e] * value[e];
    store_piece8(static_cast<E*>(a.dup) + s.row * a.ld_in + s.col, left, v);
  }
  if (a.out) {
#pragma unroll
    for (int e = 0; e < PIECE; ++e) v[e] = UP ? value[e] * u[e] : value[e];
    store_piece8(static_cast<E*>(a.out) + s.row * a.ld_out + s.col, left, v);
  }
}

template <typename F>
void for_act(int act, F&& f) {
  switch (act) {
    case CANZ_ACT_SILU: return f(std::integral_constant<int, CANZ_ACT_SILU>{});
    case CANZ_ACT_GELU: return f(std::integral_constant<int, CANZ_ACT_GELU>{});
    case CANZ_ACT_RELU: return f(std::integral_constant<int, CANZ_ACT_RELU>{});
    default: return f(std::integral_constant<int, CANZ_ACT_NONE>{});
  }
}

template <typename E>
void launch_forward(const Forward& f, int act, bool up, dim3 grid, hipStream_t st) {
  for_act(act, [&](auto kind) {
    if (up)
      k_act_forward<E, kind(), true><<<grid, EACH_THREADS, 0, st>>>(f);
    else
      k_act_forward<E, kind(), false><<<grid, EACH_THREADS, 0, st>>>(f);
  });
}

template <typename E, typename I>
void launch_backward(const Backward& b, int act, bool up, dim3 grid, hipStream_t st) {
  for_act(act, [&](auto kind) {
    if (up)
      k_act_backward<E, I, kind(), true><<<grid, EACH_THREADS, 0, st>>>(b);
    else
      k_act_backward<E, I, kind(), false><<<grid, EACH_THREADS, 0, st>>>(b);
  });
}
template <typename E>
void launch_backward(const Backward& b, int in_dtype, int act, bool up, dim3 grid, hipStream_t st) {
  if (in_dtype == CANZ_DT_MX8)
    launch_backward<E, Image8>(b, act, up, grid, st);
  else if (in_dtype == CANZ_DT_F32)
    launch_backward<E, float>(b, act, up, grid, st);
  else
    launch_backward<E, __bf16>(b, act, up, grid, st);
}

bool bad(const void* p, uintptr_t align, bool needed) { return p ? misaligned(p, align) : needed; }

template <typename A>
int check_common(const A& a, int idx) {
  if (int rc = check_extents("activation", idx, a.rows, a.cols)) return rc;
  if (!act_known(a.act)) return fail(CANZ_EUNSUPPORTED, "activation %d: unknown act %d", idx, a.act);
  if (!float_dtype(a.dtype)) return fail(CANZ_EUNSUPPORTED, "activation %d: unknown dtype", idx);
  if (a.ld_in < a.cols || a.ld_out < a.cols) return fail(CANZ_EINVAL, "activation %d: a row distance below cols", idx);
  return CANZ_OK;
}

int check_forward(const canz_act& a, int idx) {
  if (int rc = check_common(a, idx)) return rc;
  if (a.rows == 0 || a.cols == 0) return CANZ_OK;
  const uintptr_t el = element_bytes(a.dtype);
  if (!a.out && !a.gate8 && !a.up8) return fail(CANZ_EINVAL, "activation %d: nothing is asked for", idx);
  if (a.up8 && !a.up) return fail(CANZ_EINVAL, "activation %d: up8 without up", idx);
  if (bad(a.gate, el, true) || bad(a.up, el, false) || bad(a.out, el, false))
    return fail(CANZ_EINVAL, "activation %d: a matrix is null or not aligned to its elements", idx);
  if (bad(a.gate8, 256, false) || bad(a.up8, 256, false)) return fail(CANZ_EINVAL, "activation %d: an image is not 256-byte aligned", idx);
  return CANZ_OK;
}

int check_backward(const canz_act_grad& a, int idx) {
  if (int rc = check_common(a, idx)) return rc;
  if (!float_dtype(a.in_dtype) && a.in_dtype != CANZ_DT_MX8) return fail(CANZ_EUNSUPPORTED, "activation %d: unknown in_dtype", idx);
  if (a.rows == 0 || a.cols == 0) return CANZ_OK;
  const uintptr_t el = element_bytes(a.dtype), in = a.in_dtype == CANZ_DT_MX8 ? 256 : element_bytes(a.in_dtype);
  if (!a.dgate && !a.dup && !a.out) return fail(CANZ_EINVAL, "activation %d: nothing is asked for", idx);
  if (a.dup && !a.up) return fail(CANZ_EINVAL, "activation %d: dup without up", idx);
  if (bad(a.gate, in, true) || bad(a.up, in, false))
    return fail(CANZ_EINVAL, "activation %d: gate or up null or not aligned to %s", idx, in == 256 ? "256 bytes" : "its elements");
  if (bad(a.dout, el, a.dgate || a.dup) || bad(a.dgate, el, false) || bad(a.dup, el, false) || bad(a.out, el, false))
    return fail(CANZ_EINVAL, "activation %d: a matrix is null or not aligned to its elements", idx);
  if (((a.dgate && a.dgate == a.gate) || (a.dup && a.dup == a.up)) && a.in_dtype != a.dtype)
    return fail(CANZ_EINVAL, "activation %d: a gradient over its argument, which has another type", idx);
  return CANZ_OK;
}

}  // namespace
}  // namespace canz

extern "C" int canz_act_forward(const canz_act* a, int32_t n, void* hip_stream) {
  using namespace canz;
  if (n < 0 || (n > 0 && !a)) return fail(CANZ_EINVAL, "bad array");
  for (int i = 0; i < n; ++i)
    if (int rc = check_forward(a[i], i)) return rc;
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  for (int i = 0; i < n; ++i) {
    const canz_act& x = a[i];
    if (x.rows == 0 || x.cols == 0) continue;
    const Cover c = cover(x.rows, x.cols);
    const Forward f{x.gate, x.up, x.out, image8(x.gate8, x.rows, x.cols), image8(x.up8, x.rows, x.cols), x.rows, x.cols, x.ld_in, x.ld_out, c.log_tx, c.across};
    const dim3 grid(static_cast<unsigned>(c.blocks));
    if (x.dtype == CANZ_DT_F32)
      launch_forward<float>(f, x.act, x.up != nullptr, grid, st);
    else
      launch_forward<__bf16>(f, x.act, x.up != nullptr, grid, st);
    if (const hipError_t err = hipGetLastError(); err != hipSuccess) return fail(CANZ_EHIP, "activation: %s", hipGetErrorString(err));
  }
  return CANZ_OK;
}

extern "C" int canz_act_backward(const canz_act_grad* a, int32_t n, void* hip_stream) {
  using namespace canz;
  if (n < 0 || (n > 0 && !a)) return fail(CANZ_EINVAL, "bad array");
  for (int i = 0; i < n; ++i)
    if (int rc = check_backward(a[i], i)) return rc;
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  for (int i = 0; i < n; ++i) {
    const canz_act_grad& x = a[i];
    if (x.rows == 0 || x.cols == 0) continue;
    const Cover c = cover(x.rows, x.cols);
    const Backward b{x.dgate || x.dup ? x.dout : nullptr, x.gate, x.up, x.dgate, x.dup, x.out, image8(x.gate, x.rows, x.cols),
                     image8(x.up, x.rows, x.cols), x.rows, x.cols, x.ld_in, x.ld_out, c.log_tx, c.across};
    const dim3 grid(static_cast<unsigned>(c.blocks));
    if (x.dtype == CANZ_DT_F32)
      launch_backward<float>(b, x.in_dtype, x.act, x.up != nullptr, grid, st);
    else
      launch_backward<__bf16>(b, x.in_dtype, x.act, x.up != nullptr, grid, st);
    if (const hipError_t err = hipGetLastError(); err != hipSuccess) return fail(CANZ_EHIP, "activation: %s", hipGetErrorString(err));
  }
  return CANZ_OK;
}
