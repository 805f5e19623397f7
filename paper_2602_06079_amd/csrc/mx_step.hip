// canz_mx_*: host side of the microscaled images and their products.  Validates the groups and enqueues the launches on the caller's
// stream; nothing here allocates, copies to the device or synchronises.
#include <algorithm>

#include "canz_internal.h"
#include "kernels.h"
#include "mx.h"

namespace canz {

int check_mx_group(const canz_mx_group& g, int idx, bool back) {
  if (g.n_mats < 0) return fail(CANZ_EINVAL, "group %d: n_mats < 0", idx);
  if (g.rows < 0 || g.cols < 0) return fail(CANZ_EINVAL, "group %d: negative extent", idx);
  if (g.rows > MX_MAX_EXTENT || g.cols > MX_MAX_EXTENT)
    return fail(CANZ_ESHAPE, "group %d: extent above %lld", idx, static_cast<long long>(MX_MAX_EXTENT));
  if (!mx_fits_grid(g.rows, g.cols)) return fail(CANZ_ESHAPE, "group %d: more than 2^37 padded elements in a matrix", idx);
  if (g.dtype != CANZ_DT_F32 && g.dtype != CANZ_DT_BF16) return fail(CANZ_EUNSUPPORTED, "group %d: unknown dtype", idx);
  if (g.ld < g.cols) return fail(CANZ_EINVAL, "group %d: ld below cols", idx);
  if (g.n_mats == 0 || g.rows == 0 || g.cols == 0) return CANZ_OK;
  if (!g.mat) return fail(CANZ_EINVAL, "group %d: null pointer table", idx);
  if (!g.by_row && !g.by_col) return fail(CANZ_EINVAL, "group %d: neither by_row nor by_col", idx);
  if (back && g.by_row && g.by_col) return fail(CANZ_EINVAL, "group %d: one of by_row and by_col is read, both are given", idx);
  auto bad = [](const void* p, uintptr_t align) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; };
  for (int i = 0; i < g.n_mats; ++i) {
    if (bad(g.mat[i], 16)) return fail(CANZ_EINVAL, "group %d: mat[%d] null or not 16-byte aligned", idx, i);
    if (g.by_row && bad(g.by_row[i], 256)) return fail(CANZ_EINVAL, "group %d: by_row[%d] null or not 256-byte aligned", idx, i);
    if (g.by_col && bad(g.by_col[i], 256)) return fail(CANZ_EINVAL, "group %d: by_col[%d] null or not 256-byte aligned", idx, i);
    if (!back && g.noise && g.noise[i] == nullptr) return fail(CANZ_EINVAL, "group %d: noise[%d] null", idx, i);
  }
  return CANZ_OK;
}

namespace {

constexpr size_t ALIGN = 256;

// calls fn(MxMats) for every launch of a checked group
template <typename F>
int for_each_launch(const canz_mx_group& g, int scale_mode, bool noise, F&& fn) {
  if (g.rows == 0 || g.cols == 0) return CANZ_OK;
  for (int64_t first = 0; first < g.n_mats; first += MX_MAX_MATS) {
    MxMats m{};
    m.most_rows = g.rows, m.cols = g.cols, m.ld = g.ld;
    m.n = static_cast<int>(std::min<int64_t>(MX_MAX_MATS, g.n_mats - first));
    m.dtype = g.dtype, m.scale_mode = scale_mode;
    for (int i = 0; i < m.n; ++i) {
      m.rows[i] = static_cast<int>(g.rows);
      m.mat[i] = g.mat[first + i];
      m.by_row[i] = g.by_row ? static_cast<uint8_t*>(g.by_row[first + i]) : nullptr;
      m.by_col[i] = g.by_col ? static_cast<uint8_t*>(g.by_col[first + i]) : nullptr;
      m.noise[i] = noise && g.noise ? static_cast<const uint8_t*>(g.noise[first + i]) : nullptr;
    }
    const hipError_t err = fn(m);
    if (err != hipSuccess) return fail(CANZ_EHIP, "microscaled image: %s", hipGetErrorString(err));
  }
  return CANZ_OK;
}

int check_scale_mode(int32_t mode) {
  if (mode != CANZ_MX_SCALE_FLOOR && mode != CANZ_MX_SCALE_CEIL) return fail(CANZ_EUNSUPPORTED, "unknown scale_mode %d", mode);
  return CANZ_OK;
}

bool mx_idle(const canz_mx_product_group& g) { return g.n_prods == 0 || g.m == 0 || g.n == 0; }

int check_product_group(const canz_mx_product_group& g, int idx, bool need_ptrs) {
  if (g.n_prods < 0) return fail(CANZ_EINVAL, "group %d: n_prods < 0", idx);
  if (g.m < 0 || g.n < 0 || g.k < 0) return fail(CANZ_EINVAL, "group %d: negative extent", idx);
  if (g.m > MX_MAX_EXTENT || g.n > MX_MAX_EXTENT || g.k > MX_MAX_EXTENT)
    return fail(CANZ_ESHAPE, "group %d: extent above %lld", idx, static_cast<long long>(MX_MAX_EXTENT));
  if (!mx_fits_grid(g.m, g.n) || !mx_fits_grid(g.m, g.k) || !mx_fits_grid(g.n, g.k))
    return fail(CANZ_ESHAPE, "group %d: more than 2^37 padded elements in a matrix", idx);
  if (g.a_dtype != CANZ_DT_F32 && g.a_dtype != CANZ_DT_BF16 && g.a_dtype != CANZ_DT_MX)
    return fail(CANZ_EUNSUPPORTED, "group %d: unknown a_dtype", idx);
  if (g.out_dtype != CANZ_DT_F32 && g.out_dtype != CANZ_DT_BF16) return fail(CANZ_EUNSUPPORTED, "group %d: unknown out_dtype", idx);
  if (int rc = check_scale_mode(g.a_scale_mode)) return rc;
  if (g.a_dtype != CANZ_DT_MX && g.lda < g.k) return fail(CANZ_EINVAL, "group %d: lda below k", idx);
  if (g.ldc < g.n) return fail(CANZ_EINVAL, "group %d: ldc below n", idx);
  if (!need_ptrs || mx_idle(g)) return CANZ_OK;
  if (!g.c || (g.k > 0 && (!g.a || !g.b))) return fail(CANZ_EINVAL, "group %d: null pointer table", idx);
  auto bad = [](const void* p, uintptr_t align) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; };
  for (int i = 0; i < g.n_prods; ++i) {
    if (bad(g.c[i], 16)) return fail(CANZ_EINVAL, "group %d: c[%d] null or not 16-byte aligned", idx, i);
    if (g.k == 0) continue;
    const bool image = g.a_dtype == CANZ_DT_MX;
    if (bad(g.a[i], image ? 256 : 16)) return fail(CANZ_EINVAL, "group %d: a[%d] null or not %d-byte aligned", idx, i, image ? 256 : 16);
    if (bad(g.b[i], 256)) return fail(CANZ_EINVAL, "group %d: b[%d] null or not 256-byte aligned", idx, i);
  }
  return CANZ_OK;
}

// whether A is rounded by a launch of its own, into an image in the workspace
bool mx_rounded_before(const canz_mx_product_group& g) { return !mx_idle(g) && g.k > 0 && g.a_dtype != CANZ_DT_MX && !mx_rounds_on_the_way(g.m, g.n, g.k); }

// bytes of the sums of the parts that k is cut into
size_t mx_part_bytes(int64_t m, int64_t n, int64_t k) {
  const int parts = mx_parts(m, n, k);
  return parts > 1 ? (static_cast<size_t>(parts) * m * n * sizeof(float) + ALIGN - 1) / ALIGN * ALIGN : 0;
}

// room for these images, and for these sums
int product_workspace(const canz_mx_product_group* g, int32_t n_groups, size_t* bytes_out) {
  size_t need = 0;
  for (int i = 0; i < n_groups; ++i) {
    if (mx_idle(g[i])) continue;
    const size_t each = (mx_rounded_before(g[i]) ? mx_image_bytes(g[i].m, g[i].k) : 0) + mx_part_bytes(g[i].m, g[i].n, g[i].k);
    size_t group = 0;
    if (__builtin_mul_overflow(each, static_cast<size_t>(g[i].n_prods), &group) || __builtin_add_overflow(need, group, &need))
      return fail(CANZ_ESHAPE, "group %d: the workspace would have more bytes than 64 bits count", i);
  }
  *bytes_out = std::max(need, ALIGN);
  return CANZ_OK;
}

}  // namespace

int quantize_group(const canz_mx_group& g, int scale_mode, hipStream_t st) {
  return for_each_launch(g, scale_mode, true, [&](const MxMats& m) { return launch_mx_quantize(m, st); });
}

}  // namespace canz

extern "C" int canz_mx_image_bytes(int64_t rows, int64_t cols, size_t* bytes_out) {
  using namespace canz;
  if (!bytes_out) return fail(CANZ_EINVAL, "null output pointer");
  if (rows < 0 || cols < 0) return fail(CANZ_EINVAL, "negative extent");
  if (rows > MX_MAX_EXTENT || cols > MX_MAX_EXTENT) return fail(CANZ_ESHAPE, "extent above %lld", static_cast<long long>(MX_MAX_EXTENT));
  *bytes_out = static_cast<size_t>(mx_image_bytes(rows, cols));
  return CANZ_OK;
}

extern "C" int canz_mx_quantize(const canz_mx_group* g, int32_t n_groups, int32_t scale_mode, void* hip_stream) {
  using namespace canz;
  if (n_groups < 0 || (n_groups > 0 && !g)) return fail(CANZ_EINVAL, "bad group array");
  if (int rc = check_scale_mode(scale_mode)) return rc;
  for (int i = 0; i < n_groups; ++i)
    if (int rc = check_mx_group(g[i], i, false)) return rc;
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  for (int i = 0; i < n_groups; ++i)
    if (int rc = quantize_group(g[i], scale_mode, st)) return rc;
  return CANZ_OK;
}

extern "C" int canz_mx_dequantize(const canz_mx_group* g, int32_t n_groups, void* hip_stream) {
  using namespace canz;
  if (n_groups < 0 || (n_groups > 0 && !g)) return fail(CANZ_EINVAL, "bad group array");
  for (int i = 0; i < n_groups; ++i)
    if (int rc = check_mx_group(g[i], i, true)) return rc;
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  for (int i = 0; i < n_groups; ++i) {
    const int rc = for_each_launch(g[i], 0, false, [&](const MxMats& m) { return launch_mx_dequantize(m, st); });
    if (rc) return rc;
  }
  return CANZ_OK;
}

extern "C" int canz_mx_product_workspace_bytes(const canz_mx_product_group* g, int32_t n_groups, size_t* bytes_out) {
  using namespace canz;
  if (!bytes_out) return fail(CANZ_EINVAL, "null output pointer");
  if (n_groups < 0 || (n_groups > 0 && !g)) return fail(CANZ_EINVAL, "bad group array");
  for (int i = 0; i < n_groups; ++i)
    if (int rc = check_product_group(g[i], i, false)) return rc;
  return product_workspace(g, n_groups, bytes_out);
}

extern "C" int canz_mx_product(const canz_mx_product_group* g, int32_t n_groups, void* workspace, size_t workspace_bytes,
                               void* hip_stream) {
  using namespace canz;
  if (n_groups < 0 || (n_groups > 0 && !g)) return fail(CANZ_EINVAL, "bad group array");
  bool any = false;
  for (int i = 0; i < n_groups; ++i) {
    if (int rc = check_product_group(g[i], i, true)) return rc;
    any = any || !mx_idle(g[i]);
  }
  if (!any) return CANZ_OK;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & (ALIGN - 1)))
    return fail(CANZ_EWORKSPACE, "workspace null or not 256-byte aligned");
  size_t need = 0;
  if (int rc = product_workspace(g, n_groups, &need)) return rc;
  if (workspace_bytes < need) return fail(CANZ_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));

  // images of the matrices that are rounded before: those of one width, type and rule in one launch, whatever their rows (experts)
  uint8_t* const images = static_cast<uint8_t*>(workspace);
  size_t at = 0;
  MxMats mats{};
  auto round = [&]() -> int {
    if (mats.n == 0) return CANZ_OK;
    const hipError_t err = launch_mx_quantize(mats, st);
    mats.n = 0;
    return err == hipSuccess ? CANZ_OK : fail(CANZ_EHIP, "microscaled product: %s", hipGetErrorString(err));
  };
  for (int i = 0; i < n_groups; ++i) {
    const canz_mx_product_group& gi = g[i];
    if (!mx_rounded_before(gi)) continue;
    for (int x = 0; x < gi.n_prods; ++x) {
      const bool alike = mats.cols == gi.k && mats.ld == gi.lda && mats.dtype == gi.a_dtype && mats.scale_mode == gi.a_scale_mode;
      if (mats.n == MX_MAX_MATS || !alike)
        if (int rc = round()) return rc;
      if (mats.n == 0) mats.cols = gi.k, mats.ld = gi.lda, mats.dtype = gi.a_dtype, mats.scale_mode = gi.a_scale_mode, mats.most_rows = 0;
      mats.most_rows = std::max(mats.most_rows, gi.m);
      mats.rows[mats.n] = static_cast<int>(gi.m);
      mats.mat[mats.n] = const_cast<void*>(gi.a[x]);
      mats.by_row[mats.n++] = images + at;
      at += static_cast<size_t>(mx_image_bytes(gi.m, gi.k));
    }
  }
  if (int rc = round()) return rc;

  uint8_t* sums = images + at;
  at = 0;
  MxProblems ps;
  ps.n = 0;
  struct Join {
    MxProblem p;
    const float* sums;
    int parts;
  } joins[MX_MAX_PROBLEMS];
  int n_joins = 0;
  auto flush = [&]() -> int {
    hipError_t err = launch_mx_product(ps, st);
    for (int i = 0; i < n_joins && err == hipSuccess; ++i) err = launch_mx_join(joins[i].p, joins[i].sums, joins[i].parts, st);
    ps.n = n_joins = 0;
    return err == hipSuccess ? CANZ_OK : fail(CANZ_EHIP, "microscaled product: %s", hipGetErrorString(err));
  };
  for (int i = 0; i < n_groups; ++i) {
    const canz_mx_product_group& gi = g[i];
    if (mx_idle(gi)) continue;
    const bool before = mx_rounded_before(gi);
    const int parts = mx_parts(gi.m, gi.n, gi.k), units = static_cast<int>(mx_k_units(gi.k));
    for (int x = 0; x < gi.n_prods; ++x) {
      MxProblem p{};
      p.a = before ? images + at : static_cast<const uint8_t*>(gi.k > 0 ? gi.a[x] : nullptr);
      if (before) at += static_cast<size_t>(mx_image_bytes(gi.m, gi.k));
      p.a_dtype = before ? CANZ_DT_MX : gi.a_dtype, p.a_ceil = gi.a_scale_mode == CANZ_MX_SCALE_CEIL, p.lda = gi.lda;
      p.b = static_cast<const uint8_t*>(gi.k > 0 ? gi.b[x] : nullptr);
      p.c = gi.c[x];
      p.m = gi.m, p.n = gi.n, p.k = gi.k, p.ldc = gi.ldc;
      p.alpha = gi.alpha, p.beta = gi.beta, p.out_dtype = gi.out_dtype;
      p.units = units;
      if (ps.n + parts > MX_MAX_PROBLEMS)
        if (int rc = flush()) return rc;
      if (parts == 1) {
        ps.pr[ps.n++] = p;
        continue;
      }
      joins[n_joins++] = Join{p, reinterpret_cast<const float*>(sums), parts};
      for (int q = 0; q < parts; ++q) {   // whole rounds of the kernel's ring, but for the last part; at least 5 units (mx_parts)
        MxProblem& part = ps.pr[ps.n++] = p;
        part.first_unit = q * units / parts / 4 * 4;
        part.units = (q + 1 < parts ? (q + 1) * units / parts / 4 * 4 : units) - part.first_unit;
        part.c = sums + static_cast<size_t>(q) * p.m * p.n * sizeof(float);
        part.ldc = p.n, part.alpha = 1.f, part.beta = 0.f, part.out_dtype = CANZ_DT_F32;
      }
      sums += mx_part_bytes(gi.m, gi.n, gi.k);
    }
  }
  return ps.n > 0 ? flush() : CANZ_OK;
}

extern "C" int canz_muon_step_images(const canz_group* g, int32_t n_groups, const canz_muon_hparams* hp, const canz_mx_images* images,
                                     int32_t scale_mode, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace canz;
  if (n_groups < 0 || (n_groups > 0 && (!g || !images))) return fail(CANZ_EINVAL, "bad group array");
  if (!hp) return fail(CANZ_EINVAL, "null hparams");
  if (hp->out_mode != CANZ_OUT_PARAM) return fail(CANZ_EUNSUPPORTED, "images are taken of updated parameters: out_mode must be CANZ_OUT_PARAM");
  if (int rc = check_scale_mode(scale_mode)) return rc;
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  // everything is checked before the step is enqueued; the second time round the images are
  for (int pass = 0; pass < 2; ++pass) {
    for (int i = 0; i < n_groups; ++i) {
      if (!images[i].by_row && !images[i].by_col) continue;
      canz_mx_group m{};
      m.rows = g[i].rows, m.cols = g[i].cols, m.ld = g[i].cols;
      m.n_mats = g[i].n_mats, m.dtype = g[i].out_dtype;
      m.mat = g[i].out, m.by_row = images[i].by_row, m.by_col = images[i].by_col;
      const int rc = pass == 0 ? check_mx_group(m, i, false) : quantize_group(m, scale_mode, st);
      if (rc) return rc;
    }
    if (pass == 1) return CANZ_OK;
    if (int rc = canz_muon_step(g, n_groups, hp, workspace, workspace_bytes, st)) return rc;
  }
  return CANZ_OK;
}
