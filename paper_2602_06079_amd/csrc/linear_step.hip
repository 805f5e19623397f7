// canz_linear: host side.  Validates the groups, places operand copies and sums in the workspace and enqueues the launches on the caller's stream; nothing here allocates, copies to the
// device or synchronises.
#include <algorithm>

#include "canz_internal.h"
#include "linear.h"

namespace canz {
namespace {

constexpr size_t ALIGN = 256;
size_t aligned(size_t bytes) { return (bytes + ALIGN - 1) / ALIGN * ALIGN; }

bool idle(const canz_linear_group& g) { return g.n_prods == 0 || g.m == 0 || g.n == 0; }
bool sums_asked(const canz_linear_group& g) { return g.a_sums != nullptr && g.n_prods > 0 && g.m > 0; }

// One operand as it is stored.
struct Stored {
  int64_t rows, cols, ld;
  int dtype;
};
Stored stored_a(const canz_linear_group& g) { return g.a_trans ? Stored{g.k, g.m, g.lda, g.a_dtype} : Stored{g.m, g.k, g.lda, g.a_dtype}; }
Stored stored_b(const canz_linear_group& g) { return g.b_trans ? Stored{g.k, g.n, g.ldb, g.b_dtype} : Stored{g.n, g.k, g.ldb, g.b_dtype}; }

int check_group(const canz_linear_group& g, int idx, bool need_ptrs) {
  if (g.n_prods < 0) return fail(CANZ_EINVAL, "group %d: n_prods < 0", idx);
  if (g.m < 0 || g.n < 0 || g.k < 0) return fail(CANZ_EINVAL, "group %d: negative extent", idx);
  if (g.m > LINEAR_MAX_EXTENT || g.n > LINEAR_MAX_EXTENT || g.k > LINEAR_MAX_EXTENT)
    return fail(CANZ_ESHAPE, "group %d: extent above %lld", idx, static_cast<long long>(LINEAR_MAX_EXTENT));
  if (!fits_launch(g.m, g.n) || !fits_launch(g.m, g.k) || !fits_launch(g.n, g.k))
    return fail(CANZ_ESHAPE, "group %d: more than 2^34 padded elements in a matrix", idx);
  for (int32_t t : {g.a_dtype, g.b_dtype})
    if (t != CANZ_DT_BF16 && t != CANZ_DT_MX8) return fail(CANZ_EUNSUPPORTED, "group %d: an operand's dtype is neither CANZ_DT_BF16 nor CANZ_DT_MX8", idx);
  if (!float_dtype(g.out_dtype) || !float_dtype(g.bias_dtype)) return fail(CANZ_EUNSUPPORTED, "group %d: unknown out_dtype or bias_dtype", idx);
  if (!act_known(g.act)) return fail(CANZ_EUNSUPPORTED, "group %d: unknown act %d", idx, g.act);
  if ((g.a_trans & ~1) || (g.b_trans & ~1)) return fail(CANZ_EINVAL, "group %d: a_trans and b_trans are 0 or 1", idx);
  if (g.a_dtype == CANZ_DT_BF16 && g.lda < stored_a(g).cols) return fail(CANZ_EINVAL, "group %d: lda below a stored row of A", idx);
  if (g.b_dtype == CANZ_DT_BF16 && g.ldb < stored_b(g).cols) return fail(CANZ_EINVAL, "group %d: ldb below a stored row of B", idx);
  if (g.ldc < g.n) return fail(CANZ_EINVAL, "group %d: ldc below n", idx);
  if (!need_ptrs) return CANZ_OK;
  auto bad = [](const void* p, uintptr_t align) { return p == nullptr || misaligned(p, align); };
  const uintptr_t a_el = g.a_dtype == CANZ_DT_MX8 ? 256 : 2, b_el = g.b_dtype == CANZ_DT_MX8 ? 256 : 2, out = element_bytes(g.out_dtype);
  if (sums_asked(g)) {
    if (g.k > 0 && !g.a) return fail(CANZ_EINVAL, "group %d: null pointer table", idx);
    for (int i = 0; i < g.n_prods; ++i) {
      if (bad(g.a_sums[i], 4)) return fail(CANZ_EINVAL, "group %d: a_sums[%d] null or not aligned to its elements", idx, i);
      if (g.k > 0 && bad(g.a[i], a_el)) return fail(CANZ_EINVAL, "group %d: a[%d] null or not %d-byte aligned", idx, i, static_cast<int>(a_el));
    }
  }
  if (idle(g)) return CANZ_OK;
  if (!g.c || (g.k > 0 && (!g.a || !g.b))) return fail(CANZ_EINVAL, "group %d: null pointer table", idx);
  if (g.residual && g.ldr < g.n) return fail(CANZ_EINVAL, "group %d: ldr below n", idx);
  for (int i = 0; i < g.n_prods; ++i) {
    if (bad(g.c[i], out)) return fail(CANZ_EINVAL, "group %d: c[%d] null or not aligned to its elements", idx, i);
    if (g.residual && bad(g.residual[i], out)) return fail(CANZ_EINVAL, "group %d: residual[%d] null or not aligned to its elements", idx, i);
    if (g.residual && g.residual[i] == g.c[i] && g.ldr != g.ldc) return fail(CANZ_EINVAL, "group %d: residual[%d] is C with another row distance", idx, i);
    if (g.bias && bad(g.bias[i], element_bytes(g.bias_dtype))) return fail(CANZ_EINVAL, "group %d: bias[%d] null or not aligned to its elements", idx, i);
    if (g.pre8 && bad(g.pre8[i], 256)) return fail(CANZ_EINVAL, "group %d: pre8[%d] null or not 256-byte aligned", idx, i);
    if (g.k == 0) continue;
    if (bad(g.a[i], a_el)) return fail(CANZ_EINVAL, "group %d: a[%d] null or not %d-byte aligned", idx, i, static_cast<int>(a_el));
    if (bad(g.b[i], b_el)) return fail(CANZ_EINVAL, "group %d: b[%d] null or not %d-byte aligned", idx, i, static_cast<int>(b_el));
  }
  return CANZ_OK;
}

// Whether the tile kernels take an operand where it lies; otherwise they take a copy, whose rows are this long.
bool lies_well(const Stored& s, const void* at) {
  return s.dtype == CANZ_DT_BF16 && s.cols % 8 == 0 && s.ld % 8 == 0 && s.ld <= LINEAR_MAX_EXTENT && !misaligned(at, 16);
}
int64_t copy_pitch(const Stored& s) { return (s.cols + 63) / 64 * 64; }
size_t copy_bytes(const Stored& s) { return aligned(static_cast<size_t>(s.rows) * copy_pitch(s) * 2); }

// The kernel for few rows reads A in bf16 or as an image, and B in bf16, wherever they lie.
bool runs_few(const canz_linear_group& g) { return linear_few(g.m, g.a_trans, g.b_trans); }
bool copies_a(const canz_linear_group& g, const void* at) { return g.k > 0 && !runs_few(g) && !lies_well(stored_a(g), at); }
bool copies_b(const canz_linear_group& g, const void* at) { return g.k > 0 && (runs_few(g) ? g.b_dtype == CANZ_DT_MX8 : !lies_well(stored_b(g), at)); }
int parts_of(const canz_linear_group& g) { return runs_few(g) ? 1 : linear_parts(g.m, g.n, g.k); }
int64_t sum_pitch(int64_t n) { return (n + PIECE - 1) / PIECE * PIECE; }
size_t part_bytes(const canz_linear_group& g) {
  const int parts = parts_of(g);
  return parts > 1 ? aligned(static_cast<size_t>(parts) * g.m * sum_pitch(g.n) * sizeof(float)) : 0;
}
size_t column_sum_bytes(const canz_linear_group& g) {
  return sums_asked(g) && g.a_trans ? aligned(static_cast<size_t>(linear_sum_groups(g.k)) * mx8_pitch(g.m) * sizeof(float)) : 0;
}

// Pointers that are not given lie badly.
int workspace_of(const canz_linear_group* g, int32_t n_groups, size_t* bytes_out) {
  constexpr uintptr_t BADLY = 2;
  size_t need = 0;
  auto add = [&](size_t bytes) { return __builtin_add_overflow(need, bytes, &need); };
  for (int i = 0; i < n_groups; ++i) {
    const canz_linear_group& x = g[i];
    size_t each = column_sum_bytes(x), total = 0;
    if (!idle(x)) each += part_bytes(x);
    bool over = __builtin_mul_overflow(each, static_cast<size_t>(x.n_prods), &total) || add(total);
    if (!idle(x)) {
      const size_t a = copy_bytes(stored_a(x)), b = copy_bytes(stored_b(x));
      const void* const bad = reinterpret_cast<const void*>(BADLY);
      if (!x.a && copies_a(x, bad)) over = over || __builtin_mul_overflow(a, static_cast<size_t>(x.n_prods), &total) || add(total);
      if (!x.b && copies_b(x, bad)) over = over || __builtin_mul_overflow(b, static_cast<size_t>(x.n_prods), &total) || add(total);
      for (int q = 0; q < x.n_prods && (x.a || x.b) && !over; ++q) {
        if (x.a && copies_a(x, x.a[q])) over = over || add(a);
        if (x.b && copies_b(x, x.b[q])) over = over || add(b);
      }
    }
    if (over) return fail(CANZ_ESHAPE, "group %d: the workspace would have more bytes than 64 bits count", i);
  }
  *bytes_out = std::max(need, ALIGN);
  return CANZ_OK;
}

// The launches that a product with a k may be part of.
enum Kind { TILES, FEW = TILES + 4, KINDS = FEW + 6 };
int kind_of(const canz_linear_group& g) {
  if (!runs_few(g)) return TILES + 2 * g.a_trans + g.b_trans;
  return FEW + (g.a_dtype == CANZ_DT_MX8 ? 3 : 0) + linear_few_width(g.n, g.pre8 != nullptr);
}

int hip_failed(hipError_t err) { return err == hipSuccess ? CANZ_OK : fail(CANZ_EHIP, "linear: %s", hipGetErrorString(err)); }

// Problems wait here until their launch is full.
class Launches {
 public:
  explicit Launches(hipStream_t st) : st_(st) {
    for (auto& ps : waiting_) ps.n = 0;
    joins_.n = 0;
  }
  int add(int kind, const LinearProblem& p) {
    LinearProblems& ps = waiting_[kind];
    ps.pr[ps.n++] = p;
    return ps.n == LINEAR_PROBLEMS ? flush(kind) : CANZ_OK;
  }
  // behind the products that have been added
  int join(const LinearProblem& p, const float* sums, int64_t pitch, int parts) {
    joins_.jn[joins_.n++] = LinearJoin{p.end, p.m, p.n, pitch, sums, parts, 0, 0};
    return joins_.n == LINEAR_JOINS ? flush() : CANZ_OK;
  }
  int flush() {
    for (int kind = 0; kind < KINDS; ++kind)
      if (int rc = flush(kind)) return rc;
    const int rc = joins_.n > 0 ? hip_failed(launch_linear_joins(joins_, st_)) : CANZ_OK;
    joins_.n = 0;
    return rc;
  }

 private:
  int flush(int kind) {
    LinearProblems& ps = waiting_[kind];
    if (ps.n == 0) return CANZ_OK;
    const hipError_t err = kind >= FEW ? launch_linear_few(ps, st_) : launch_linear_tiles(ps, (kind - TILES) & 2, (kind - TILES) & 1, st_);
    ps.n = 0;
    return hip_failed(err);
  }
  hipStream_t st_;
  LinearProblems waiting_[KINDS];
  LinearJoins joins_;
};

int run(const canz_linear_group* g, int32_t n_groups, uint8_t* ws, hipStream_t st) {
  // copies of operands that lie badly; every product's place is found again below in the same order
  size_t at = 0;
  {
    LinearCopies cs;
    cs.n = 0;
    auto flush = [&]() -> int {
      const int rc = cs.n > 0 ? hip_failed(launch_linear_copies(cs, st)) : CANZ_OK;
      cs.n = 0;
      return rc;
    };
    auto copy = [&](const Stored& s, const void* from) -> int {
      const bool image = s.dtype == CANZ_DT_MX8;
      const Image8 im = image8(from, s.rows, s.cols);
      cs.cp[cs.n++] = LinearCopy{from, image ? im.scales : nullptr, reinterpret_cast<__bf16*>(ws + at), s.rows, s.cols, s.ld, copy_pitch(s)};
      at += copy_bytes(s);
      return cs.n == LINEAR_COPIES ? flush() : CANZ_OK;
    };
    for (int i = 0; i < n_groups; ++i) {
      if (idle(g[i]) || g[i].k == 0) continue;
      for (int q = 0; q < g[i].n_prods; ++q) {
        if (copies_a(g[i], g[i].a[q]))
          if (int rc = copy(stored_a(g[i]), g[i].a[q])) return rc;
        if (copies_b(g[i], g[i].b[q]))
          if (int rc = copy(stored_b(g[i]), g[i].b[q])) return rc;
      }
    }
    if (int rc = flush()) return rc;
  }
  const uint8_t* copies = ws;
  Launches launches(st);
  for (int i = 0; i < n_groups; ++i) {
    const canz_linear_group& x = g[i];
    for (int q = 0; q < x.n_prods; ++q) {
      if (sums_asked(x)) {
        const Stored s = stored_a(x);
        const bool image = s.dtype == CANZ_DT_MX8;
        const LinearSums sums{x.k > 0 ? x.a[q] : nullptr, image && x.k > 0 ? image8(x.a[q], s.rows, s.cols).scales : nullptr, s.rows, s.cols, s.ld, x.a_trans, x.alpha,
                              x.beta, reinterpret_cast<float*>(ws + at), static_cast<float*>(x.a_sums[q])};
        at += column_sum_bytes(x);
        if (int rc = hip_failed(launch_linear_sums(sums, st))) return rc;
      }
      if (idle(x)) continue;
      LinearProblem p{};
      p.m = x.m, p.n = x.n, p.k = x.k;
      p.end = LinearEnd{x.c[q], x.residual ? x.residual[q] : x.c[q], x.bias ? x.bias[q] : nullptr, image8(x.pre8 ? x.pre8[q] : nullptr, x.m, x.n), x.ldc,
                        x.residual ? x.ldr : x.ldc, x.alpha, x.beta, x.act, x.out_dtype == CANZ_DT_F32, x.bias_dtype == CANZ_DT_F32};
      if (x.k == 0) {
        if (int rc = launches.join(p, nullptr, sum_pitch(x.n), 0)) return rc;
        continue;
      }
      const bool few = runs_few(x);
      auto place = [&](const Stored& s, const void* from, bool copied, const void*& to, int64_t& ld, int& k, bool trans) {
        to = copied ? copies : from;
        ld = copied ? copy_pitch(s) : s.ld;
        if (copied) copies += copy_bytes(s);
        k = static_cast<int>(copied && !trans ? ld : x.k);
      };
      const Stored a = stored_a(x), b = stored_b(x);
      place(a, x.a[q], copies_a(x, x.a[q]), p.a, p.lda, p.k_a, x.a_trans);
      place(b, x.b[q], copies_b(x, x.b[q]), p.b, p.ldb, p.k_b, x.b_trans);
      if (few && x.a_dtype == CANZ_DT_MX8) {
        const Image8 im = image8(x.a[q], a.rows, a.cols);
        p.a_scales = im.scales, p.lda = im.pitch;
      }
      const int steps = static_cast<int>((x.k + LINEAR_K - 1) / LINEAR_K), parts = parts_of(x), kind = kind_of(x);
      if (parts == 1) {
        p.steps = steps;
        if (int rc = launches.add(kind, p)) return rc;
        continue;
      }
      float* const sums = reinterpret_cast<float*>(ws + at);
      at += part_bytes(x);
      const int64_t pitch = sum_pitch(x.n);
      LinearProblem part = p;
      for (int z = 0; z < parts; ++z) {   // whole rounds of the kernel's ring, but for the last part
        part.first_step = static_cast<int>(static_cast<int64_t>(z) * steps / parts / 4 * 4);
        part.steps = (z + 1 < parts ? static_cast<int>(static_cast<int64_t>(z + 1) * steps / parts / 4 * 4) : steps) - part.first_step;
        part.end = LinearEnd{sums + z * x.m * pitch, nullptr, nullptr, Image8{nullptr, nullptr, 0}, pitch, pitch, 1.f, 0.f, CANZ_ACT_NONE, 1, 1};
        if (int rc = launches.add(kind, part)) return rc;
      }
      if (int rc = launches.join(p, sums, pitch, parts)) return rc;
    }
  }
  return launches.flush();
}

}  // namespace
}  // namespace canz

extern "C" int canz_linear_workspace_bytes(const canz_linear_group* g, int32_t n_groups, size_t* bytes_out) {
  using namespace canz;
  if (!bytes_out) return fail(CANZ_EINVAL, "null output pointer");
  if (n_groups < 0 || (n_groups > 0 && !g)) return fail(CANZ_EINVAL, "bad group array");
  for (int i = 0; i < n_groups; ++i)
    if (int rc = check_group(g[i], i, false)) return rc;
  return workspace_of(g, n_groups, bytes_out);
}

extern "C" int canz_linear(const canz_linear_group* g, int32_t n_groups, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace canz;
  if (n_groups < 0 || (n_groups > 0 && !g)) return fail(CANZ_EINVAL, "bad group array");
  bool any = false;
  for (int i = 0; i < n_groups; ++i) {
    if (int rc = check_group(g[i], i, true)) return rc;
    any = any || !idle(g[i]) || sums_asked(g[i]);
  }
  if (!any) return CANZ_OK;
  if (!workspace || misaligned(workspace, ALIGN)) return fail(CANZ_EWORKSPACE, "workspace null or not 256-byte aligned");
  size_t need = 0;
  if (int rc = workspace_of(g, n_groups, &need)) return rc;
  if (workspace_bytes < need) return fail(CANZ_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  return run(g, n_groups, static_cast<uint8_t*>(workspace), st);
}
