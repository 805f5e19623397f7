// canz_mx_eight_store and canz_mx_eight_load: matrices to 8-bit images and back (layout and rounding: mx8.h).
#include "canz_internal.h"
#include "mx8.h"

namespace canz {

int check_extents(const char* what, int idx, int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return fail(CANZ_EINVAL, "%s %d: negative extent", what, idx);
  if (rows > MX_MAX_EXTENT || cols > MX_MAX_EXTENT) return fail(CANZ_ESHAPE, "%s %d: extent above %lld", what, idx, static_cast<long long>(MX_MAX_EXTENT));
  if (!fits_launch(rows, cols)) return fail(CANZ_ESHAPE, "%s %d: more than 2^34 padded elements in a matrix", what, idx);
  return CANZ_OK;
}

namespace {

// A thread takes a piece of one row, its quad the block that shares a scale.  Every element goes by once, so memory is what bounds them.  us for 8192 x 5120, 1 / 2 / 4 / 8 rows of a thread with their
// loads in flight together: fp32 to an image 47.4 / 49.1 / 50.5 / 53.1 (211 MB, 4.5 TB/s), back 40.6 / 41.8 / 45.4 / 47.4 (5.2 TB/s).  Many wavefronts with little to do each keep more on its way than
// few with much.
template <typename E>
__global__ __launch_bounds__(EACH_THREADS) void k_mx8_store(const E* mat, int64_t ld, Image8 image, int64_t rows, int64_t cols, int log_tx, int across) {
  const Spot s = spot(blockIdx.x, log_tx, across);
  if (s.row >= rows) return;   // a row's quads are whole
  store_codes(image, s.row, s.col, cols, round8(widen(load_raw(mat + s.row * ld + s.col, cols - s.col))));
}

template <typename E>
__global__ __launch_bounds__(EACH_THREADS) void k_mx8_load(E* mat, int64_t ld, Image8 image, int64_t rows, int64_t cols, int log_tx, int across) {
  const Spot s = spot(blockIdx.x, log_tx, across);
  if (s.row < rows && s.col < cols) store_piece8(mat + s.row * ld + s.col, cols - s.col, widen(load_raw(image, s.row, s.col)));
}

int check_group(const canz_mx8_group& g, int idx) {
  if (g.n_mats < 0) return fail(CANZ_EINVAL, "group %d: n_mats < 0", idx);
  if (int rc = check_extents("group", idx, g.rows, g.cols)) return rc;
  if (!float_dtype(g.dtype)) return fail(CANZ_EUNSUPPORTED, "group %d: unknown dtype", idx);
  if (g.ld < g.cols) return fail(CANZ_EINVAL, "group %d: ld below cols", idx);
  if (g.n_mats == 0 || g.rows == 0 || g.cols == 0) return CANZ_OK;
  if (!g.mat || !g.image) return fail(CANZ_EINVAL, "group %d: null pointer table", idx);
  for (int i = 0; i < g.n_mats; ++i) {
    if (!g.mat[i] || misaligned(g.mat[i], element_bytes(g.dtype))) return fail(CANZ_EINVAL, "group %d: mat[%d] null or not aligned to its elements", idx, i);
    if (!g.image[i] || misaligned(g.image[i], 256)) return fail(CANZ_EINVAL, "group %d: image[%d] null or not 256-byte aligned", idx, i);
  }
  return CANZ_OK;
}

template <typename E>
void launch(const canz_mx8_group& g, bool back, hipStream_t st) {
  const Cover c = cover(g.rows, g.cols);
  for (int i = 0; i < g.n_mats; ++i) {
    const Image8 image = image8(g.image[i], g.rows, g.cols);
    E* const mat = static_cast<E*>(g.mat[i]);
    const dim3 grid(static_cast<unsigned>(c.blocks));
    if (back)
      k_mx8_load<<<grid, EACH_THREADS, 0, st>>>(mat, g.ld, image, g.rows, g.cols, c.log_tx, c.across);
    else
      k_mx8_store<<<grid, EACH_THREADS, 0, st>>>(static_cast<const E*>(mat), g.ld, image, g.rows, g.cols, c.log_tx, c.across);
  }
}

int run(const canz_mx8_group* g, int32_t n_groups, bool back, void* hip_stream) {
  if (n_groups < 0 || (n_groups > 0 && !g)) return fail(CANZ_EINVAL, "bad group array");
  for (int i = 0; i < n_groups; ++i)
    if (int rc = check_group(g[i], i)) return rc;
  const hipStream_t st = stream_of(hip_stream);
  const StreamDevice on(st);
  if (on.error() != hipSuccess) return fail(CANZ_EHIP, "stream: %s", hipGetErrorString(on.error()));
  for (int i = 0; i < n_groups; ++i) {
    if (g[i].n_mats == 0 || g[i].rows == 0 || g[i].cols == 0) continue;
    if (g[i].dtype == CANZ_DT_F32)
      launch<float>(g[i], back, st);
    else
      launch<__bf16>(g[i], back, st);
    if (const hipError_t err = hipGetLastError(); err != hipSuccess) return fail(CANZ_EHIP, "8-bit image: %s", hipGetErrorString(err));
  }
  return CANZ_OK;
}

}  // namespace
}  // namespace canz

extern "C" int canz_mx_eight_bytes(int64_t rows, int64_t cols, size_t* bytes_out) {
  using namespace canz;
  if (!bytes_out) return fail(CANZ_EINVAL, "null output pointer");
  if (rows < 0 || cols < 0) return fail(CANZ_EINVAL, "negative extent");
  if (rows > MX_MAX_EXTENT || cols > MX_MAX_EXTENT) return fail(CANZ_ESHAPE, "extent above %lld", static_cast<long long>(MX_MAX_EXTENT));
  *bytes_out = static_cast<size_t>(mx8_bytes(rows, cols));
  return CANZ_OK;
}

extern "C" int canz_mx_eight_store(const canz_mx8_group* g, int32_t n_groups, void* hip_stream) { return canz::run(g, n_groups, false, hip_stream); }
extern "C" int canz_mx_eight_load(const canz_mx8_group* g, int32_t n_groups, void* hip_stream) { return canz::run(g, n_groups, true, hip_stream); }
