// What goes on beside the products of canz_linear: operands that lie badly are copied, sums of parts joined, the rows of A summed.
#include <algorithm>

#include "linear.h"

namespace canz {
namespace {

// ---- copies ---------------------------------------------------------------------------------------------------------------------
typedef const __attribute__((address_space(4))) LinearCopies* CopyArgs;

// A block has 16 rows of 128 columns.  Memory bounds it: an image of 8192 x 4096 to bf16 21 us (102 MB, 4.9 TB/s).
constexpr int COPY_ROWS = 16, COPY_COLS = 16 * PIECE;
__global__ __launch_bounds__(EACH_THREADS) void k_linear_copy(LinearCopies) {
  const CopyArgs cs = (CopyArgs)__builtin_amdgcn_kernarg_segment_ptr();
  int j = 0;
  while (blockIdx.x >= cs->first_block[j + 1]) ++j;
  const auto& c = cs->cp[j];
  const unsigned slot = blockIdx.x - cs->first_block[j], across = static_cast<unsigned>((c.pitch + COPY_COLS - 1) / COPY_COLS);
  const int64_t row = static_cast<int64_t>(slot / across) * COPY_ROWS + threadIdx.x / 16, col = static_cast<int64_t>(slot % across) * COPY_COLS + threadIdx.x % 16 * PIECE;
  if (row >= c.rows || col >= c.pitch) return;
  bf16x8 v;
  if (c.scales) {
    const int64_t pitch = mx8_pitch(c.cols);
    const Image8 im{const_cast<uint8_t*>(static_cast<const uint8_t*>(c.from)), const_cast<uint8_t*>(c.scales), pitch};
    const f32x8 x = widen(load_raw(im, row, col));
#pragma unroll
    for (int e = 0; e < PIECE; ++e) v[e] = static_cast<__bf16>(col + e < c.cols ? x[e] : 0.f);   // exact but for blocks below 2^-124, which images made elsewhere may have; a NaN block's padding is not NaN
  } else {
    v = load_raw(static_cast<const __bf16*>(c.from) + row * c.ld + col, c.cols - col).v;
  }
  *reinterpret_cast<bf16x8*>(c.to + row * c.pitch + col) = v;
}

// ---- sums of parts of k ---------------------------------------------------------------------------------------------------------
typedef const __attribute__((address_space(4))) LinearJoins* JoinArgs;

// A thread has eight columns of a row, its quad a block of 32; rows that are not there fill up the last block of threads.  Every part's sum goes by once, out of L2 or the cache behind it: five parts of
// 400 x 1536 and eight of 128 x 1536 (19 MB) in 5.5 us.
__global__ __launch_bounds__(EACH_THREADS) void k_linear_join(LinearJoins) {
  const JoinArgs js = (JoinArgs)__builtin_amdgcn_kernarg_segment_ptr();
  int j = 0;
  while (blockIdx.x >= js->first_block[j + 1]) ++j;
  const auto& q = js->jn[j];
  const Spot s = spot(blockIdx.x - js->first_block[j], q.log_tx, q.across);
  const int64_t part_elements = q.m * q.pitch;
  const int parts = q.parts;
  f32x8 z[1] = {f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
  if (s.row < q.m && s.col < q.pitch) {
    const float* const p = q.sums + s.row * q.pitch + s.col;
    Raw<float> part[LINEAR_MAX_PARTS];
#pragma unroll
    for (int i = 0; i < LINEAR_MAX_PARTS; ++i)
      if (i < parts) part[i] = load_raw(p + i * part_elements, PIECE);   // all on their way before the first is added
#pragma unroll
    for (int i = 0; i < LINEAR_MAX_PARTS; ++i)
      if (i < parts) z[0] += part[i].v;
  }
  linear_end<false, 1>(linear_end_of(q.end), s.row, 0, s.col, q.m, q.n, z);
}

// ---- sums of A's rows -----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ f32x8 piece_of(const LinearSums& a, int64_t row, int64_t col) {
  if (a.scales) {
    const Image8 im{const_cast<uint8_t*>(static_cast<const uint8_t*>(a.from)), const_cast<uint8_t*>(a.scales), mx8_pitch(a.cols)};
    f32x8 v = widen(load_raw(im, row, col));
#pragma unroll
    for (int e = 0; e < PIECE; ++e) v[e] = col + e < a.cols ? v[e] : 0.f;
    return v;
  }
  return widen(load_raw(static_cast<const __bf16*>(a.from) + row * a.ld + col, a.cols - col));
}

// Along k: a wavefront to a row; every element goes by once.
__global__ __launch_bounds__(EACH_THREADS) void k_linear_row_sums(LinearSums a) {
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  f32x8 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int64_t col = static_cast<int64_t>(threadIdx.x & 63) * PIECE; col < a.cols; col += 64 * PIECE) s += piece_of(a, row, col);
  const float t = wave_sum(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
  if ((threadIdx.x & 63) == 0) a.sums[row] = a.beta != 0.f ? __builtin_fmaf(a.beta, a.sums[row], a.alpha * t) : a.alpha * t;
}

// Across k: a block has 512 columns (64 pieces) of a group of rows, of which its four wavefronts take one each by turns, eight of them on their way at a time; the groups' sums are added up by
// k_linear_join_sums.  8192 x 12288 takes 55 us (201 MB, 3.7 TB/s) and 5 for the join behind a product; by themselves one after another 41 together.
__global__ __launch_bounds__(EACH_THREADS) void k_linear_column_sums(LinearSums a, int across) {
  __shared__ f32x8 part[3][64];
  const unsigned group = blockIdx.x / static_cast<unsigned>(across), along = blockIdx.x - group * across;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t groups = linear_sum_groups(a.rows), col = (static_cast<int64_t>(along) * 64 + lane) * PIECE, step = 4 * groups;
  f32x8 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (col < a.cols) {
    int64_t row = group + wave * groups;
    if (!a.scales && col + PIECE <= a.cols) {
      constexpr int AHEAD = 8;
      const __bf16* p = static_cast<const __bf16*>(a.from) + row * a.ld + col;
      for (; row + (AHEAD - 1) * step < a.rows; row += AHEAD * step, p += AHEAD * step * a.ld) {
        Raw<__bf16> v[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) v[i] = load_raw(p + i * step * a.ld, PIECE);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) s += widen(v[i]);
      }
    }
    for (; row < a.rows; row += step) s += piece_of(a, row, col);
  }
  if (wave > 0) part[wave - 1][lane] = s;
  __syncthreads();
  if (wave > 0 || col >= a.cols) return;
  s = (s + part[0][lane]) + (part[1][lane] + part[2][lane]);
  store_piece8(a.partial + group * mx8_pitch(a.cols) + col, PIECE, s);
}
constexpr int JOIN = 32;
__global__ __launch_bounds__(JOIN * 8) void k_linear_join_sums(LinearSums a) {
  __shared__ float part[8][JOIN];
  const int tx = threadIdx.x & (JOIN - 1), ty = threadIdx.x / JOIN;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * JOIN + tx, groups = linear_sum_groups(a.rows), pitch = mx8_pitch(a.cols);
  float s = 0.f;
  if (col < a.cols) {
#pragma unroll 8
    for (int64_t g = ty; g < groups; g += 8) s += a.partial[g * pitch + col];
  }
  part[ty][tx] = s;
  __syncthreads();
  if (ty != 0 || col >= a.cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += part[i][tx];
  a.sums[col] = a.beta != 0.f ? __builtin_fmaf(a.beta, a.sums[col], a.alpha * s) : a.alpha * s;
}

}  // namespace

hipError_t launch_linear_copies(LinearCopies& cs, hipStream_t st) {
  int64_t blocks = 0;
  LinearCopies rest;
  rest.n = 0;
  for (int i = 0; i < cs.n; ++i) {
    const int64_t each = (cs.cp[i].rows + COPY_ROWS - 1) / COPY_ROWS * ((cs.cp[i].pitch + COPY_COLS - 1) / COPY_COLS);
    if (blocks + each > MOST_BLOCKS) {
      rest.n = cs.n - i, cs.n = i;
      std::copy_n(cs.cp + i, rest.n, rest.cp);
      break;
    }
    cs.first_block[i] = static_cast<unsigned>(blocks);
    blocks += each;
  }
  cs.first_block[cs.n] = static_cast<unsigned>(blocks);
  k_linear_copy<<<dim3(static_cast<unsigned>(blocks)), EACH_THREADS, 0, st>>>(cs);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess && rest.n > 0 ? launch_linear_copies(rest, st) : err;
}

hipError_t launch_linear_joins(LinearJoins& js, hipStream_t st) {
  int64_t blocks = 0;
  LinearJoins rest;
  rest.n = 0;
  for (int i = 0; i < js.n; ++i) {
    const Cover c = cover(js.jn[i].m, js.jn[i].n);
    if (blocks + c.blocks > MOST_BLOCKS) {
      rest.n = js.n - i, js.n = i;
      std::copy_n(js.jn + i, rest.n, rest.jn);
      break;
    }
    js.jn[i].log_tx = c.log_tx, js.jn[i].across = c.across;
    js.first_block[i] = static_cast<unsigned>(blocks);
    blocks += c.blocks;
  }
  js.first_block[js.n] = static_cast<unsigned>(blocks);
  k_linear_join<<<dim3(static_cast<unsigned>(blocks)), EACH_THREADS, 0, st>>>(js);
  const hipError_t err = hipGetLastError();
  return err == hipSuccess && rest.n > 0 ? launch_linear_joins(rest, st) : err;
}

hipError_t launch_linear_sums(const LinearSums& s, hipStream_t st) {
  if (!s.trans) {
    k_linear_row_sums<<<dim3(static_cast<unsigned>((s.rows + 3) / 4)), EACH_THREADS, 0, st>>>(s);
  } else {
    const int across = static_cast<int>((s.cols + 64 * PIECE - 1) / (64 * PIECE));
    const int64_t groups = linear_sum_groups(s.rows);
    if (groups > 0) k_linear_column_sums<<<dim3(static_cast<unsigned>(groups * across)), EACH_THREADS, 0, st>>>(s, across);
    k_linear_join_sums<<<dim3(static_cast<unsigned>((s.cols + JOIN - 1) / JOIN)), JOIN * 8, 0, st>>>(s);
  }
  return hipGetLastError();
}

}  // namespace canz
