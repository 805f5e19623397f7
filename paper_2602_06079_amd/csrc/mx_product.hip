// Products of microscaled 4-bit images: C[i][j] = alpha sum_k A[i][k] B[j][k] + beta C[i][j], fp32 sums.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows of either image over 128 k, scales included; a product of two elements is exact
// in fp32.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "device_util.h"
#include "mx.h"

namespace canz {
namespace {

constexpr int THREADS = 256;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

#define CANZ_LDS(p) ((__attribute__((address_space(3))) void*)(p))
#define CANZ_GLB(p) ((const __attribute__((address_space(1))) void*)(p))
#define CANZ_INLINE __attribute__((always_inline))
#define CANZ_FENCE() __builtin_amdgcn_sched_barrier(0)

using Yes = std::true_type;
using No = std::false_type;

template <typename F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for(f, std::make_integer_sequence<int, N>{});
}

// acc[16 slots of p][16 slots of q] += P Q^T over 128 k; SP, SQ: which byte of its scale register belongs to the unit
template <int SP, int SQ>
__device__ __forceinline__ f32x4 mfma(i32x4 p, i32x4 q, f32x4 acc, int scale_p, int scale_q) {
  constexpr int FP4 = 4;   // operand format E2M1: four registers of the eight other formats take
  const i32x8 a = {p[0], p[1], p[2], p[3], 0, 0, 0, 0}, b = {q[0], q[1], q[2], q[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, FP4, FP4, SP, scale_p, SQ, scale_q);
}

// Eight consecutive elements of a row of C, of which `left` are there.
template <typename E>
__device__ __forceinline__ f32x8 load_old(const E* c, int64_t left) {
  f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (left >= 8) {
    typedef E vec __attribute__((ext_vector_type(8), aligned(sizeof(E))));
    const vec x = *reinterpret_cast<const vec*>(c);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x[e]);
  } else {
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {   // a rolled loop: the vector turns instead of being indexed
      const float x = e < left ? static_cast<float>(c[e]) : 0.f;
      v = f32x8{v[1], v[2], v[3], v[4], v[5], v[6], v[7], x};
    }
  }
  return v;
}
template <typename E>
__device__ __forceinline__ void store_eight(E* c, int64_t left, f32x8 v) {
  if (left >= 8) {
    typedef E vec __attribute__((ext_vector_type(8), aligned(sizeof(E))));
    vec x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = static_cast<E>(v[e]);
    *reinterpret_cast<vec*>(c) = x;
  } else {
#pragma unroll 1
    for (int e = 0; e < left; ++e) {
      c[e] = static_cast<E>(v[0]);
      v = f32x8{v[1], v[2], v[3], v[4], v[5], v[6], v[7], 0.f};
    }
  }
}

// ---- one wavefront per 32 x 32 part of C, operands straight from memory: few rows, and k = 0 -------------------------------
constexpr int FEW = 64;   // rows and columns of a block's tile
template <typename E, bool BETA>
__global__ __launch_bounds__(THREADS) void k_mx_product_few(MxProblems ps) {
  int j = 0;
  while (j + 1 < ps.n && static_cast<int>(blockIdx.x) >= ps.pr[j + 1].first_tile) ++j;
  const MxProblem p = ps.pr[j];
  const int tile = blockIdx.x - p.first_tile, tiles_m = static_cast<int>((p.m + FEW - 1) / FEW);
  const int64_t m0 = static_cast<int64_t>(tile % tiles_m) * FEW, n0 = static_cast<int64_t>(tile / tiles_m) * FEW;
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
    i32x4 fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = *reinterpret_cast<const i32x4*>(a + (i * ks + u) * MX_UNIT_BYTES);
      fb[i] = *reinterpret_cast<const i32x4*>(b + (i * ks + u) * MX_UNIT_BYTES);
    }
    // the wavefront's two units are bytes 0 and 1 or 2 and 3 of the scale registers
    const int va = *reinterpret_cast<const int*>(sa + u * MX_SCALE_BYTES) >> (wave >> 1) * 16;
    const int vb = *reinterpret_cast<const int*>(sb + u * MX_SCALE_BYTES) >> (wave & 1) * 16;
    acc[0][0] = mfma<0, 0>(fb[0], fa[0], acc[0][0], vb, va);
    acc[0][1] = mfma<1, 0>(fb[1], fa[0], acc[0][1], vb, va);
    acc[1][0] = mfma<0, 1>(fb[0], fa[1], acc[1][0], vb, va);
    acc[1][1] = mfma<1, 1>(fb[1], fa[1], acc[1][1], vb, va);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t row = row_w + mx_row(i, lane & 15), col = col_w + (lane >> 4) * 8;
    if (row >= p.m || col >= p.n) continue;
    E* const c = static_cast<E*>(p.c) + row * p.ldc + col;
    f32x8 v, old;
    if constexpr (BETA) old = load_old(c, p.n - col);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = p.alpha * acc[i][e >> 2][e & 3];
      if constexpr (BETA) v[e] = __builtin_fmaf(p.beta, old[e], v[e]);
    }
    store_eight(c, p.n - col, v);
  }
}

// ---- tiles through LDS ------------------------------------------------------------------------------------------------------
// A block of four wavefronts (2 x 2) owns a tile of C, 2 W units of A by 2 W of B (W = 8: 256 x 256, W = 4: 128 x 128); a wavefront has
// W x W MFMA tiles.  A stage is one k unit of the tile's units, codes as they lie in the images (a wavefront copies 1 KiB per instruction
// straight into LDS) and scales.
//
// Four stages form a ring over the k units of all tiles of the block, one tile after another without a gap: while unit t is multiplied from
// registers, the operands of t + 1 are read from LDS into a second set, t + 2 and t + 3 are in flight and t + 4 is requested into the stage of
// t, which every wavefront has read before the barrier at the start of the step.  So there is one barrier per k unit, W W MFMAs long.
constexpr int N_XCD = 8;
constexpr int BAND = 4;   // tile rows that are walked column by column

template <int W>
struct Stage {
  static constexpr int codes = 2 * W * MX_UNIT_BYTES;       // of one operand
  static constexpr int scales = 2 * W / 4 * MX_SCALE_BYTES;
  static constexpr int bytes = 2 * (codes + scales);        // A codes, B codes, A scales, B scales
  static constexpr int code_loads = W, scale_loads = W / 4, loads = code_loads + scale_loads;   // of one wavefront
};

// What a block has to do and has to load next: the tiles slot, slot + grid, ...
// The kernel's argument where it lies: scalar loads at any index, and no copy of it.
typedef const __attribute__((address_space(4))) MxProblems* KernArgs;
struct Tile {
  int problem;   // -1: none
  int m0, n0;    // in units of 16 rows
};
template <int W>
__device__ __forceinline__ Tile tile_at(KernArgs ps, int logical) {
  if (logical >= ps->tiles) return Tile{-1, 0, 0};
  int j = 0;
  while (j + 1 < ps->n && logical >= ps->pr[j + 1].first_tile) ++j;
  const int tix = logical - ps->pr[j].first_tile;
  const int tiles_m = static_cast<int>((ps->pr[j].m + 32 * W - 1) / (32 * W)), tiles_n = static_cast<int>((ps->pr[j].n + 32 * W - 1) / (32 * W));
  const int band = tix / (BAND * tiles_n), in_band = tix - band * BAND * tiles_n, rows = min(BAND, tiles_m - band * BAND);
  const int tn = in_band / rows;
  return Tile{j, (band * BAND + in_band - tn * rows) * 2 * W, tn * 2 * W};
}

__device__ __attribute__((aligned(1024))) const uint8_t zero_page[MX_UNIT_BYTES] = {};

template <int W, typename E, bool BETA>
__global__ __launch_bounds__(THREADS, W == 8 ? 1 : 2) void k_mx_product(MxProblems) {
  using S = Stage<W>;
  const KernArgs ps = (KernArgs)__builtin_amdgcn_kernarg_segment_ptr();
  // one array per stage: the compiler then knows that a fetch into one stage does not alias the reads of another
  __shared__ __attribute__((aligned(1024))) uint8_t st0[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st1[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st2[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st3[S::bytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  // the blocks of one XCD (blockIdx % 8) are neighbours in every round, a patch of tiles that share operands in its L2
  int slot;
  {
    const int per = gridDim.x / N_XCD, rem = gridDim.x % N_XCD, xcd = blockIdx.x % N_XCD, q = blockIdx.x / N_XCD;
    slot = xcd < rem ? xcd * (per + 1) + q : rem * (per + 1) + (xcd - rem) * per + q;
  }

  // ---- loading: this wavefront's pieces of the next four stages.  Every tile takes whole rounds of the ring, so its loop has no exit
  // inside and the accumulators stay where they are; units behind the last one are read from a page of zeros.
  int next_logical = slot, load_u = 0, load_ks = 0;
  const uint8_t* src[S::loads];
  auto next_round = [&]() CANZ_INLINE {
    load_u += 4;
    if (load_u < load_ks) return;
    load_u = 0;
    const Tile t = tile_at<W>(ps, next_logical);
    load_ks = 0;
    if (t.problem < 0) return;   // nothing left: zeros
    next_logical += gridDim.x;
    const uint8_t *const a = ps->pr[t.problem].a, *const b = ps->pr[t.problem].b;
    load_ks = static_cast<int>(mx_k_units(ps->pr[t.problem].k));
    const int units_m = static_cast<int>(mx_row_tiles(ps->pr[t.problem].m)), units_n = static_cast<int>(mx_row_tiles(ps->pr[t.problem].n));
    const int64_t row_bytes = static_cast<int64_t>(load_ks) * MX_UNIT_BYTES, scale_bytes = static_cast<int64_t>(load_ks) * MX_SCALE_BYTES;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int piece = wave + 4 * i;   // of 4 W: A's, then B's
      src[i] = piece < 2 * W ? a + min(t.m0 + piece, units_m - 1) * row_bytes : b + min(t.n0 + piece - 2 * W, units_n - 1) * row_bytes;
    }
#pragma unroll
    for (int i = 0; i < S::scale_loads; ++i) {
      const int piece = wave + 4 * i;   // of W
      src[W + i] = piece < W / 2 ? a + units_m * row_bytes + min(t.m0 / 4 + piece, units_m / 4 - 1) * scale_bytes
                                 : b + units_n * row_bytes + min(t.n0 / 4 + piece - W / 2, units_n / 4 - 1) * scale_bytes;
    }
  };
  auto fetch_one = [&](uint8_t* st, int u, auto idx) CANZ_INLINE {
    constexpr int I = decltype(idx)::value;
    const bool there = u < load_ks;
    if constexpr (I < W) {
      const uint8_t* const from = there ? src[I] + static_cast<int64_t>(u) * MX_UNIT_BYTES : zero_page;
      __builtin_amdgcn_global_load_lds(CANZ_GLB(from + lane * 16), CANZ_LDS(st + (wave + 4 * I) * MX_UNIT_BYTES), 16, 0, 0);
    } else {
      const uint8_t* const from = there ? src[I] + static_cast<int64_t>(u) * MX_SCALE_BYTES : zero_page;
      __builtin_amdgcn_global_load_lds(CANZ_GLB(from + lane * 4), CANZ_LDS(st + 2 * S::codes + (wave + 4 * (I - W)) * MX_SCALE_BYTES), 4, 0, 0);
    }
  };

  // ---- operands in registers, two sets: W units of A and of B, and their scales, four units to a register
  i32x4 fa[2][W], fb[2][W];
  int sa[2][W / 4], sb[2][W / 4];
  f32x4 acc[W][W];
  constexpr int READS = 2 * W + W / 2;
  auto read_one = [&](const uint8_t* st, int set, auto idx) CANZ_INLINE {
    constexpr int I = decltype(idx)::value;
    if constexpr (I < W / 4)
      sb[set][I] = *reinterpret_cast<const int*>(st + 2 * S::codes + S::scales + (wn * (W / 4) + I) * MX_SCALE_BYTES + lane * 4);
    else if constexpr (I < W / 2)
      sa[set][I - W / 4] = *reinterpret_cast<const int*>(st + 2 * S::codes + (wm * (W / 4) + I - W / 4) * MX_SCALE_BYTES + lane * 4);
    else if constexpr (I < W / 2 + W)
      fb[set][I - W / 2] = *reinterpret_cast<const i32x4*>(st + S::codes + (wn * W + I - W / 2) * MX_UNIT_BYTES + lane * 16);
    else
      fa[set][I - W / 2 - W] = *reinterpret_cast<const i32x4*>(st + (wm * W + I - W / 2 - W) * MX_UNIT_BYTES + lane * 16);
  };
  // vmcnt(n) lgkmcnt(0)
  constexpr auto wait_code = [](int vm) { return (vm & 15) | 0x70 | (vm >> 4) << 14; };

  // One k unit from register set `set`; `nxt` holds the next one, `cur` (read by everybody at the barrier) takes unit `u` of the next round.
  auto step = [&](auto set_c, uint8_t* cur, const uint8_t* nxt, int u) CANZ_INLINE {
    constexpr int set = decltype(set_c)::value;
    __builtin_amdgcn_s_waitcnt(wait_code(2 * S::loads));
    __builtin_amdgcn_s_barrier();
    CANZ_FENCE();
    static_for<W * W>([&](auto x) CANZ_INLINE {
      constexpr int idx = decltype(x)::value, i = idx / W, j = idx % W;
      acc[i][j] = mfma<j % 4, i % 4>(fb[set][j], fa[set][i], acc[i][j], sb[set][j / 4], sa[set][i / 4]);
      constexpr int PACE = W * W / READS;   // MFMAs per read
      if constexpr (idx % PACE == 0 && idx / PACE < READS) {
        CANZ_FENCE();
        read_one(nxt, set ^ 1, std::integral_constant<int, idx / PACE>{});
        CANZ_FENCE();
      }
      constexpr int LPACE = W * W / S::loads;
      if constexpr (idx % LPACE == LPACE / 2 && idx / LPACE < S::loads) {
        CANZ_FENCE();
        fetch_one(cur, u, std::integral_constant<int, idx / LPACE>{});
        CANZ_FENCE();
      }
    });
  };

  auto store_tile = [&](const Tile& t) CANZ_INLINE {
    int lane = threadIdx.x & 63;   // opaque, or every address that depends on it is kept across the tiles
    asm volatile("" : "+v"(lane));
    const int64_t rows = ps->pr[t.problem].m, ldc = ps->pr[t.problem].ldc;
    const int64_t row0 = (t.m0 + wm * W) * MX_UNIT_ROWS, col0 = (t.n0 + wn * W) * MX_UNIT_ROWS + (lane >> 4) * 8;
    const int64_t left = ps->pr[t.problem].n - col0;   // columns from this lane's first one on
    const float alpha = ps->pr[t.problem].alpha, beta = ps->pr[t.problem].beta;
    E* const c = static_cast<E*>(ps->pr[t.problem].c) + col0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int64_t row = row0 + mx_row(i, lane & 15);
      if (row < rows) {
        E* const at = c + row * ldc;
        f32x8 old[W / 2];
        if constexpr (BETA)
#pragma unroll
          for (int jp = 0; jp < W / 2; ++jp) old[jp] = load_old(at + jp * 32, left - jp * 32);
#pragma unroll
        for (int jp = 0; jp < W / 2; ++jp) {
          f32x8 v;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = alpha * acc[i][2 * jp + (e >> 2)][e & 3];
            if constexpr (BETA) v[e] = __builtin_fmaf(beta, old[jp][e], v[e]);
          }
          store_eight(at + jp * 32, left - jp * 32, v);
        }
      }
      CANZ_FENCE();
    }
  };
  using Set0 = std::integral_constant<int, 0>;
  using Set1 = std::integral_constant<int, 1>;
  next_round();
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st0, load_u, idx); });
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st1, load_u + 1, idx); });
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st2, load_u + 2, idx); });
  static_for<S::loads>([&](auto idx) CANZ_INLINE { fetch_one(st3, load_u + 3, idx); });
  __builtin_amdgcn_s_waitcnt(wait_code(3 * S::loads));
  __builtin_amdgcn_s_barrier();
  CANZ_FENCE();
  static_for<READS>([&](auto idx) CANZ_INLINE { read_one(st0, 0, idx); });

  for (int logical = slot;; logical += gridDim.x) {
    const Tile t = tile_at<W>(ps, logical);
    if (t.problem < 0) break;
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int rounds = static_cast<int>((mx_k_units(ps->pr[t.problem].k) + 3) / 4); rounds > 0; --rounds) {
      next_round();
      step(Set0{}, st0, st1, load_u);
      step(Set1{}, st1, st2, load_u + 1);
      step(Set0{}, st2, st3, load_u + 2);
      step(Set1{}, st3, st0, load_u + 3);
    }
    store_tile(t);
  }
  __builtin_amdgcn_s_waitcnt(wait_code(0));   // the requests behind the last tile have landed before the block leaves
}

// sets first_tile of every problem for square tiles of `edge`; the number of tiles
int64_t count_tiles(MxProblems& ps, int edge) {
  int64_t tiles = 0;
  for (int i = 0; i < ps.n; ++i) {
    ps.pr[i].first_tile = static_cast<int>(tiles);
    tiles += (ps.pr[i].m + edge - 1) / edge * ((ps.pr[i].n + edge - 1) / edge);
  }
  ps.tiles = static_cast<int>(tiles);
  return tiles;
}

constexpr int N_CU = 256;

template <typename E, bool BETA>
hipError_t launch_of(MxProblems& ps, hipStream_t st) {
  // products of few rows (and of none along k) go to the kernel without LDS
  MxProblems few, many;
  few.n = many.n = 0;
  for (int i = 0; i < ps.n; ++i) {
    MxProblems& to = ps.pr[i].k == 0 || ps.pr[i].m <= FEW ? few : many;
    to.pr[to.n++] = ps.pr[i];
  }
  if (few.n > 0) {
    const int64_t tiles = count_tiles(few, FEW);
    k_mx_product_few<E, BETA><<<dim3(static_cast<unsigned>(tiles)), THREADS, 0, st>>>(few);
  }
  if (many.n > 0) {
    const int64_t tiles = count_tiles(many, 256);
    if (tiles >= N_CU / 2) {
      k_mx_product<8, E, BETA><<<dim3(static_cast<unsigned>(std::min<int64_t>(tiles, N_CU))), THREADS, 0, st>>>(many);
    } else {
      const int64_t small = count_tiles(many, 128);
      k_mx_product<4, E, BETA><<<dim3(static_cast<unsigned>(std::min<int64_t>(small, 2 * N_CU))), THREADS, 0, st>>>(many);
    }
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_product(const MxProblems& ps, hipStream_t st) {
  // a launch has one type of result, and reads the old one or not
  for (int kind = 0; kind < 4; ++kind) {
    MxProblems part;
    part.n = 0;
    for (int i = 0; i < ps.n; ++i)
      if ((ps.pr[i].out_dtype == CANZ_DT_F32 ? 0 : 1) + (ps.pr[i].beta != 0.f ? 2 : 0) == kind) part.pr[part.n++] = ps.pr[i];
    if (part.n == 0) continue;
    const hipError_t err = kind == 0   ? launch_of<float, false>(part, st)
                           : kind == 1 ? launch_of<__bf16, false>(part, st)
                           : kind == 2 ? launch_of<float, true>(part, st)
                                       : launch_of<__bf16, true>(part, st);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace canz
