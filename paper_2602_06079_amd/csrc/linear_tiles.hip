// Products of bf16 matrices by tiles through LDS (canz_linear): z = A B^T with either operand stored along k or across it.
//
// A block of four wavefronts (2 x 2) owns a tile of C, 64 W rows by 64 W columns (W = 4: 256 x 256, W = 2: 128 x 128); a wavefront has 2 W x 2 W tiles of
// v_mfma_f32_16x16x32_bf16.  256 x 256 is what the accumulators allow (256 of a wavefront's 512 registers), and the larger the tile the fewer bytes go from L2 into LDS and from there into
// registers for an operation.  What bounds long products is power, and from registers alone, on normal random operands, these instructions reach 2060 TFLOP/s where the 32 x 32 x 16 ones
// reach 1800.
//
// A stage holds 64 k of the tile's rows of A and of B, copied straight into LDS (a wavefront instruction moves 1 KiB; every lane names its own 16 bytes in memory, so the order in LDS is free,
// and 64 k are a whole line of a row that lies along k).  Two stages (or four) are filled by turns, over the steps of all tiles of the block, one tile after another without a gap.  A stage is two
// steps of 32 k: while a step is multiplied from registers, the operands of the next one are read from LDS, B's into a second set, each of A's behind the row of tiles that it was for.  So during a
// stage's first step its second half is read, and behind the barrier that follows nobody needs it any more: in its second step it takes the stage after the next, which has 1.5 steps to arrive,
// while the next one's operands are read.  One wavefront to a SIMD issues an instruction every four cycles and a matrix instruction takes 16, so what goes on beside them has to be few instructions.
//
// Order in LDS, so that reads have no bank conflicts:
//   along k    rows of 64 k (128 bytes), their eight 16-byte chunks turned by row % 8: ds_read_b128 takes 8 k of a row
//   across k   rows of k (64 W rows of the matrix side by side, 128 W bytes), their 64-byte pieces turned by k % 4 and the halves of these by (k / 8) % 2: ds_read_b64_tr_b16 takes 4 k of
//              16 rows, and hands each lane the 4 k of one row
#include <algorithm>
#include <type_traits>
#include <utility>

#include "linear.h"

namespace canz {
namespace {

constexpr int THREADS = 256;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define CANZ_LDS(p) ((__attribute__((address_space(3))) void*)(p))
#define CANZ_INLINE __attribute__((always_inline))
#define CANZ_FENCE() __builtin_amdgcn_sched_barrier(0)

template <typename F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for(f, std::make_integer_sequence<int, N>{});
}

// 16 bytes a lane from base + lane_off + off + IMM straight into LDS at lds + IMM, lane after lane; zeros for lanes whose lane_off + IMM is `room` or more.
template <int IMM>
__device__ __forceinline__ void buffer_to_lds(const uint8_t* base, unsigned room, uint8_t* lds, unsigned lane_off, unsigned off) {
#if defined(__HIP_DEVICE_COMPILE__)   // the descriptor's type is the device's only
  constexpr int RAW = 0x00027000;     // a raw buffer of dwords
  const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), static_cast<short>(0), static_cast<int>(room), RAW);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, CANZ_LDS(lds), 16, static_cast<int>(lane_off), static_cast<int>(off), IMM, 0);
#endif
}
// Operands begin SHIFT bytes behind the buffer's base, so that what IMM adds can be taken from every lane's offset.
// Along k the descriptor's size only tells NOTHING from an offset: 255 rows of 2^22 elements, all of k and SHIFT stay below it.
constexpr unsigned SHIFT = 4096, ROOM = 0x7FFFF000u, NOTHING = 0x7FFFF800u;

constexpr int STAGE_K = 2 * LINEAR_K;
template <int W>
struct Stage {
  static constexpr int side = 64 * W;                 // rows of an operand
  static constexpr int operand = side * STAGE_K * 2;  // bytes
  static constexpr int bytes = 2 * operand;
  static constexpr int loads = 2 * W;                 // of one wavefront, for one operand
};

// What a block has to do and has to load next: of the launch's tiles those numbered blockIdx.x, blockIdx.x + gridDim.x, ... (tile_at)
struct Tile {
  int problem;   // NONE: there is none; OUTSIDE: a quarter of a tile that lies outside of C
  int m0, n0;
};
constexpr int NONE = -1, OUTSIDE = -2;
// Number `logical` of the launch's tiles.  Every XCD (blockIdx % 8, and logical % 8, since a grid has a multiple of 8 blocks) has an eighth of each product, in one piece: what its blocks
// work on at a time is a patch of neighbours that share operands in its L2.
constexpr int N_XCD = 8, BAND = 4;   // tile rows that are walked column by column
template <int W>
__device__ __forceinline__ Tile tile_at(LinearArgs ps, int logical) {
  const int xcd = logical % N_XCD;
  int q = logical / N_XCD, quarter = 0, side = 64 * W;
  if (W == 2 && ps->quarters) quarter = q & 3, q >>= 2, side = 256;
  q += ps->from;
  if (q >= ps->to) return Tile{NONE, 0, 0};
  for (int j = 0; j < ps->n; ++j) {
    const int tiles = ps->first_tile[j + 1] - ps->first_tile[j];
    const int begin = static_cast<int>(static_cast<int64_t>(tiles) * xcd / N_XCD), count = static_cast<int>(static_cast<int64_t>(tiles) * (xcd + 1) / N_XCD) - begin;
    if (q >= count) {
      q -= count;
      continue;
    }
    const int tix = begin + q;
    const int tiles_m = static_cast<int>((ps->pr[j].m + side - 1) / side), tiles_n = static_cast<int>((ps->pr[j].n + side - 1) / side);
    const int band = tix / (BAND * tiles_n), in_band = tix - band * BAND * tiles_n, rows = min(BAND, tiles_m - band * BAND);
    const int tn = in_band / rows;
    const int m0 = (band * BAND + in_band - tn * rows) * side + (quarter >> 1) * 128, n0 = tn * side + (quarter & 1) * 128;
    return Tile{m0 < ps->pr[j].m && n0 < ps->pr[j].n ? j : OUTSIDE, m0, n0};
  }
  return Tile{NONE, 0, 0};
}

// One operand of the tile that is being loaded: TRANS: stored across k.  MASK: stored along k, which is no multiple of 64.
template <int W, bool TRANS, bool MASK>
struct Source {
  using S = Stage<W>;
  const uint8_t* base;     // of the tile's first row, at the round's first k (TRANS) or the first one of all, less SHIFT
  int64_t row_bytes;       // TRANS: of a row of k
  unsigned at;             // of the round's first k
  int left;                // k from the round's first one on
  unsigned off[S::loads];  // this lane's part of its pieces, and SHIFT, less what the instruction adds
  int lane_k;              // this lane's first k of a stage

  __device__ __forceinline__ void begin(const void* matrix, int64_t ld, int64_t extent, int first, int k_first, int k_there, int wave, int lane) {
    // TRANS: whole chunks of 8, which rows of k have (copies are padded with zeros); rows that are not there are read as the last
    const int there = static_cast<int>(min(TRANS ? (extent - first + 7) / 8 * 8 : extent - first, static_cast<int64_t>(S::side)));
    left = k_there - k_first;
    const uint8_t* const m = static_cast<const uint8_t*>(matrix) - SHIFT;
    row_bytes = ld * 2;
    if constexpr (TRANS) {
      base = m + static_cast<int64_t>(first) * 2 + k_first * row_bytes;
      at = 0, lane_k = 0;
      constexpr int ROW = 2 * S::side, EACH = 1024 / ROW;   // bytes of a row of k, rows of k of a piece
      const int in_row = lane * 16 % ROW;
#pragma unroll
      for (int i = 0; i < S::loads; ++i) {
        const int row_k = (wave * S::loads + i) * EACH + lane * 16 / ROW;
        const int row = (((in_row >> 6) ^ (row_k & 3)) << 5) + (((in_row >> 5 & 1) ^ (row_k >> 3 & 1)) << 4) + (in_row & 31) / 2;
        off[i] = static_cast<unsigned>(row_k * row_bytes + min(row, there - 8) * 2) + SHIFT - (i & 3) * 1024;
      }
    } else {
      base = m + first * row_bytes;
      at = static_cast<unsigned>(k_first) * 2;
      const int chunk = (lane & 7) ^ (lane >> 3);
      lane_k = chunk * 8;
#pragma unroll
      for (int i = 0; i < S::loads; ++i)
        off[i] = static_cast<unsigned>(min((wave * S::loads + i) * 8 + (lane >> 3), there - 1) * row_bytes + chunk * 16) + SHIFT - (i & 3) * 1024;
    }
  }
  template <int STAGES>
  __device__ __forceinline__ void next_round() {
    left -= STAGES * STAGE_K;
    if constexpr (TRANS)
      base += STAGES * STAGE_K * row_bytes;
    else
      at += STAGES * STAGE_K * 2;
  }
  // Piece I of this wavefront of the round's stage ST.  Across k the descriptor ends with the last k; along k a stage is there or not, or (MASK) a lane whose k is not there asks for nothing:
  // 8192^3 takes 847 us with these selects and 807 without.
  template <int ST, int I>
  __device__ __forceinline__ void fetch(uint8_t* st, int wave) const {
    uint8_t* const to = st + (wave * S::loads + (I & ~3)) * 1024;
    const int there = left - ST * STAGE_K;
    if constexpr (TRANS) {
      const int rows = __builtin_amdgcn_readfirstlane(there > STAGE_K ? STAGE_K : there > 0 ? there : 0);   // (uniform, which the compiler may lose sight of)
      buffer_to_lds<(I & 3) * 1024>(base + ST * STAGE_K * row_bytes, static_cast<unsigned>(rows) * static_cast<unsigned>(row_bytes) + SHIFT, to, off[I], 0);
    } else {
      const unsigned from = __builtin_amdgcn_readfirstlane(at + ST * STAGE_K * 2);
      if constexpr (MASK)
        buffer_to_lds<(I & 3) * 1024>(base, ROOM, to, lane_k < there ? off[I] : NOTHING, from);
      else
        buffer_to_lds<(I & 3) * 1024>(base, __builtin_amdgcn_readfirstlane(there > 0 ? ROOM : 0u), to, off[I], from);
    }
  }
};

// A wavefront's operand of 16 rows and 32 k from a stage: lane l has 8 consecutive k (from 8 (l / 16) on) of row l % 16.
template <int W, bool TRANS>
struct Reader {
  int at[TRANS ? W : 2];   // this lane's offsets in the operand's part of a stage: by pieces of 32 rows, or by halves

  __device__ __forceinline__ void begin(int side, int lane) {   // side: which of the block's two parts of 32 W rows
    const int l = lane & 15, k8 = lane >> 4;
    if constexpr (TRANS) {
#pragma unroll
      for (int t = 0; t < W; ++t)
        at[t] = (8 * k8 + (l >> 2)) * (128 * W) + (((side * W + t) ^ (l >> 2)) << 6) + ((k8 & 1) << 5) + 8 * (l & 3);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) at[h] = (side * 32 * W + l) * 128 + (((4 * h + k8) ^ (l & 7)) << 4);
    }
  }
  // tile T of the wavefront's 2 W, half HALF of the stage
  template <int T, int HALF>
  __device__ __forceinline__ bf16x8 read(const uint8_t* st) const {
    if constexpr (TRANS) {
      typedef __attribute__((address_space(3))) s16x4 lds_vec;
      const uint8_t* const from = st + (at[T / 2] ^ (T % 2 * 32)) + HALF * 32 * (128 * W);   // an odd tile is the other half of its piece
      const s16x4 v[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_vec*)CANZ_LDS(from)), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_vec*)CANZ_LDS(from + 4 * (128 * W)))};
      return __builtin_bit_cast(bf16x8, v);
    } else {
      return *reinterpret_cast<const bf16x8*>(st + at[HALF] + T * 16 * 128);
    }
  }
};

// acc += P Q^T.  ASM: accumulators that fill one half of the registers stay there, each where it is; through the builtin the compiler moves some of them around in every round, where an
// operand is read across k.  What it knows about these instructions and does not see here: their operands come from LDS, behind a wait; the same accumulator is needed again 63 instructions
// later; and settle() follows every round, before anything else can read accumulators (it takes as long as the last instruction).  tests/test_linear_hazards.py looks for these distances in
// the assembly.
template <bool ASM>
__device__ __forceinline__ void multiply(f32x4& acc, const bf16x8& p, const bf16x8& q) {
  if constexpr (ASM)
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(p), "v"(q));
  else
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, acc, 0, 0, 0);
}
template <bool ASM>
__device__ __forceinline__ void settle() {
  if constexpr (ASM) asm volatile("s_nop 15");   // 16 wait states, where the results of instructions of 4 passes need 8, of 8 passes 12
}

// STAGES: of the ring.  Where small tiles leave a CU with one block, whose steps are short, four of them give what is on its way as long as it needs.
template <int W, int STAGES, bool AT, bool BT, bool MASK>
__global__ __launch_bounds__(THREADS, W == 2 && STAGES == 2 ? 2 : 1) void k_linear(LinearProblems) {
  using S = Stage<W>;
  const LinearArgs ps = (LinearArgs)__builtin_amdgcn_kernarg_segment_ptr();
  // one array per stage: the compiler then knows that a fetch into one stage does not alias the reads of another
  __shared__ __attribute__((aligned(1024))) uint8_t st0[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st1[S::bytes];
  __shared__ __attribute__((aligned(1024))) uint8_t st2[STAGES > 2 ? S::bytes : 16];
  __shared__ __attribute__((aligned(1024))) uint8_t st3[STAGES > 2 ? S::bytes : 16];
  auto stage_at = [&](auto number) CANZ_INLINE -> uint8_t* {
    constexpr int N = decltype(number)::value % STAGES;
    return N == 0 ? st0 : N == 1 ? st1 : N == 2 ? st2 : st3;
  };
  constexpr int CW = 16 * W;                                  // columns of a piece of the wavefront's part that goes through LDS at a time
  __shared__ __attribute__((aligned(1024))) float turn[4][32 * CW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  // ---- loading: this wavefront's pieces of the next round, all of its stages.  Every tile takes whole rounds; what lies behind the last k gives zeros.
  Tile next_tile;   // the one that is loaded: the next one, from the last round of a tile on
  int next_logical = blockIdx.x;
  Source<W, AT, MASK> sa;
  Source<W, BT, MASK> sb;
  auto load_next_tile = [&]() CANZ_INLINE {
    Tile t;
    do {
      t = tile_at<W>(ps, next_logical);
      next_logical += gridDim.x;
    } while (W == 2 && t.problem == OUTSIDE);
    next_tile = t;
    sa.left = sb.left = 0;
    if (t.problem < 0) return;   // nothing left: zeros
    const auto& p = ps->pr[t.problem];
    const int first = p.first_step * LINEAR_K, k_end = first + p.steps * LINEAR_K;
    sa.begin(p.a, p.lda, p.m, t.m0, first, min(p.k_a, k_end), wave, lane);
    sb.begin(p.b, p.ldb, p.n, t.n0, first, min(p.k_b, k_end), wave, lane);
  };
  constexpr int LOADS = 2 * S::loads;
  auto fetch_one = [&](auto stage, uint8_t* st, auto idx) CANZ_INLINE {
    constexpr int I = decltype(idx)::value, ST = decltype(stage)::value;
    if constexpr (I < S::loads)
      sa.template fetch<ST, I>(st, wave);
    else
      sb.template fetch<ST, I - S::loads>(st + S::operand, wave);
  };

  // ---- operands in registers: two sets of B's, which every row of tiles needs; one of A's, each of which is read anew behind its row of tiles
  Reader<W, AT> ra;
  Reader<W, BT> rb;
  ra.begin(wm, lane);
  rb.begin(wn, lane);
  constexpr int T = 2 * W;   // tiles of a wavefront along either side
  bf16x8 fa[T], fb[2][T];
  f32x4 acc[T][T];
  // vmcnt(n) lgkmcnt(0)
  constexpr auto wait_code = [](int vm) { return (vm & 15) | 0x70 | (vm >> 4) << 14; };

  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;
  // One step, from half HALF of stage `stage`; the next one's operands lie in its other half, or in the next stage.  The second half's step fetches the stage of the next round.
  auto step = [&](auto half, auto stage) CANZ_INLINE {
    constexpr int H = decltype(half)::value, N = T * T;
    uint8_t* const cur = stage_at(stage);
    const uint8_t* const nxt = stage_at(std::integral_constant<int, decltype(stage)::value + H>{});
    if constexpr (H == 1) {
      __builtin_amdgcn_s_waitcnt(wait_code((STAGES - 2) * LOADS));
      __builtin_amdgcn_s_barrier();
      CANZ_FENCE();
    }
    static_for<N>([&](auto x) CANZ_INLINE {
      constexpr int idx = decltype(x)::value, i = idx / T, j = idx % T;
      // B first: a lane then has 4 consecutive columns of a row of C; and the first operand changes from one instruction to the next while the second stays, which costs less power
      multiply<W == 4>(acc[i][j], fb[H][j], fa[i]);
      if constexpr (j == T - 1) {
        CANZ_FENCE();
        fa[i] = ra.template read<i, 1 - H>(nxt);
        CANZ_FENCE();
      }
      constexpr int PACE = T / 2;   // B's are there before the next step begins
      if constexpr (idx < N / 2 && idx % PACE == 1) {
        CANZ_FENCE();
        fb[1 - H][idx / PACE] = rb.template read<idx / PACE, 1 - H>(nxt + S::operand);
        CANZ_FENCE();
      }
      if constexpr (H == 1) {
        // evenly over the step: asked for in its first half, which would give them longer to arrive, they wait for one another (12288 x 4096 x 8192 735 us instead of 684)
        static_for<(idx + 1) * LOADS / N - idx * LOADS / N>([&](auto y) CANZ_INLINE {
          CANZ_FENCE();
          fetch_one(stage, cur, std::integral_constant<int, idx * LOADS / N + decltype(y)::value>{});
          CANZ_FENCE();
        });
      }
    });
  };
  auto round = [&]() CANZ_INLINE {
    static_for<STAGES>([&](auto stage) CANZ_INLINE {
      step(Zero{}, stage);
      step(One{}, stage);
    });
  };

  // Accumulator register r of lane l in tile (i, j) is row 16 i + l % 16, column 16 j + 4 (l / 16) + r of the wavefront's part.  Pieces of 32 x CW of it go through LDS, 16-byte
  // chunks turned by the row, so that a lane has eight consecutive columns and a store instruction long pieces of rows.
  auto store_tile = [&](const Tile& t) CANZ_INLINE {
    int l = threadIdx.x & 63;   // opaque, or every address that depends on it is kept across the tiles
    asm volatile("" : "+v"(l));
    const LinearEnd e = linear_end_of(ps->pr[t.problem].end);
    const int64_t m = ps->pr[t.problem].m, n = ps->pr[t.problem].n;
    constexpr int CHUNKS = CW / 4, COLS = CW / 8, ROWS = 64 / COLS;   // of a row; lanes along a row, rows at a time
    float* const mine = turn[wave];
    // One copy of what is done to a piece, to its four or eight rows at once: 4096 x 4096 x 256 takes 18.6 us, with a copy for each piece (100 KB of instructions) and its rows one after
    // another 24.9.
#pragma clang loop unroll(disable)
    for (int piece = 0; piece < 2 * W; ++piece) {
      static_for<2 * W>([&](auto x) CANZ_INLINE {
        constexpr int P = decltype(x)::value, i = P / 2, q = P % 2;
        if (piece != P) return;
#pragma unroll
        for (int ii = 0; ii < 2; ++ii)
#pragma unroll
          for (int jj = 0; jj < W; ++jj) {
            const int r = ii * 16 + (l & 15), chunk = (jj * 4 + (l >> 4)) ^ (r & (CHUNKS - 1));
            *reinterpret_cast<f32x4*>(mine + r * CW + chunk * 4) = acc[2 * i + ii][q * W + jj];
          }
        asm volatile("; piece %0" ::"n"(P));   // apart, or the stores are merged into one of an accumulator by its number, and the accumulators go to memory
      });
      const int64_t row0 = t.m0 + wm * 32 * W + (piece >> 1) * 32 + l / COLS, col0 = t.n0 + wn * 32 * W + (piece & 1) * CW, col = col0 + l % COLS * 8;
      constexpr int R = 32 / ROWS;
      auto finish = [&](auto whole) CANZ_INLINE {
        f32x8 z[R];
#pragma unroll
        for (int x = 0; x < R; ++x) {
          const int r = x * ROWS + l / COLS, c = l % COLS;
          const f32x4 lo = *reinterpret_cast<const f32x4*>(mine + r * CW + ((2 * c) ^ (r & (CHUNKS - 1))) * 4);
          const f32x4 hi = *reinterpret_cast<const f32x4*>(mine + r * CW + ((2 * c + 1) ^ (r & (CHUNKS - 1))) * 4);
          z[x] = f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        }
        linear_end<decltype(whole)::value, R>(e, row0, ROWS, col, m, n, z);
      };
      if (t.m0 + 64 * W <= m && t.n0 + 64 * W <= n)
        finish(std::true_type{});
      else
        finish(std::false_type{});
    }
  };

  load_next_tile();
  if (next_tile.problem < 0) return;   // this XCD's share is one tile less than others'
  static_for<STAGES>([&](auto stage) CANZ_INLINE {
    static_for<LOADS>([&](auto idx) CANZ_INLINE { fetch_one(stage, stage_at(stage), idx); });
  });
  __builtin_amdgcn_s_waitcnt(wait_code((STAGES - 1) * LOADS));
  __builtin_amdgcn_s_barrier();
  CANZ_FENCE();
  static_for<T>([&](auto idx) CANZ_INLINE {
    constexpr int I = decltype(idx)::value;
    fa[I] = ra.template read<I, 0>(st0);
    fb[0][I] = rb.template read<I, 0>(st0 + S::operand);
  });

  for (;;) {
    const Tile t = next_tile;
    if (t.problem < 0) break;
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int j = 0; j < T; ++j) {
        acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (W == 4) asm volatile("" : "+a"(acc[i][j]));   // zeros that the compiler does not know: it would make them anew where a tile has but one round
      }
    // the last round, which loads the next tile's first one, apart: with both in one loop, what the loads need is copied to and fro in every round
    for (int rounds = (ps->pr[t.problem].steps + 2 * STAGES - 1) / (2 * STAGES); rounds > 1; --rounds) {
      sa.template next_round<STAGES>(), sb.template next_round<STAGES>();
      round();
      settle<W == 4>();
    }
    load_next_tile();
    round();
    settle<W == 4>();
    store_tile(t);
  }
  __builtin_amdgcn_s_waitcnt(wait_code(0));   // the requests behind the last tile have landed before the block leaves
}

// sets first_tile of every problem for tiles of `side` x `side`; the number of tiles
int64_t count_tiles(LinearProblems& ps, int side) {
  int64_t tiles = 0;
  for (int i = 0; i < ps.n; ++i) {
    ps.first_tile[i] = static_cast<int>(tiles);
    tiles += (ps.pr[i].m + side - 1) / side * ((ps.pr[i].n + side - 1) / side);
  }
  ps.first_tile[ps.n] = static_cast<int>(tiles);
  return tiles;
}

// An XCD has at most this many of the tiles: an eighth of each product, rounded up.
int longest_share(const LinearProblems& ps) {
  int64_t longest = 0;
  for (int i = 0; i < ps.n; ++i) longest += (ps.first_tile[i + 1] - ps.first_tile[i] + N_XCD - 1) / N_XCD;
  return static_cast<int>(longest);
}
// Blocks for `each` tiles on every XCD, `most` (a multiple of 8) at a time.
dim3 tile_grid(int64_t each, int most) { return dim3(static_cast<unsigned>(std::min<int64_t>(N_XCD * each, most))); }

template <int W, int STAGES, bool MASK>
void launch(const LinearProblems& ps, bool at, bool bt, dim3 grid, hipStream_t st) {
  if (at && bt)
    k_linear<W, STAGES, true, true, false><<<grid, THREADS, 0, st>>>(ps);
  else if (at)
    k_linear<W, STAGES, true, false, MASK><<<grid, THREADS, 0, st>>>(ps);
  else if (bt)
    k_linear<W, STAGES, false, true, MASK><<<grid, THREADS, 0, st>>>(ps);
  else
    k_linear<W, STAGES, false, false, MASK><<<grid, THREADS, 0, st>>>(ps);
}
template <int W, int STAGES>
void launch(const LinearProblems& ps, bool at, bool bt, dim3 grid, hipStream_t st) {
  bool mask = false;
  for (int i = 0; i < ps.n; ++i) mask = mask || (!at && ps.pr[i].k_a % STAGE_K != 0) || (!bt && ps.pr[i].k_b % STAGE_K != 0);
  if (mask)
    launch<W, STAGES, true>(ps, at, bt, grid, st);
  else
    launch<W, STAGES, false>(ps, at, bt, grid, st);
}
// `each` small tiles on every XCD, `alone`: one to a CU at a time
void launch_small(const LinearProblems& ps, int64_t each, bool alone, bool at, bool bt, hipStream_t st) {
  if (alone || N_XCD * each <= LINEAR_CU)
    launch<2, 4>(ps, at, bt, tile_grid(each, LINEAR_CU), st);
  else
    launch<2, 2>(ps, at, bt, tile_grid(each, 2 * LINEAR_CU), st);
}

}  // namespace

hipError_t launch_linear_tiles(LinearProblems& ps, bool a_trans, bool b_trans, hipStream_t st) {
  std::sort(ps.pr, ps.pr + ps.n, [](const LinearProblem& x, const LinearProblem& y) { return x.steps > y.steps; });   // the longest begin
  const int64_t large = count_tiles(ps, 256), small = count_tiles(ps, 128);
  int64_t steps = 0;   // of all small tiles
  for (int i = 0; i < ps.n; ++i) steps += static_cast<int64_t>(ps.first_tile[i + 1] - ps.first_tile[i]) * ps.pr[i].steps;
  const bool alone = linear_alone(ps.pr[0].steps, steps);
  steps = (steps + small - 1) / small;
  ps.from = 0, ps.to = longest_share(ps), ps.quarters = 0;
  if (!linear_large_tiles(large, small, steps)) {
    launch_small(ps, ps.to, alone, a_trans, b_trans, st);
    return hipGetLastError();
  }
  count_tiles(ps, 256);
  const int all = longest_share(ps), whole = static_cast<int>(linear_whole_rounds(large, steps)) * (LINEAR_CU / N_XCD);
  ps.to = whole > 0 ? std::min(whole, all) : all;
  launch<4, 2>(ps, a_trans, b_trans, tile_grid(ps.to, LINEAR_CU), st);
  if (ps.to < all) {   // what the last round would leave most CUs without
    ps.from = ps.to, ps.to = all, ps.quarters = 1;
    launch_small(ps, int64_t{4} * (ps.to - ps.from), false, a_trans, b_trans, st);
  }
  return hipGetLastError();
}

}  // namespace canz
