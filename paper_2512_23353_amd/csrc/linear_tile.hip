// The policy's linear layer in bf16: Y = act(X W^T + b) + R, and dX = Delta W, on the matrix cores.
//
// Bound by the matrix cores and, with random operands, by the board's power limit; of few tokens by reading W.  16384 x 4096 -> 14336: 1.33 - 1.40 ms,
// 1.37 - 1.45 PFLOP/s (dX 1.29 - 1.36 ms; SiLU and Z, 470 MB more to write, add 0.08; a library's plain product 1.25); one token 4096 -> 14336: 22 - 26
// us, 4.5 - 5.3 TB/s of W.  A workgroup forms BO outputs x BT tokens, 64 of the sum's terms (a block) at a time:
//  * Both operands go from memory straight into LDS, 16 bytes a lane, NS blocks in flight.  X, Delta and W of the forward pass have the
//    sum's index contiguous: rows of 128 bytes (whole lines) in LDS, whose eight 16-byte columns are permuted by the row so that fragment reads meet
//    all banks.  W of dX = Delta W has the sum's index slow: rows of BO outputs, read through the LDS transpose.  The loads' cost is per line they
//    touch: with blocks of 32 terms, half lines, five of them in flight, 1451 -> 1698 us (k = 4160).
//  * The buffer descriptors end with the last valid row: rows past it arrive as zeros.  Columns past the sum's end, which would be the next row's
//    numbers, are given an offset outside the descriptor: zeros too, on both sides, so that no NaN meets a zero there.
//  * A block is two steps of 16x16x32 MFMAs (they cost less power per flop than 32x32x16).  The first half of step 0 carries the fragment reads of step 1; then this
//    stage is free, and the second half of step 0 and the first of step 1 carry the loads of the block NS ahead into it.  Step 1, before which the
//    next block has landed, carries that one's first reads.
//  * Where the time of the large product goes (us, random / zero operands, on copies of the kernel): as it is 1476 / 1141; every tile from the same
//    rows, so from the L2s, 1306 / 1005; without loads 1200 / 934.  Tried and not kept: four waves of 128 x 128 with the accumulators in AGPRs (1451 -> 1500),
//    the next block awaited half a step later (1479), XCDs that start at different blocks of the sum (level).
//  * The outputs are the MFMA's rows, the tokens its columns, and which outputs a pair of row blocks stands for is chosen so that a lane ends
//    with eight neighbouring outputs of a token: 16-byte accesses to R, bias and the workspace.
//  * Few tiles: the sum is split over workgroups, whose fp32 parts a second launch adds in order and finishes.
#include <cmath>
#include <utility>

#include "activation.h"
#include "policy.h"
#include "row_sum.h"
#include "seq_grad_stream.h"

namespace isopo {
namespace {

constexpr int kTerms = 64;                       // terms of the sum per block
constexpr int kRowBytes = kTerms * 2;

struct TileParams {
  LinearArgs a;
  TileGrid grid;                                 // m: token tiles, n: output tiles
  unsigned workgroups;                           // of the product; behind them those of a.then
  int tiles, blocks_per_part;                    // blocks of the sum per part
  float* parts;                                  // [parts][rows][n_out], or NULL: the sum is whole
};

typedef const __attribute__((address_space(3))) bf16x8* lds_frag_ptr;

// which 16-byte column of an LDS row global column `c` is in: rows of X or Delta (fragments take 16 rows in a row), rows of W (fragments take
// rows 0-3, 8-11, 16-19, 24-27 of 32, or four more), and rows of a W whose rows are the sum's terms (32 columns and more)
__device__ __forceinline__ int swz_token(int row) { return row & 7; }
__device__ __forceinline__ int swz_out(int row) { return (row & 3) | ((row >> 3 & 1) << 2); }
__device__ __forceinline__ int swz_term(int row) { return ((row & 3) << 2) ^ (row >> 3 & 1) ^ ((row >> 4 & 1) << 1); }

// f(0) .. f(N - 1), the index a constant
template <class F, int... I>
__device__ __forceinline__ void unrolled(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}

typedef unsigned loose_u32x4 __attribute__((ext_vector_type(4), aligned(2)));       // a bias is aligned to an element
__device__ __forceinline__ void add8(u32x4 w, float (&z)[8]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    z[2 * q] += __builtin_bit_cast(float, (unsigned)w[q] << 16);
    z[2 * q + 1] += __builtin_bit_cast(float, (unsigned)w[q] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 bias8(const void* bias, int col) { return *reinterpret_cast<const loose_u32x4*>(static_cast<const u16*>(bias) + col); }
__device__ __forceinline__ u32x4 load8(const void* from, long long at) { return *reinterpret_cast<const u32x4*>(static_cast<const u16*>(from) + at); }
__device__ __forceinline__ u32x4 pack8(const float (&z)[8]) {
  return u32x4{pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])};
}

// BO x BT: outputs and tokens of a tile; WO x WT: its waves; NS: stages.  TERM_ROWS: W's rows are the sum's terms.
template <int BO, int BT, int WO, int WT, int NS, bool TERM_ROWS>
__global__ __launch_bounds__(64 * WO * WT, 2) void linear_tile_kernel(TileParams p) {
  constexpr int NW = WO * WT, FO = BO / WO / 16, FT = BT / WT / 16;        // 16-wide row and column blocks of a wave
  constexpr unsigned OUT_BYTES = BO * kRowBytes, STAGE = OUT_BYTES + BT * kRowBytes;
  constexpr int LO = OUT_BYTES / 1024 / NW, LT = BT * kRowBytes / 1024 / NW, LPT = LO + LT;       // 1 KiB loads of a wave per block
  static_assert(FO % 2 == 0 && LO * 1024 * NW == (int)OUT_BYTES && LT * 1024 * NW == BT * kRowBytes, "whole loads");
  constexpr unsigned PITCH = BO * 2;                                        // TERM_ROWS: LDS row of a term
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const unsigned base = (unsigned)(size_t)(lds_void_ptr)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wo = wave / WT, wt = wave % WT;
  const LinearArgs& a = p.a;
  if (blockIdx.x >= p.workgroups) {
    row_sum<64 * NW>(a.then, blockIdx.x - p.workgroups, reinterpret_cast<float*>(smem));
    return;
  }

  const int id = (int)xcd_contiguous(blockIdx.x, p.workgroups);
  const int part = id / p.tiles;
  int tile_t, tile_o;
  tile_coords<0>(id - part * p.tiles, p.grid, tile_t, tile_o);
  const long long t0 = (long long)tile_t * BT;
  const int o0 = tile_o * BO;
  const int k0 = part * p.blocks_per_part * kTerms;
  const int k_end = a.k - k0 < p.blocks_per_part * kTerms ? a.k : k0 + p.blocks_per_part * kTerms;
  const int n_blocks = (k_end - k0 + kTerms - 1) / kTerms;

  // the loads' cursor: first bytes of the next block in X (or Delta) and in W, bytes to the end of the last valid row, terms left
  const int rows = a.rows - t0 < BT ? (int)(a.rows - t0) : BT;
  const long long ldw = TERM_ROWS ? a.n_out : a.k;
  auto uniform64 = [](const void* q) {
    const unsigned long long v = (unsigned long long)q;
    const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)v), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(v >> 32));
    return (unsigned long long)hi << 32 | lo;
  };
  unsigned long long pt = uniform64(static_cast<const u16*>(a.A) + t0 * a.lda + k0);
  unsigned long long pw = uniform64(static_cast<const u16*>(a.B) + (TERM_ROWS ? (long long)k0 * ldw + o0 : o0 * ldw + k0));
  const int outs = a.n_out - o0 < BO ? a.n_out - o0 : BO;
  int k_left = k_end - k0;
  // offsets within a block: lane l of a load brings row l / 8, LDS column l % 8 (or, of a term row, column l % (BO / 8))
  unsigned off_t[LT], off_o[LO];
  const int col_t = (lane & 7) ^ swz_token(lane >> 3);
#pragma unroll
  for (int q = 0; q < LT; ++q) off_t[q] = (unsigned)(((wave * LT + q) * 8 + (lane >> 3)) * a.lda * 2 + col_t * 16);
#pragma unroll
  for (int q = 0; q < LO; ++q) {
    if constexpr (TERM_ROWS) {
      constexpr int COLS = BO / 8, RPL = 64 / COLS;
      const int r = (wave * LO + q) * RPL + lane / COLS;
      off_o[q] = (unsigned)(r * ldw * 2 + ((lane % COLS) ^ swz_term(r)) * 16);
    } else {
      const int r = (wave * LO + q) * 8 + (lane >> 3);
      off_o[q] = (unsigned)(r * ldw * 2 + ((lane & 7) ^ swz_out(r)) * 16);
    }
  }
  constexpr unsigned OUTSIDE = 0x80000000u;      // past every descriptor
  struct Block { v4i t, w; int left; };
  auto next_block = [&](Block& b) {
    const int left = k_left > 0 ? k_left : 0;
    const bool any = left > 0;
    b.left = left;
    b.t[0] = (int)(unsigned)pt; b.t[1] = (int)((unsigned)(pt >> 32) & 0xffffu);
    b.t[2] = any ? (int)(((unsigned)(rows - 1) * (unsigned)a.lda + (unsigned)left) * 2u) : 0; b.t[3] = 0x00020000;
    b.w[0] = (int)(unsigned)pw; b.w[1] = (int)((unsigned)(pw >> 32) & 0xffffu);
    if constexpr (TERM_ROWS) b.w[2] = any ? (int)(((unsigned)((left < kTerms ? left : kTerms) - 1) * (unsigned)ldw + (unsigned)outs) * 2u) : 0;
    else b.w[2] = any ? (int)(((unsigned)(outs - 1) * (unsigned)ldw + (unsigned)left) * 2u) : 0;
    b.w[3] = 0x00020000;
    pt += kRowBytes;
    pw += TERM_ROWS ? (unsigned long long)kTerms * ldw * 2 : (unsigned long long)kRowBytes;
    k_left -= kTerms;
  };
  auto issue = [&](auto which, const Block& b, unsigned stage) {
    constexpr int q = decltype(which)::value;
    // (left is a multiple of 8: a column is inside or outside as a whole)
    if constexpr (q < LO) {
      unsigned off = off_o[q];
      if constexpr (!TERM_ROWS) {
        const int col = (lane & 7) ^ swz_out((wave * LO + q) * 8 + (lane >> 3));
        off = col * 8 < b.left ? off : OUTSIDE;
      }
      load_lds16(b.w, stage + (unsigned)(wave * LO + q) * 1024, off);
    } else {
      load_lds16(b.t, stage + OUT_BYTES + (unsigned)(wave * LT + (q - LO)) * 1024, col_t * 8 < b.left ? off_t[q - LO] : OUTSIDE);
    }
  };

  // Fragment addresses within a stage.  Row r of row block i stands for output 32 (i / 2) + 8 (r / 4) + r % 4 of the wave's, plus 4 in odd blocks
  // (TERM_ROWS: in odd blocks where r / 4 is even, in even ones where it is odd: two lane groups then read different halves of 16 bytes).  The
  // permutations leave one address per operand, that a block or step changes by a constant.
  const int l15 = lane & 15, g4 = lane >> 4;
  unsigned ad_o, ad_t;
  {
    const int r = wt * (BT / WT) + l15;                                     // r & 7 is that of every 16th row on
    ad_t = OUT_BYTES + (unsigned)(r * kRowBytes + ((g4 ^ swz_token(r)) << 4));
    if constexpr (TERM_ROWS) {
      // the transposing read: lane l brings four outputs of term row l / 4 of its group's eight, and is left with four terms of output l % 16
      const int q = l15 & 3, o = wo * (BO / WO) + q * 8 + 4 * (q & 1), k = g4 * 8 + (l15 >> 2);
      ad_o = (unsigned)(k * PITCH + (((o >> 3) ^ swz_term(k)) << 4) + (o & 7) * 2);
    } else {
      const int o = wo * (BO / WO) + (l15 >> 2) * 8 + (l15 & 3);            // swz_out is that of every 32nd row and of the fourth after
      ad_o = (unsigned)(o * kRowBytes + ((g4 ^ swz_out(o)) << 4));
    }
  }
  // of step s (its four columns of 16 bytes are the first's with bit 2 flipped) and block i or j
  auto frag_t = [&](unsigned stage_t, auto s, auto j) __attribute__((always_inline)) {
    return *(lds_frag_ptr)(size_t)((stage_t ^ (decltype(s)::value << 6)) + decltype(j)::value * 16 * kRowBytes);
  };
  auto frag_o = [&](unsigned stage_o, auto s, auto at) __attribute__((always_inline)) {
    constexpr int i = decltype(at)::value;
    if constexpr (TERM_ROWS) {
      const unsigned from = (stage_o ^ ((unsigned)(i >> 1) << 6 | (unsigned)(i & 1) << 3)) + decltype(s)::value * 32 * PITCH;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(size_t)from);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(size_t)(from + 4 * PITCH));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *(lds_frag_ptr)(size_t)((stage_o ^ (decltype(s)::value << 6)) + ((i >> 1) * 32 + 4 * (i & 1)) * kRowBytes);
    }
  };

  f32x4 acc[FO][FT];
#pragma unroll
  for (int i = 0; i < FO; ++i)
#pragma unroll
    for (int j = 0; j < FT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 fo[2][FO], ft[2][FT];

  Block nb;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    next_block(nb);
    unrolled(std::make_integer_sequence<int, LPT>{}, [&](auto q) __attribute__((always_inline)) { issue(q, nb, base + s * STAGE); });
  }
  // everyone's loads of a block have landed, and what was read before has been read: at most `rest` loads of this wave still fly
#define ISOPO_MEET(rest)                                                                                            \
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(rest) : "memory")
  ISOPO_MEET((NS - 1) * LPT);
  constexpr std::integral_constant<int, 0> s0{};
  unrolled(std::make_integer_sequence<int, FT>{}, [&](auto j) __attribute__((always_inline)) { ft[0][j] = frag_t(base + ad_t, s0, j); });
  unrolled(std::make_integer_sequence<int, FO>{}, [&](auto i) __attribute__((always_inline)) { fo[0][i] = frag_o(base + ad_o, s0, i); });
  next_block(nb);

  constexpr int M = FO * FT, R = FO + FT, EARLY = M / 2, L0 = LPT / 2;
  unsigned stage = 0;                            // of the block being multiplied
  for (int it = 0; it < n_blocks; ++it) {
    const unsigned now = base + stage * STAGE;
    stage = stage + 1 == NS ? 0 : stage + 1;
    const unsigned next = base + stage * STAGE;
    // step 0: behind its first half the reads of step 1, then this stage is free for the block NS ahead; step 1: the next block's first reads
    unrolled(std::make_integer_sequence<int, 2 * M>{}, [&](auto at) __attribute__((always_inline)) {
      constexpr int s = decltype(at)::value / M, idx = decltype(at)::value % M, i = idx / FT, j = idx % FT;
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fo[s][i], ft[s][j], acc[i][j], 0, 0, 0);
      constexpr int SPAN = s == 0 ? EARLY * 3 / 4 : M * 3 / 4;
      constexpr int r0 = idx * R / SPAN < R ? idx * R / SPAN : R, r1 = (idx + 1) * R / SPAN < R ? (idx + 1) * R / SPAN : R;
      unrolled(std::make_integer_sequence<int, r1 - r0>{}, [&](auto k) __attribute__((always_inline)) {
        constexpr int r = r0 + decltype(k)::value;
        constexpr std::integral_constant<int, s ^ 1> other{};
        if constexpr (r < FT) ft[s ^ 1][r] = frag_t((s == 0 ? now : next) + ad_t, other, std::integral_constant<int, r>{});
        else fo[s ^ 1][r - FT] = frag_o((s == 0 ? now : next) + ad_o, other, std::integral_constant<int, r - FT>{});
      });
      if constexpr (s == 0 && idx == EARLY - 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
      constexpr int q0 = s == 0 ? (idx < EARLY ? 0 : (idx - EARLY) * L0 / (M - EARLY)) : L0 + (idx < EARLY ? idx * (LPT - L0) / EARLY : LPT - L0);
      constexpr int q1 = s == 0 ? (idx < EARLY ? 0 : (idx + 1 - EARLY) * L0 / (M - EARLY)) : L0 + (idx < EARLY ? (idx + 1) * (LPT - L0) / EARLY : LPT - L0);
      unrolled(std::make_integer_sequence<int, q1 - q0>{}, [&](auto k) __attribute__((always_inline)) {
        issue(std::integral_constant<int, q0 + decltype(k)::value>{}, nb, now);
      });
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (s == 0 && idx == M - 1) ISOPO_MEET((NS - 2) * LPT + L0);
    });
    next_block(nb);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#undef ISOPO_MEET

  // lane (l15, g4) holds, of row blocks 2 i and 2 i + 1 and column block j, outputs 8 g4 .. + 7 of 32 and token l15
  auto eight = [&](int i, int j, float (&z)[8]) {
    const bool swap = TERM_ROWS && (g4 & 1);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float x = acc[2 * i][j][v], y = acc[2 * i + 1][j][v];
      z[v] = swap ? y : x;
      z[4 + v] = swap ? x : y;
    }
  };
  const long long row0 = t0 + wt * (BT / WT);
  const int col0 = o0 + wo * (BO / WO);
  if (p.parts) {
    float* const to = p.parts + (size_t)part * a.rows * a.n_out;
#pragma unroll
    for (int j = 0; j < FT; ++j)
#pragma unroll
      for (int i = 0; i < FO / 2; ++i) {
        const long long row = row0 + j * 16 + l15;
        const int col = col0 + i * 32 + g4 * 8;
        if (row >= a.rows || col >= a.n_out) continue;
        float z[8];
        eight(i, j, z);
        f32x4* o = reinterpret_cast<f32x4*>(to + row * a.n_out + col);
        o[0] = f32x4{z[0], z[1], z[2], z[3]};
        o[1] = f32x4{z[4], z[5], z[6], z[7]};
      }
    return;
  }
  // Y and Z go through LDS, each wave's part by itself, and leave as whole rows of the wave's outputs, past the caches: whole lines, and X
  // and W stay in the caches that the outputs (940 MB at 16384 x 4096 -> 14336 with Z) would wash out.  That case 1565 -> 1477 us, 9999 x
  // 1536 -> 8960 level; past the caches without LDS, in pieces of 64 bytes, 1482, but 9999 x 1536 -> 8960 268 -> 281.
  __syncthreads();
  constexpr int CH = BO / WO / 8, TPI = 64 / CH;                            // 16-byte columns of such a row, rows per store
  const unsigned mine = base + (unsigned)wave * (BO / WO * BT / WT * 2);
  typedef __attribute__((address_space(3))) u32x4* lds_out_ptr;
  // all of the epilogue's loads at once, not one by one where they are used: 16384 x 4096 -> 14336 with bias, SiLU and Z 1484 -> 1452 us, 9999 x 1536 ->
  // 8960 288 -> 272, 2001 x 1000 -> 2728 with all of it 30.5 -> 27.0
  constexpr u32x4 none = {0u, 0u, 0u, 0u};
  u32x4 bias[FO / 2], res[FT][FO / 2];
#pragma unroll
  for (int i = 0; i < FO / 2; ++i) {
    const int col = col0 + i * 32 + g4 * 8;
    bias[i] = a.bias && col < a.n_out ? bias8(a.bias, col) : none;
#pragma unroll
    for (int j = 0; j < FT; ++j) {
      const long long row = row0 + j * 16 + l15;
      res[j][i] = a.residual && row < a.rows && col < a.n_out ? load8(a.residual, row * a.ldr + col) : none;
    }
  }
  auto put = [&](void* to, long long ld, auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < FT; ++j)
#pragma unroll
      for (int i = 0; i < FO / 2; ++i) {
        float z[8];
        eight(i, j, z);
        if (a.bias) add8(bias[i], z);
        f(j, i, z);
        *(lds_out_ptr)(size_t)(mine + (j * 16 + l15) * (CH * 16) + (((i * 4 + g4) ^ (l15 & (CH - 1))) << 4)) = pack8(z);
      }
#pragma unroll
    for (int q = 0; q < FT * 16 / TPI; ++q) {
      const int t = q * TPI + lane / CH, c = lane % CH, col = col0 + c * 8;
      const u32x4 v = *(lds_out_ptr)(size_t)(mine + t * (CH * 16) + ((c ^ (t & (CH - 1))) << 4));
      if (row0 + t < a.rows && col < a.n_out) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(static_cast<u16*>(to) + (row0 + t) * ld + col));
    }
  };
  if (a.Z) put(a.Z, a.n_out, [&](int, int, float (&)[8]) {});
  auto finish = [&](auto act) __attribute__((always_inline)) {
    put(a.C, a.ldc, [&](int j, int i, float (&z)[8]) {
#pragma unroll
      for (int q = 0; q < 8; ++q) z[q] = activate<decltype(act)::value>(z[q]);
      if (a.residual) add8(res[j][i], z);
    });
  };
  if (a.act == Act::kSilu) finish(std::integral_constant<Act, Act::kSilu>{});
  else if (a.act == Act::kGelu) finish(std::integral_constant<Act, Act::kGelu>{});
  else if (a.act == Act::kRelu) finish(std::integral_constant<Act, Act::kRelu>{});
  else finish(std::integral_constant<Act, Act::kNone>{});
}

// The parts of split sums, added in order, and the rest of the layer: eight outputs of a token per thread.
template <Act A>
__global__ __launch_bounds__(256) void linear_parts_kernel(LinearArgs a, const float* __restrict__ parts, int n_parts) {
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8, n = a.rows * a.n_out;
  if (i >= n) return;
  float z[8] = {};
#pragma unroll 4
  for (int q = 0; q < n_parts; ++q) {
    const f32x4* x = reinterpret_cast<const f32x4*>(parts + (size_t)q * n + i);
    const f32x4 lo = x[0], hi = x[1];
#pragma unroll
    for (int v = 0; v < 4; ++v) { z[v] += lo[v]; z[4 + v] += hi[v]; }
  }
  const long long row = i / a.n_out;
  const int col = (int)(i - row * a.n_out);
  if (a.bias) add8(bias8(a.bias, col), z);
  if (a.Z) *reinterpret_cast<u32x4*>(static_cast<u16*>(a.Z) + i) = pack8(z);
#pragma unroll
  for (int q = 0; q < 8; ++q) z[q] = activate<A>(z[q]);
  if (a.residual) add8(load8(a.residual, row * a.ldr + col), z);
  *reinterpret_cast<u32x4*>(static_cast<u16*>(a.C) + row * a.ldc + col) = pack8(z);
}

// Tiles and parts of a product: the smallest modelled time, in microseconds.  A workgroup costs a start and, per block, what it takes of its compute
// unit: 256 x 256 tiles, one to a unit, 5 and 1.2; 128 x 128, two to a unit, 2 and 0.5 (two together 1.7 times one).  Parts cost a second
// launch, 0.12 each and the workspace's traffic at 8 bytes per output and part.  Within 10 % of what was measured on 16 products of 1 .. 14119 tokens, 2 to
// 12 points each; what the model takes is at most 8 % from the best of them.
LinearPlan plan(long long rows, int k, int n_out, bool may_split) {
  const auto tiles = [&](int b) { return (double)((rows + b - 1) / b) * ((n_out + b - 1) / b); };
  const int blocks = (k + kTerms - 1) / kTerms;
  const double big = (5.0 + 1.2 * blocks) * std::ceil(tiles(256) / 256.0), small = tiles(128), outputs = (double)rows * n_out;
  LinearPlan best = {rows, 256, 1, 1, blocks};
  double least = big;
  for (const int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
    if (want > 1 && (!may_split || want > blocks / 2 || small * want > 2048.0)) break;
    const int per = (blocks + want - 1) / want, parts = (blocks + per - 1) / per;
    const double wgs = small * parts, rounds = wgs <= 256.0 ? 1.0 : wgs <= 512.0 ? 1.7 : wgs / 256.0;
    const double time = (2.0 + 0.5 * per) * rounds + (parts > 1 ? 3.0 + parts * (0.12 + outputs * 1e-6) : 0.0);
    if (time < least) {
      least = time;
      best = {rows, 128, 1, parts, per};
    }
  }
  return best;
}

template <int BO, int BT, int WO, int WT, int NS, bool TERM_ROWS>
hipError_t launch(const TileParams& p, unsigned blocks, hipStream_t s) {
  constexpr size_t smem = (size_t)NS * (BO + BT) * kRowBytes;
  auto kern = linear_tile_kernel<BO, BT, WO, WT, NS, TERM_ROWS>;
  // once per process and instantiation (static initialisation is thread-safe); a failure is returned by every call
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(64 * WO * WT), smem, s, p);
  return hipGetLastError();
}

template <bool TERM_ROWS>
hipError_t launch_plan(const TileParams& p, const LinearPlan& pl, unsigned blocks, hipStream_t s) {
  return pl.side == 256 ? launch<256, 256, 2, 4, 2, TERM_ROWS>(p, blocks, s) : launch<128, 128, 2, 2, 2, TERM_ROWS>(p, blocks, s);
}

}  // namespace

LinearPlan linear_tile_plan(long long rows, int k, int n_out, bool may_split) { return plan(rows, k, n_out, may_split); }

hipError_t launch_linear_tile(const LinearArgs& a, const LinearPlan& pl, hipStream_t s) {
  TileParams p;
  p.a = a;
  const long long mt = (a.rows + pl.side - 1) / pl.side, nt = (a.n_out + pl.side - 1) / pl.side;
  if (mt * nt * pl.parts > 0x7fffffffLL) return hipErrorInvalidValue;
  p.grid = tile_grid((int)mt, (int)nt);
  p.tiles = (int)(mt * nt);
  p.blocks_per_part = pl.blocks_per_part;
  p.parts = pl.parts > 1 ? a.workspace : nullptr;
  p.workgroups = (unsigned)(p.tiles * pl.parts);
  const unsigned blocks = p.workgroups + row_sum_blocks(a.then);
  hipError_t e = a.b_rows_are_k ? launch_plan<true>(p, pl, blocks, s) : launch_plan<false>(p, pl, blocks, s);
  if (e != hipSuccess || pl.parts == 1) return e;
  const long long threads = a.rows * a.n_out / 8;
  with_act(a.act, [&](auto act) {
    hipLaunchKernelGGL(linear_parts_kernel<decltype(act)::value>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, p.parts, pl.parts);
  });
  return hipGetLastError();
}

}  // namespace isopo
