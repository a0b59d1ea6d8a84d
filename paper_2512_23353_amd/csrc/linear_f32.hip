// The policy's linear layer in fp32: Y = act(X W^T + b) + R, and dX = Delta W, on the matrix cores.
//
// Bound by the matrix cores.  The fp32 MFMA has a sixteenth of the bf16 MFMA's rate, so every value enters as the sum of three
// bf16 values, 2^24 x = h + m + l (8 + 8 + 8 significant bits; so scaled, no value's parts are too small for bf16), and a product is formed
// from hh, hm, mh, mm, hl, lh; what is left out is at most 2^-24 of the product.  A tile whose sums are not finite (theirs or
// their inputs' magnitudes are past 2^79 or 2^103, or not finite either) is formed again with fp32 MFMAs from the same values.
//
// A workgroup of four waves forms BT x BT outputs and tokens (128 or 64), 16 of the sum's terms a stage (32 on the small tile, whose stages
// are all latency), two stages of LDS, one barrier a stage.  A thread loads four terms of a row (X, Delta, W of the forward pass) or of a column
// (W of dX = Delta W, whose rows are the sum's terms), splits them in registers and stores 8 bytes a part: units of 16 bytes hold eight terms
// of a row and part, which is the MFMA's operand.  A step is multiplied while the next is split and stored and the one after it is on its way.
// 9999 x 1536 -> 1536: 255 us, 185 TFLOP/s of fp32 products, 1.11 PFLOP/s of bf16 ones (a library's fp32 product of that size takes
// 377 us); of its 948 workgroups 768, three to a unit, are a full round, and the other 180 are alone on theirs for the last quarter of the time.
// Where even the 64 x 64 tiles are few and the sums long, four or eight waves split a tile's sum instead: they wait for none of the others
// before its end, and fewer launches need parts in the workspace (2001 x 1220 -> 300 as dX 25.5 -> 18.8 us, 1024 x 1024 -> 1024 25.6 -> 19.8).
// They are bound by the MFMAs and the splits, whose times add up on a SIMD (with no loads 51 of 61 us at 1024 x 4096 -> 1024).
// The outputs are the MFMA's rows and the tokens its columns: a lane ends with four neighbouring outputs of a token.  Few tiles: the sum is
// split over workgroups too, whose parts a second launch adds in order.
#include <cmath>
#include <type_traits>

#include "activation.h"
#include "policy.h"
#include "row_sum.h"
#include "seq_grad_stream.h"

namespace isopo {
namespace {

constexpr int kTerms = 16, kParts = 3, kUnit = 16;
constexpr float kScale = 0x1p24f, kUnscale = 0x1p-48f;       // of a value before it is split; of a sum of products of two

struct SplitParams {
  LinearArgs a;
  TileGrid grid;                                 // m: token tiles, n: output tiles
  unsigned workgroups;                           // of the product; behind them those of a.then
  int tiles, blocks_per_part;
  float* parts;
};

typedef float loose_f32x4 __attribute__((ext_vector_type(4), aligned(4)));           // a bias is aligned to an element
__device__ __forceinline__ f32x4 bias4(const void* bias, int col) { return *reinterpret_cast<const loose_f32x4*>(static_cast<const float*>(bias) + col); }
__device__ __forceinline__ f32x4 load4(const void* from, long long at) { return *reinterpret_cast<const f32x4*>(static_cast<const float*>(from) + at); }

template <Act A>
__device__ __forceinline__ void finish4(const LinearArgs& a, long long row, int col, f32x4 z, f32x4 bias, f32x4 res) {
  if (a.bias) z += bias;
  if (a.Z) *reinterpret_cast<f32x4*>(static_cast<float*>(a.Z) + row * a.n_out + col) = z;
#pragma unroll
  for (int q = 0; q < 4; ++q) z[q] = activate<A>(z[q]);
  if (a.residual) z += res;
  *reinterpret_cast<f32x4*>(static_cast<float*>(a.C) + row * a.ldc + col) = z;
}

// A tile's sums: to the workspace, or as outputs.  each(f) calls f(row, col, sums, bias, residual).
template <typename Each>
__device__ __forceinline__ void finish_tile(const SplitParams& p, int part, Each& each) {
  const LinearArgs& a = p.a;
  if (p.parts) {
    float* const to = p.parts + (size_t)part * a.rows * a.n_out;
    each([&](long long r, int col, f32x4 z, f32x4, f32x4) __attribute__((always_inline)) { *reinterpret_cast<f32x4*>(to + r * a.n_out + col) = z; });
    return;
  }
  auto finish = [&](auto act) __attribute__((always_inline)) {
    each([&](long long r, int col, f32x4 z, f32x4 bias, f32x4 res) __attribute__((always_inline)) { finish4<decltype(act)::value>(a, r, col, z, bias, res); });
  };
  if (a.act == Act::kSilu) finish(std::integral_constant<Act, Act::kSilu>{});
  else if (a.act == Act::kGelu) finish(std::integral_constant<Act, Act::kGelu>{});
  else if (a.act == Act::kRelu) finish(std::integral_constant<Act, Act::kRelu>{});
  else finish(std::integral_constant<Act, Act::kNone>{});
}

// Two values times kScale -> their three bf16 parts, packed low half first.
__device__ __forceinline__ void split2(float x0, float x1, unsigned& h, unsigned& m, unsigned& l) {
  const auto pack = [](float a, float b) {
    unsigned r;
    asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
  };
  x0 *= kScale;
  x1 *= kScale;
  h = pack(x0, x1);
  x0 -= __builtin_bit_cast(float, h << 16);
  x1 -= __builtin_bit_cast(float, h & 0xffff0000u);
  m = pack(x0, x1);
  x0 -= __builtin_bit_cast(float, m << 16);
  x1 -= __builtin_bit_cast(float, m & 0xffff0000u);
  l = pack(x0, x1);
}

// NB x NB blocks of 32 x 32 per wave; KS: blocks of 16 terms per stage; TERM_ROWS: W's rows are the sum's terms.
template <int NB, int KS, bool TERM_ROWS>
__global__ __launch_bounds__(256, 3) void linear_split_kernel(SplitParams p) {
  constexpr int BT = 64 * NB, SIDE = 2 * BT * kUnit, PLANE = 2 * SIDE, BLOCK = kParts * PLANE, STAGE = KS * BLOCK;      // outputs' side, then tokens'
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wo = wave >> 1, wt = wave & 1;
  const LinearArgs& a = p.a;
  if (blockIdx.x >= p.workgroups) {
    row_sum<256>(a.then, blockIdx.x - p.workgroups, reinterpret_cast<float*>(lds));
    return;
  }
  const int id = (int)xcd_contiguous(blockIdx.x, p.workgroups);
  const int part = id / p.tiles;
  int tile_t, tile_o;
  tile_coords<0>(id - part * p.tiles, p.grid, tile_t, tile_o);
  const long long t0 = (long long)tile_t * BT;
  const int o0 = tile_o * BT;
  const int k0 = part * p.blocks_per_part * kTerms;
  const int k_end = a.k - k0 < p.blocks_per_part * kTerms ? a.k : k0 + p.blocks_per_part * kTerms;
  const int n_blocks = (k_end - k0 + kTerms - 1) / kTerms;
  const int rows = a.rows - t0 < BT ? (int)(a.rows - t0) : BT, outs = a.n_out - o0 < BT ? a.n_out - o0 : BT;
  const long long ldw = TERM_ROWS ? a.n_out : a.k;
  const float* const from_t = static_cast<const float*>(a.A) + t0 * a.lda + k0;
  const float* const from_w = static_cast<const float*>(a.B) + (TERM_ROWS ? (long long)k0 * ldw + o0 : o0 * ldw + k0);

  // row side: thread's rows tid / 4 + 64 u, terms 4 (tid % 4) ..; term side: output tid % BT, terms 4 (NB (tid / BT) + u) ..
  const int row = threadIdx.x >> 2, quad = threadIdx.x & 3;
  const int out = threadIdx.x & (BT - 1), quad0 = NB * (threadIdx.x / BT);
  constexpr unsigned OUTSIDE = 0x80000000u;
  float rt[2][KS][NB][4], rw[2][KS][NB][4];      // two steps in flight
  auto gload = [&](float (&t)[NB][4], float (&w)[NB][4], int block) {
    const int left = block < n_blocks ? k_end - k0 - block * kTerms : 0;
    const auto rsrc_t = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from_t + (left ? block * kTerms : 0)), 0,
                                                          left ? (int)(((unsigned)(rows - 1) * (unsigned)a.lda + (unsigned)left) * 4u) : 0, 0x00020000);
    const unsigned col = quad * 4 < left ? quad * 16 : OUTSIDE;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const f32x4 v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc_t, (int)((unsigned)(row + 64 * u) * (unsigned)a.lda * 4u + col), 0, 0));
#pragma unroll
      for (int q = 0; q < 4; ++q) t[u][q] = v[q];
    }
    if constexpr (TERM_ROWS) {
      const int terms = left < kTerms ? left : kTerms;
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from_w + (left ? (long long)block * kTerms * ldw : 0)), 0,
                                                          left ? (int)(((unsigned)(terms - 1) * (unsigned)ldw + (unsigned)outs) * 4u) : 0, 0x00020000);
#pragma unroll
      for (int u = 0; u < NB; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          w[u][q] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)((unsigned)((quad0 + u) * 4 + q) * (unsigned)ldw * 4u + out * 4u), 0, 0));
    } else {
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from_w + (left ? block * kTerms : 0)), 0,
                                                          left ? (int)(((unsigned)(outs - 1) * (unsigned)ldw + (unsigned)left) * 4u) : 0, 0x00020000);
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const f32x4 v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)((unsigned)(row + 64 * u) * (unsigned)ldw * 4u + col), 0, 0));
#pragma unroll
        for (int q = 0; q < 4; ++q) w[u][q] = v[q];
      }
    }
  };

  // place of (row, half) in a side: the halves' rows swap fours, so that the 8-byte stores of sixteen lanes meet all banks
  auto place = [](int r, int half) { return (half * BT + (r ^ (half << 2))) * kUnit; };
  auto sstore = [&](auto split, const float (&t)[NB][4], const float (&w)[NB][4], int at) {
    if constexpr (split) {
      unsigned char* const to = lds + at;
      auto four = [&](const float (&x)[4], unsigned (&h)[2], unsigned (&m)[2], unsigned (&l)[2]) {
        split2(x[0], x[1], h[0], m[0], l[0]);
        split2(x[2], x[3], h[1], m[1], l[1]);
      };
      auto store = [&](unsigned char* at, const float (&x)[4]) {
        unsigned h[2], m[2], l[2];
        four(x, h, m, l);
        *reinterpret_cast<uint2*>(at) = make_uint2(h[0], h[1]);
        *reinterpret_cast<uint2*>(at + PLANE) = make_uint2(m[0], m[1]);
        *reinterpret_cast<uint2*>(at + 2 * PLANE) = make_uint2(l[0], l[1]);
      };
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        store(to + SIDE + place(row + 64 * u, quad >> 1) + 8 * (quad & 1), t[u]);
        if constexpr (!TERM_ROWS) store(to + place(row + 64 * u, quad >> 1) + 8 * (quad & 1), w[u]);
      }
      if constexpr (TERM_ROWS) {
        if constexpr (NB == 2) {
          unsigned h[2][2], m[2][2], l[2][2];
#pragma unroll
          for (int u = 0; u < 2; ++u) four(w[u], h[u], m[u], l[u]);
          unsigned char* const at = to + place(out, quad0 >> 1);
          *reinterpret_cast<uint4*>(at) = make_uint4(h[0][0], h[0][1], h[1][0], h[1][1]);
          *reinterpret_cast<uint4*>(at + PLANE) = make_uint4(m[0][0], m[0][1], m[1][0], m[1][1]);
          *reinterpret_cast<uint4*>(at + 2 * PLANE) = make_uint4(l[0][0], l[0][1], l[1][0], l[1][1]);
        } else {
          store(to + place(out, quad0 >> 1) + 8 * (quad0 & 1), w[0]);
        }
      }
    } else {
      float* const to = reinterpret_cast<float*>(lds + at);              // [term][outputs, tokens]
#pragma unroll
      for (int u = 0; u < NB; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          to[(quad * 4 + q) * 2 * BT + BT + row + 64 * u] = t[u][q];
          if constexpr (TERM_ROWS) to[((quad0 + u) * 4 + q) * 2 * BT + out] = w[u][q];
          else to[(quad * 4 + q) * 2 * BT + row + 64 * u] = w[u][q];
        }
    }
  };

  f32x16 acc[NB][NB];
  const int l31 = lane & 31, half = lane >> 5;
  auto compute = [&](auto split, int at) {
    if constexpr (split) {
      constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};          // small products first: lh, hl, mm, mh, hm, hh
      const unsigned char* const from = lds + at;
      bf16x8 w[NB][kParts], t[NB][kParts];
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int s = 0; s < kParts; ++s) {
          w[i][s] = *reinterpret_cast<const bf16x8*>(from + s * PLANE + place(wo * 32 * NB + i * 32 + l31, half));
          t[i][s] = *reinterpret_cast<const bf16x8*>(from + SIDE + s * PLANE + place(wt * 32 * NB + i * 32 + l31, half));
        }
#pragma unroll
      for (int s = 0; s < 6; ++s)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[i][pa[s]], t[j][pb[s]], acc[i][j], 0, 0, 0);
    } else {
      const float* const from = reinterpret_cast<const float*>(lds + at) + half * 2 * BT + l31;
#pragma unroll
      for (int k = 0; k < kTerms; k += 2) {
        float w[NB], t[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          w[i] = from[k * 2 * BT + wo * 32 * NB + i * 32];
          t[i] = from[k * 2 * BT + BT + wt * 32 * NB + i * 32];
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[i], t[j], acc[i][j], 0, 0, 0);
      }
    }
  };

  auto pass = [&](auto split) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    auto fetch = [&](float (&t)[KS][NB][4], float (&w)[KS][NB][4], int step) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < KS; ++q) gload(t[q], w[q], step * KS + q);
    };
    const int n_steps = (n_blocks + KS - 1) / KS;
    fetch(rt[0], rw[0], 0);
    fetch(rt[1], rw[1], 1);
#pragma unroll
    for (int q = 0; q < KS; ++q) sstore(split, rt[0][q], rw[0][q], q * BLOCK);
    __syncthreads();
    // the step in LDS buffer `buf` multiplied, the next one (in registers) split and stored in the other, the one after it fetched
    auto step = [&](int at, int buf, float (&t)[KS][NB][4], float (&w)[KS][NB][4], float (&t2)[KS][NB][4], float (&w2)[KS][NB][4]) __attribute__((always_inline)) {
      fetch(t2, w2, at + 2);
#pragma unroll
      for (int q = 0; q < KS; ++q) {
        compute(split, buf * STAGE + q * BLOCK);
        sstore(split, t[q], w[q], (buf ^ 1) * STAGE + q * BLOCK);
      }
      __syncthreads();
    };
    for (int at = 0; at < n_steps; at += 2) {
      step(at, 0, rt[1], rw[1], rt[0], rw[0]);
      if (at + 1 >= n_steps) break;
      step(at + 1, 1, rt[0], rw[0], rt[1], rw[1]);
    }
  };

  pass(std::true_type{});
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const unsigned bits = __builtin_bit_cast(unsigned, (float)acc[i][j][v]) & 0x7fffffffu;
        top = bits > top ? bits : top;
      }
  const bool again = __syncthreads_or(top >= 0x7f800000u);
  if (again) pass(std::false_type{});
  const float unit = again ? 1.f : kUnscale;

  // lane l holds token l % 32 and, of every eight outputs, four from 4 (l / 32) on.  `f` gets a column of blocks' bias and residual, which are
  // loaded all at once.
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    const bool whole = !p.parts;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      f32x4 bias[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int col = o0 + wo * 32 * NB + i * 32 + v * 8 + half * 4;
        bias[v] = whole && a.bias && col < a.n_out ? bias4(a.bias, col) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const long long r = t0 + wt * 32 * NB + j * 32 + l31;
        f32x4 res[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int col = o0 + wo * 32 * NB + i * 32 + v * 8 + half * 4;
          res[v] = whole && a.residual && r < a.rows && col < a.n_out ? load4(a.residual, r * a.ldr + col) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int col = o0 + wo * 32 * NB + i * 32 + v * 8 + half * 4;
          if (r < a.rows && col < a.n_out)
            f(r, col, f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]} * unit, bias[v], res[v]);
        }
      }
    }
  };
  finish_tile(p, part, each);
}

// A 64 x 64 tile by NW waves that share nothing until their sums: each takes every NW-th block of 16 terms through two stages of LDS of
// its own, filled by DMA, and splits the next block between this one's MFMAs.  The waves' sums are added in order through LDS.
template <int NW, bool TERM_ROWS>
__global__ __launch_bounds__(64 * NW, 2) void linear_wave_kernel(SplitParams p) {
  constexpr int BT = 64, NB = 2;
  constexpr unsigned SIDE = BT * kTerms * 4, STAGE = 2 * SIDE;             // outputs' side, then tokens'
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const LinearArgs& a = p.a;
  if (blockIdx.x >= p.workgroups) {
    row_sum<64 * NW>(a.then, blockIdx.x - p.workgroups, reinterpret_cast<float*>(lds));
    return;
  }
  const int id = (int)xcd_contiguous(blockIdx.x, p.workgroups);
  const int part = id / p.tiles;
  int tile_t, tile_o;
  tile_coords<0>(id - part * p.tiles, p.grid, tile_t, tile_o);
  const long long t0 = (long long)tile_t * BT;
  const int o0 = tile_o * BT;
  const int k0 = part * p.blocks_per_part * kTerms;
  const int k_end = a.k - k0 < p.blocks_per_part * kTerms ? a.k : k0 + p.blocks_per_part * kTerms;
  const int n_blocks = (k_end - k0 + kTerms - 1) / kTerms;
  const int n_mine = (n_blocks - wave + NW - 1) / NW;
  const int rows = a.rows - t0 < BT ? (int)(a.rows - t0) : BT, outs = a.n_out - o0 < BT ? a.n_out - o0 : BT;
  const long long ldw = TERM_ROWS ? a.n_out : a.k;
  const float* const from_t = static_cast<const float*>(a.A) + t0 * a.lda + k0;
  const float* const from_w = static_cast<const float*>(a.B) + (TERM_ROWS ? (long long)k0 * ldw + o0 : o0 * ldw + k0);
  const int l31 = lane & 31, half = lane >> 5;
  constexpr unsigned OUTSIDE = 0x80000000u;      // past every descriptor

  // Loads of 1 KiB: 16 rows' 64 bytes (or, of W's term rows, four terms' 256).  LDS keeps a row's four columns of 16 bytes in an order that
  // changes every fourth row, so that eight lanes reading one column of eight rows meet all banks.
  const int row = lane >> 2, col = (lane & 3) ^ (row >> 2);
  unsigned off_t[4], off_w[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    off_t[q] = (unsigned)(q * 16 + row) * (unsigned)a.lda * 4u + col * 16u;
    off_w[q] = TERM_ROWS ? (unsigned)(q * 4 + (lane >> 4)) * (unsigned)ldw * 4u + (lane & 15) * 16u : (unsigned)(q * 16 + row) * (unsigned)ldw * 4u + col * 16u;
  }
  const unsigned mine = (unsigned)(size_t)(lds_void_ptr)lds + (unsigned)wave * (2 * STAGE);
  auto fetch = [&](unsigned stage, int block) __attribute__((always_inline)) {
    const int left = block < n_blocks ? k_end - k0 - block * kTerms : 0, terms = left < kTerms ? left : kTerms;
    auto rsrc = [](const float* from, unsigned floats) {
      const unsigned long long v = (unsigned long long)from;
      v4i r;
      r[0] = __builtin_amdgcn_readfirstlane((int)(unsigned)v);
      r[1] = __builtin_amdgcn_readfirstlane((int)((unsigned)(v >> 32) & 0xffffu));
      r[2] = __builtin_amdgcn_readfirstlane((int)(floats * 4u));
      r[3] = 0x00020000;
      return r;
    };
    const v4i t = rsrc(from_t + (left ? block * kTerms : 0), left ? (unsigned)(rows - 1) * (unsigned)a.lda + (unsigned)left : 0u);
    const v4i w = TERM_ROWS ? rsrc(from_w + (left ? (long long)block * kTerms * ldw : 0), left ? (unsigned)(terms - 1) * (unsigned)ldw + (unsigned)outs : 0u)
                            : rsrc(from_w + (left ? block * kTerms : 0), left ? (unsigned)(outs - 1) * (unsigned)ldw + (unsigned)left : 0u);
    const bool in = col * 4 < left;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      load_lds16(w, mine + stage * STAGE + q * 1024, TERM_ROWS || in ? off_w[q] : OUTSIDE);
      load_lds16(t, mine + stage * STAGE + SIDE + q * 1024, in ? off_t[q] : OUTSIDE);
    }
  };
  float rt[NB][8], rw[NB][8];                    // a block: lane's terms 8 (lane / 32) .. of its two rows
  auto read = [&](unsigned stage) __attribute__((always_inline)) {
    const unsigned char* const from = lds + wave * (2 * STAGE) + stage * STAGE;
    auto rows_of = [&](float (&x)[NB][8], const unsigned char* side) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < NB; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(side + (u * 32 + l31) * 64 + (((half * 2 + h) ^ ((l31 >> 2) & 3)) << 4));
#pragma unroll
          for (int q = 0; q < 4; ++q) x[u][h * 4 + q] = v[q];
        }
    };
    if constexpr (TERM_ROWS) {
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int u = 0; u < NB; ++u) rw[u][q] = *reinterpret_cast<const float*>(from + (half * 8 + q) * 256 + (u * 32 + l31) * 4);
    } else {
      rows_of(rw, from);
    }
    rows_of(rt, from + SIDE);
  };
  // a stage's loads have arrived but for those of the one issued after it; its reads have arrived before it is filled again
  auto next = [&](unsigned stage, int block) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    read(stage);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    fetch(stage, block);
  };

  typedef unsigned Parts[kParts][4];
  auto split8 = [&](const float (&x)[8], Parts& to) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < 4; ++q) split2(x[2 * q], x[2 * q + 1], to[0][q], to[1][q], to[2][q]);
  };
  auto operand = [](const unsigned (&x)[4]) __attribute__((always_inline)) {
    const uint4 v = make_uint4(x[0], x[1], x[2], x[3]);
    return __builtin_bit_cast(bf16x8, v);
  };

  f32x16 acc[NB][NB];
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  };
  clear();
  Parts w[2][NB], t[2][NB];
  fetch(0, wave);
  fetch(1, wave + NW);
  next(0, wave + 2 * NW);
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    split8(rw[u], w[0][u]);
    split8(rt[u], t[0][u]);
  }
  // the parts in set `now` multiplied, the next block read and split into the other set, the third after it fetched
  auto step = [&](auto now, int at) __attribute__((always_inline)) {
    constexpr int c = decltype(now)::value, n = c ^ 1;
    constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};            // small products first: lh, hl, mm, mh, hm, hh
    next(n, wave + NW * (at + 3));
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      split8(rw[u], w[n][u]);
      split8(rt[u], t[n][u]);
    }
#pragma unroll
    for (int s = 0; s < 6; ++s)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(w[c][i][pa[s]]), operand(t[c][j][pb[s]]), acc[i][j], 0, 0, 0);
  };
  for (int at = 0; at < n_mine; at += 2) {
    step(std::integral_constant<int, 0>{}, at);
    if (at + 1 >= n_mine) break;
    step(std::integral_constant<int, 1>{}, at + 1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const unsigned bits = __builtin_bit_cast(unsigned, (float)acc[i][j][v]) & 0x7fffffffu;
        top = bits > top ? bits : top;
      }
  const bool again = __syncthreads_or(top >= 0x7f800000u);
  if (again) {
    clear();
    for (int at = 0; at < n_mine; ++at) {
      fetch(0, wave + NW * at);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      read(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(rw[i][q], rt[j][q], acc[i][j], 0, 0, 0);
    }
  }

  // [wave][unit][lane] (a wave's in its own stages), a unit four outputs of a block of 32 x 32: a wave adds and finishes 16 / NW units
  constexpr int NU = 16 / NW;
  f32x4* const sums = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        sums[(wave * 16 + (i * 2 + j) * 4 + v) * 64 + lane] = f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]};
  const int first = wave * NU;
  const float unit = again ? 1.f : kUnscale;
  const bool whole = !p.parts;
  auto row_of = [&](int u) { return t0 + ((first + u) >> 2 & 1) * 32 + l31; };
  auto col_of = [&](int u) { return o0 + ((first + u) >> 3) * 32 + ((first + u) & 3) * 8 + half * 4; };
  f32x4 bias[NU], res[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const long long r = row_of(u);
    const int col = col_of(u);
    bias[u] = whole && a.bias && col < a.n_out ? bias4(a.bias, col) : f32x4{0.f, 0.f, 0.f, 0.f};
    res[u] = whole && a.residual && r < a.rows && col < a.n_out ? load4(a.residual, r * a.ldr + col) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();
  auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      f32x4 z = sums[(first + u) * 64 + lane];
#pragma unroll
      for (int q = 1; q < NW; ++q) z += sums[(q * 16 + first + u) * 64 + lane];
      const long long r = row_of(u);
      const int col = col_of(u);
      if (r < a.rows && col < a.n_out) f(r, col, z * unit, bias[u], res[u]);
    }
  };
  finish_tile(p, part, each);
}

template <Act A>
__global__ __launch_bounds__(256) void linear_f32_parts_kernel(LinearArgs a, const float* __restrict__ parts, int n_parts) {
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4, n = a.rows * a.n_out;
  if (i >= n) return;
  f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int q = 0; q < n_parts; ++q) z += *reinterpret_cast<const f32x4*>(parts + (size_t)q * n + i);
  const long long row = i / a.n_out;
  const int col = (int)(i - row * a.n_out);
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  finish4<A>(a, row, col, z, a.bias ? bias4(a.bias, col) : zero, a.residual ? load4(a.residual, row * a.ldr + col) : zero);
}

enum class Tile { k128, k64, k64By4, k64By8 };      // By: by waves that split the sum
constexpr int side_of(Tile t) { return t == Tile::k128 ? 128 : 64; }
constexpr int sum_waves_of(Tile t) { return t == Tile::k64By4 ? 4 : t == Tile::k64By8 ? 8 : 1; }

// Tiles and parts of a product: the smallest modelled time, in microseconds.  A workgroup costs a start and, per block or block of each wave, what
// it takes of its compute unit: 128 x 128 tiles, three to a unit, 2 and 0.64 (alone 0.75); 64 x 64, 1 and 0.23 (alone 0.3); by four waves that split
// the sum 2.5 (alone 1.5) and 0.79; by eight, where none waits for a unit, 1.5 and 1.45.  Parts cost a second launch, 0.12 each and the workspace's
// traffic at 8 bytes per output and part (a little much beside the kernels' time, as the second launch costs the host more).  With 4 us for the
// launch it is 14 % below to 28 % above what was measured on 40 products of 1 .. 40000 tokens.  Past one full round it takes rounds as divisible,
// which they are on many: a few workgroups behind a full round cost more than it says (9999 x 1536 -> 1536: 235 modelled, 255 measured).
LinearPlan plan(long long rows, int k, int n_out, bool may_split) {
  const int blocks = (k + kTerms - 1) / kTerms;
  const double outputs = (double)rows * n_out;
  LinearPlan best = {rows, 128, 1, 1, blocks};
  double least = 1e300;
  for (const Tile tile : {Tile::k128, Tile::k64, Tile::k64By4, Tile::k64By8}) {
    const int side = side_of(tile);
    const double tiles = (double)((rows + side - 1) / side) * ((n_out + side - 1) / side);
    for (const int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (want > 1 && (!may_split || want > blocks / 4 || tiles * want > 2048.0)) break;
      const int per = (blocks + want - 1) / want, parts = (blocks + per - 1) / per;
      const double wgs = tiles * parts, rounds = wgs <= 768.0 ? std::ceil(wgs / 256.0) : wgs / 256.0;
      const bool alone = wgs <= 256.0;
      if (tile == Tile::k64By8 && !alone) break;
      const double one = tile == Tile::k128    ? 2.0 + (alone ? 0.75 : 0.64) * per
                         : tile == Tile::k64   ? 1.0 + (alone ? 0.30 : 0.23) * per
                         : tile == Tile::k64By4 ? (alone ? 1.5 : 2.5) + 0.79 * ((per + 3) / 4)
                                                : 1.5 + 1.45 * ((per + 7) / 8);
      const double time = one * rounds + (parts > 1 ? 3.0 + parts * (0.12 + outputs * 1e-6) : 0.0);
      if (time < least) {
        least = time;
        best = {rows, side, sum_waves_of(tile), parts, per};
      }
    }
  }
  return best;
}

template <typename Kernel>
hipError_t launch(Kernel kern, unsigned blocks, int waves, size_t smem, const SplitParams& p, hipStream_t s) {
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(64 * waves), smem, s, p);
  return hipGetLastError();
}

template <int NB, int KS, bool TERM_ROWS>
hipError_t launch_split(const SplitParams& p, unsigned blocks, hipStream_t s) {
  constexpr size_t smem = (size_t)2 * KS * kParts * 4 * 64 * NB * kUnit;
  auto kern = linear_split_kernel<NB, KS, TERM_ROWS>;
  // once per process and instantiation (static initialisation is thread-safe); a failure is returned by every call
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  return attr != hipSuccess ? attr : launch(kern, blocks, 4, smem, p, s);
}

template <int NW, bool TERM_ROWS>
hipError_t launch_wave(const SplitParams& p, unsigned blocks, hipStream_t s) {
  constexpr size_t smem = (size_t)NW * 64 * 64 * sizeof(float);
  auto kern = linear_wave_kernel<NW, TERM_ROWS>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  return attr != hipSuccess ? attr : launch(kern, blocks, NW, smem, p, s);
}

template <bool TERM_ROWS>
hipError_t launch_plan(const SplitParams& p, const LinearPlan& pl, unsigned blocks, hipStream_t s) {
  if (pl.side == 128) return launch_split<2, 1, TERM_ROWS>(p, blocks, s);
  if (pl.sum_waves == 1) return launch_split<1, 2, TERM_ROWS>(p, blocks, s);
  return pl.sum_waves == 4 ? launch_wave<4, TERM_ROWS>(p, blocks, s) : launch_wave<8, TERM_ROWS>(p, blocks, s);
}

}  // namespace

LinearPlan linear_split_plan(long long rows, int k, int n_out, bool may_split) { return plan(rows, k, n_out, may_split); }

hipError_t launch_linear_split(const LinearArgs& a, const LinearPlan& pl, hipStream_t s) {
  SplitParams p;
  p.a = a;
  const long long mt = (a.rows + pl.side - 1) / pl.side, nt = (a.n_out + pl.side - 1) / pl.side;
  if (mt * nt * pl.parts > 0x7fffffffLL) return hipErrorInvalidValue;
  p.grid = tile_grid((int)mt, (int)nt);
  p.tiles = (int)(mt * nt);
  p.blocks_per_part = pl.blocks_per_part;
  p.parts = pl.parts > 1 ? a.workspace : nullptr;
  p.workgroups = (unsigned)(p.tiles * pl.parts);
  const unsigned blocks = p.workgroups + row_sum_blocks(a.then);
  const hipError_t e = a.b_rows_are_k ? launch_plan<true>(p, pl, blocks, s) : launch_plan<false>(p, pl, blocks, s);
  if (e != hipSuccess || pl.parts == 1) return e;
  const long long threads = a.rows * a.n_out / 4;
  with_act(a.act, [&](auto act) {
    hipLaunchKernelGGL(linear_f32_parts_kernel<decltype(act)::value>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, p.parts, pl.parts);
  });
  return hipGetLastError();
}

}  // namespace isopo
