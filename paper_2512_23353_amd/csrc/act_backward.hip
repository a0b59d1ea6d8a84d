// Delta = dY act'(Z), what the layer step and dX are formed from, and db = sum over tokens of Delta, in one pass over dY and Z.
//
// bf16: Delta is rounded, and dX formed from the rounded one, the MFMA's operand: two parts of each value would double the product's time (9999 x
// 8960 x 1536: 200 us).  dX is then 0.0023 from the 64-bit form in norm, where rounding itself costs 0.0017; dW sees the same Delta.
//
// Bound by HBM: 9999 x 8960 bf16, 538 MB, 90 us, 6.0 TB/s.  A workgroup takes 32 vectors of 16 bytes side by side and a chunk of
// rows, eight rows at a time; db's sums are formed from the unrounded products, in fp32: per thread, over the eight rows in LDS, and
// over the chunks, always in the same order.  The sum over the chunks is no launch of its own where dX is formed: workgroups behind
// those of its product take it (512^3 bf16, whole backward call: 16.7 us with the launch, 14.2 us without).
#include "activation.h"
#include "policy.h"
#include "row_sum.h"

namespace isopo {
namespace {

constexpr int kVecs = 32, kRows = 8;
constexpr int kOneChunk = 128;           // up to so many rows one workgroup's sums are db's: no second launch
// rows of a chunk: enough chunks to fill the chip, not so many that their sums weigh
long long chunk_rows(long long rows, int cols) {
  if (rows <= kOneChunk) return kOneChunk;
  const long long wide = (cols + 255) / 256;
  long long c = (rows * wide + 1023) / 1024;
  c = (c + kRows - 1) / kRows * kRows;
  return c < 64 ? 64 : c;
}
long long chunks_of(long long rows, int cols) { return (rows + chunk_rows(rows, cols) - 1) / chunk_rows(rows, cols); }

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <bool ONCE, class V>
__device__ __forceinline__ V load(const void* at) {
  if constexpr (ONCE) return __builtin_nontemporal_load(static_cast<const V*>(at));
  else return *static_cast<const V*>(at);
}

struct Params {
  ActBackwardArgs a;
  long long chunk;
};

// ONCE: dY and Z are read for the last time and need not be kept in the caches.
template <bool BF16, Act A, bool ONCE>
__global__ __launch_bounds__(256) void act_backward_kernel(Params p) {
  constexpr int V = BF16 ? 8 : 4;
  __shared__ float red[kRows][kVecs * V + 4];
  const ActBackwardArgs& a = p.a;
  const int vec = threadIdx.x % kVecs, row = threadIdx.x / kVecs;
  const int col = (blockIdx.x * kVecs + vec) * V;
  const long long r0 = blockIdx.y * p.chunk, r1 = r0 + p.chunk < a.rows ? r0 + p.chunk : a.rows;
  float sum[V] = {};
  if (col < a.cols) {
    for (long long r = r0 + row; r < r1; r += kRows) {
      float d[V];
      if constexpr (BF16) {
        const u32x4 w = load<ONCE, u32x4>(static_cast<const unsigned short*>(a.dY) + r * a.ldy + col);
        u32x4 z = {0, 0, 0, 0};
        if constexpr (A != Act::kNone) z = load<ONCE, u32x4>(static_cast<const unsigned short*>(a.Z) + r * a.cols + col);
        unsigned o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          d[2 * q] = __builtin_bit_cast(float, (unsigned)w[q] << 16) * act_slope<A>(__builtin_bit_cast(float, (unsigned)z[q] << 16));
          d[2 * q + 1] = __builtin_bit_cast(float, (unsigned)w[q] & 0xffff0000u) * act_slope<A>(__builtin_bit_cast(float, (unsigned)z[q] & 0xffff0000u));
          o[q] = (unsigned)f32_to_bf16_bits(d[2 * q]) | (unsigned)f32_to_bf16_bits(d[2 * q + 1]) << 16;
        }
        if (a.Delta) *reinterpret_cast<uint4*>(static_cast<unsigned short*>(a.Delta) + r * a.cols + col) = make_uint4(o[0], o[1], o[2], o[3]);
      } else {
        const f32x4 x = load<ONCE, f32x4>(static_cast<const float*>(a.dY) + r * a.ldy + col);
        f32x4 z = {0.f, 0.f, 0.f, 0.f};
        if constexpr (A != Act::kNone) z = load<ONCE, f32x4>(static_cast<const float*>(a.Z) + r * a.cols + col);
        f32x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = d[q] = x[q] * act_slope<A>(z[q]);
        if (a.Delta) *reinterpret_cast<f32x4*>(static_cast<float*>(a.Delta) + r * a.cols + col) = o;
      }
#pragma unroll
      for (int q = 0; q < V; ++q) sum[q] += d[q];
    }
  }
  if (!a.db) return;
#pragma unroll
  for (int q = 0; q < V; ++q) red[row][vec * V + q] = sum[q];
  __syncthreads();
  const int c0 = blockIdx.x * kVecs * V, c = threadIdx.x;
  if (c < kVecs * V && c0 + c < a.cols) {
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) t += red[r][c];
    if (gridDim.y == 1) a.db[c0 + c] = t;
    else a.workspace[(size_t)blockIdx.y * a.cols + c0 + c] = t;
  }
}

constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void row_sum_kernel(RowSum r) {
  __shared__ float lds[kSumThreads];
  row_sum<kSumThreads>(r, blockIdx.x, lds);
}

}  // namespace

size_t act_backward_workspace(long long rows, int cols) {
  const long long chunks = chunks_of(rows, cols);
  return chunks > 1 ? (size_t)chunks * cols * sizeof(float) : 0;
}

hipError_t launch_act_backward(const ActBackwardArgs& a, hipStream_t s, RowSum* rest) {
  const int per = kVecs * (a.bf16 ? 8 : 4);
  const long long chunks = chunks_of(a.rows, a.cols);
  if (chunks > 65535) return hipErrorInvalidValue;
  if (a.rows > 0) {
    const Params p = {a, chunk_rows(a.rows, a.cols)};
    const dim3 grid((a.cols + per - 1) / per, (unsigned)chunks);
    // Where dY, Z and Delta are more than the last-level cache holds, the first two are not kept there: Delta is, for the product that reads it
    // next (act "none": dY is that).  9999 x 8960 x 1536 bf16, whole backward call 303 -> 284 us; between the products before and after it 774 ->
    // 768.  Smaller ones found there again: 2048^3 30.5 against 33.4.
    const bool once = 3 * a.rows * a.cols * (a.bf16 ? 2 : 4) > kLastLevelCache;
    with_act(a.act, [&](auto act) {
      constexpr Act A = decltype(act)::value;
      const auto go = [&](auto bf16) {
        constexpr bool BF16 = decltype(bf16)::value;
        if (once) hipLaunchKernelGGL((act_backward_kernel<BF16, A, A != Act::kNone>), grid, dim3(256), 0, s, p);
        else hipLaunchKernelGGL((act_backward_kernel<BF16, A, false>), grid, dim3(256), 0, s, p);
      };
      if (a.bf16) go(std::true_type{});
      else go(std::false_type{});
    });
  }
  if (a.db && chunks != 1) {             // (no rows: sums of nothing)
    RowSum sum;
    sum.parts = a.workspace; sum.out = a.db; sum.n = (int)chunks; sum.cols = a.cols;
    if (rest && chunks > 1) *rest = sum;
    else hipLaunchKernelGGL(row_sum_kernel, dim3((a.cols + 63) / 64), dim3(kSumThreads), 0, s, sum);
  }
  return hipGetLastError();
}

}  // namespace isopo
