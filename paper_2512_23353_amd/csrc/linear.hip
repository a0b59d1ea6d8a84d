// Which kernel forms a linear layer's product, and in how many launches.
#include "policy.h"

namespace isopo {
namespace {

// Rows of one launch: a grid holds no more than 2^32 threads (tens of millions of tokens of a narrow layer have more tiles than that).
constexpr long long kTilesPerLaunch = 1 << 22;
long long rows_per_launch(int n_out) {
  const long long across = (n_out + 63) / 64;
  return (kTilesPerLaunch / across + 1) / 4 * 256 + 256;
}

}  // namespace

// The launches of a product that is cut split no sums, however few rows the last one has: they share the call's workspace, which holds no parts.
LinearPlan linear_plan(long long rows, int k, int n_out, bool bf16, long long first) {
  const long long most = rows_per_launch(n_out), here = rows - first < most ? rows - first : most;
  const bool may_split = rows <= most;
  return bf16 ? linear_tile_plan(here, k, n_out, may_split) : linear_split_plan(here, k, n_out, may_split);
}

size_t linear_workspace(const LinearPlan& p, int n_out) { return p.parts > 1 ? (size_t)p.parts * p.rows * n_out * sizeof(float) : 0; }

hipError_t launch_linear(const LinearArgs& a, hipStream_t s) {
  const size_t e = a.bf16 ? 2 : 4;
  for (long long r = 0; r < a.rows;) {
    const LinearPlan pl = linear_plan(a.rows, a.k, a.n_out, a.bf16, r);
    if (pl.parts > 1 && !a.workspace) return hipErrorInvalidValue;
    LinearArgs b = a;
    if (r > 0) b.then = RowSum();
    b.rows = pl.rows;
    b.A = static_cast<const char*>(a.A) + r * a.lda * e;
    b.C = static_cast<char*>(a.C) + r * a.ldc * e;
    if (a.Z) b.Z = static_cast<char*>(a.Z) + r * a.n_out * e;
    if (a.residual) b.residual = static_cast<const char*>(a.residual) + r * a.ldr * e;
    const hipError_t err = a.bf16 ? launch_linear_tile(b, pl, s) : launch_linear_split(b, pl, s);
    if (err != hipSuccess) return err;
    r += pl.rows;
  }
  return hipSuccess;
}

}  // namespace isopo
