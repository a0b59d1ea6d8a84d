// Host-callable launchers of the operators around the layer step: linear layer, token log-probability, AdamW.  Internal to the
// library: the public surface is include/isopo.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/isopo.h"

namespace isopo {

enum class Act;

constexpr long long kLastLevelCache = 256LL << 20;     // bytes

// out [cols] = the sum of `n` rows of parts [n, cols], in order: what act_backward leaves for db.  n 0: nothing to do.
struct RowSum {
  const float* parts = nullptr;
  float* out = nullptr;
  int n = 0, cols = 0;
};

// C = act(A B^T + bias) + residual (b_rows_are_k false: B is [n_out, k]) or C = A B (true: B is [k, n_out]).
struct LinearArgs {
  const void* A;               // [rows, k], rows lda apart
  const void* B;               // dense
  const void* bias;            // [n_out] or NULL
  const void* residual;        // [rows, n_out], rows ldr apart, or NULL
  void* C;                     // rows ldc apart
  void* Z;                     // dense [rows, n_out] or NULL: what the activation is applied to
  long long rows, lda, ldr, ldc;
  int k, n_out;
  bool bf16, b_rows_are_k;
  Act act;
  float* workspace;
  RowSum then;                 // formed by workgroups of the same launch behind the product's
};
// One launch of a product.
struct LinearPlan {
  long long rows;              // its rows
  int side;                    // outputs and tokens of a tile
  int sum_waves;               // waves that split a tile's sum (1: they share its blocks)
  int parts, blocks_per_part;  // of the sum, by different workgroups; parts 1: it is whole
};
// The launch that starts at row `first` (0, or where the launch before ends).
LinearPlan linear_plan(long long rows, int k, int n_out, bool bf16, long long first);
size_t linear_workspace(const LinearPlan& p, int n_out);
hipError_t launch_linear(const LinearArgs& a, hipStream_t s);
// bf16, tiles of 128 or 256 outputs and tokens (launch_linear routes to it).  may_split false: there is no workspace for parts.
LinearPlan linear_tile_plan(long long rows, int k, int n_out, bool may_split);
hipError_t launch_linear_tile(const LinearArgs& a, const LinearPlan& pl, hipStream_t s);
// fp32, tiles of 64 or 128
LinearPlan linear_split_plan(long long rows, int k, int n_out, bool may_split);
hipError_t launch_linear_split(const LinearArgs& a, const LinearPlan& pl, hipStream_t s);

// Delta = dY act'(Z) (NULL: not written) and its column sums (db NULL: none).  *rest: NULL, or set to what is left to sum for db.
struct ActBackwardArgs {
  const void* dY;              // rows ldy apart
  const void* Z;               // dense
  void* Delta;                 // dense
  float* db;
  float* workspace;            // act_backward_workspace bytes, with db
  long long rows, ldy;
  int cols;
  bool bf16;
  Act act;
};
size_t act_backward_workspace(long long rows, int cols);
hipError_t launch_act_backward(const ActBackwardArgs& a, hipStream_t s, RowSum* rest);

struct TokenLogprobArgs {
  const void* logits;
  bool bf16;
  long long n_tokens, ld, ldd;
  int vocab;
  const int32_t* targets;
  float inv_temperature;
  float* logp;                 // outputs of the forward pass, each may be NULL
  float* lse;
  float* entropy;
  const float* weight;         // with dlogits
  void* dlogits;
};
hipError_t launch_token_logprob(const TokenLogprobArgs& a, hipStream_t s);

struct TokenLogprobBackwardArgs {
  const void* logits;
  bool bf16;
  long long n_tokens, ld, ldd;
  int vocab;
  const int32_t* targets;
  float inv_temperature;
  const float* lse;
  const float* grad_logp;
  const float* entropy;        // both or neither
  const float* grad_entropy;
  void* dlogits;
};
hipError_t launch_token_logprob_backward(const TokenLogprobBackwardArgs& a, hipStream_t s);

struct AdamwArgs {
  const isopo_adamw_tensor* tensors;  // host
  const void* const* grads;    // host
  int n_tensors;
  bool param_bf16, grad_bf16, bits8, maximize;
  double lr, beta1, beta2, eps, weight_decay, max_norm;
  long long step;
  uint32_t seed;
  float* norm = nullptr;       // NULL: gradients are taken as they are
  const double* norm_parts = nullptr; // NULL: norm is there;  else what launch_grad_norm left to sum, for norm to be written
  int n_norm_parts = 0;
};
hipError_t launch_adamw(const AdamwArgs& a, hipStream_t s);
size_t grad_norm_workspace(const isopo_adamw_tensor* tensors, int n_tensors);
// few: NULL, or set to how many parts in the workspace are left to the update to sum (0: norm is written).
hipError_t launch_grad_norm(const isopo_adamw_tensor* tensors, const void* const* grads, int n_tensors, bool bf16, float* norm, double* workspace,
                            hipStream_t s, int* few);
hipError_t launch_adamw_state(const void* m, const float* m_scale, const void* v, const float* v_scale, long long n, bool bf16, void* m_out,
                              void* v_out, hipStream_t s);

}  // namespace isopo
