// C ABI of the operators around the layer step: argument checks and workspace layout.  No arithmetic of an operator lives here.
#include <cstring>

#include "activation.h"
#include "policy.h"

namespace {

using namespace isopo;

constexpr long long kMaxTokens = 0x7fffffffLL;
constexpr int64_t kMaxPitch = ((int64_t)1 << 22) - 8;   // elements: the 256 rows of a tile stay within 2^31 bytes, the buffer loads' offsets

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }

// An enum argument may hold any int: its bytes are looked at before anything loads it as the enum type.
template <class E>
bool enum_in(const E& e, int lo, int hi) {
  static_assert(sizeof(E) == sizeof(int), "C enums of this header are ints");
  int v;
  std::memcpy(&v, &e, sizeof v);
  return v >= lo && v <= hi;
}

isopo_status of(hipError_t e) { return e == hipSuccess ? ISOPO_OK : ISOPO_ERR_HIP; }

isopo_status check_shape(int64_t n, int32_t d_in, int32_t d_out, const isopo_dtype& dtype) {
  if (!enum_in(dtype, ISOPO_F32, ISOPO_BF16)) return ISOPO_ERR_UNSUPPORTED;
  if (n < 0 || d_in <= 0 || d_out <= 0) return ISOPO_ERR_INVALID_ARG;
  const int vec = dtype == ISOPO_BF16 ? 8 : 4;
  if (n > kMaxTokens || d_in % vec || d_out % vec || d_in > kMaxPitch || d_out > kMaxPitch) return ISOPO_ERR_UNSUPPORTED;
  return ISOPO_OK;
}

// A row pitch as given (0: dense); false where it cannot be one.
bool pitch(int64_t given, int32_t row, int vec, long long* out) {
  *out = given ? given : row;
  return *out >= row && *out % vec == 0 && *out <= kMaxPitch;
}

bool check_ws(const void* ws, size_t have, size_t need, isopo_status* st) {
  *st = ISOPO_OK;
  if (!need) return true;
  if (!ws || !aligned(ws, 256)) *st = ISOPO_ERR_INVALID_ARG;
  else if (have < need) *st = ISOPO_ERR_WORKSPACE_TOO_SMALL;
  return *st == ISOPO_OK;
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

Act act_of(isopo_activation a) { return static_cast<Act>(a); }
static_assert((int)Act::kNone == ISOPO_ACT_NONE && (int)Act::kRelu == ISOPO_ACT_RELU && (int)Act::kGelu == ISOPO_ACT_GELU &&
              (int)Act::kSilu == ISOPO_ACT_SILU, "one numbering");

}  // namespace

extern "C" {

size_t isopo_linear_workspace(int64_t n_tokens, int32_t d_in, int32_t d_out, isopo_dtype dtype) {
  if (check_shape(n_tokens, d_in, d_out, dtype) != ISOPO_OK || n_tokens == 0) return 0;
  return linear_workspace(linear_plan(n_tokens, d_in, d_out, dtype == ISOPO_BF16, 0), d_out);
}

size_t isopo_linear_backward_workspace(int64_t n_tokens, int32_t d_in, int32_t d_out, isopo_dtype dtype) {
  if (check_shape(n_tokens, d_in, d_out, dtype) != ISOPO_OK || n_tokens == 0) return 0;
  return align_up(act_backward_workspace(n_tokens, d_out)) + linear_workspace(linear_plan(n_tokens, d_out, d_in, dtype == ISOPO_BF16, 0), d_in);
}

isopo_status isopo_linear_plan(int64_t n_tokens, int32_t d_in, int32_t d_out, isopo_dtype dtype, int32_t backward, int64_t first_token,
                               isopo_linear_plan_info* plan) {
  const isopo_status st = check_shape(n_tokens, d_in, d_out, dtype);
  if (st != ISOPO_OK) return st;
  if (!plan || first_token < 0 || first_token >= n_tokens) return ISOPO_ERR_INVALID_ARG;
  const int k = backward ? d_out : d_in, n_out = backward ? d_in : d_out;
  const LinearPlan head = linear_plan(n_tokens, k, n_out, dtype == ISOPO_BF16, 0);
  if (first_token % head.rows) return ISOPO_ERR_INVALID_ARG;
  const LinearPlan p = linear_plan(n_tokens, k, n_out, dtype == ISOPO_BF16, first_token);
  plan->tokens = p.rows;
  plan->tile = p.side;
  plan->sum_waves = p.sum_waves;
  plan->parts = p.parts;
  plan->workspace_end = linear_workspace(p, n_out);
  if (backward && p.parts > 1) plan->workspace_end += align_up(act_backward_workspace(n_tokens, d_out));
  return ISOPO_OK;
}

isopo_status isopo_linear(const isopo_linear_layer* l, void* Y, void* Z, void* workspace, size_t ws_bytes, void* stream) {
  if (!l) return ISOPO_ERR_INVALID_ARG;
  isopo_status st = check_shape(l->n_tokens, l->d_in, l->d_out, l->dtype);
  if (st != ISOPO_OK) return st;
  if (!enum_in(l->act, ISOPO_ACT_NONE, ISOPO_ACT_SILU)) return ISOPO_ERR_INVALID_ARG;
  LinearArgs a;
  const bool bf16 = l->dtype == ISOPO_BF16;
  const int vec = bf16 ? 8 : 4;
  if (!pitch(l->ldx, l->d_in, vec, &a.lda) || !pitch(l->ldr, l->d_out, vec, &a.ldr) || !pitch(l->ldy, l->d_out, vec, &a.ldc))
    return ISOPO_ERR_INVALID_ARG;
  if (l->n_tokens == 0) return ISOPO_OK;
  if (!l->X || !l->W || !Y) return ISOPO_ERR_INVALID_ARG;
  if (!aligned16(l->X) || !aligned16(l->W) || !aligned16(Y) || !aligned16(Z) || !aligned16(l->residual) || !aligned(l->bias, bf16 ? 2 : 4))
    return ISOPO_ERR_INVALID_ARG;
  if (Y == l->X || Z == Y || (Z && (Z == l->X || Z == l->residual)) || (l->residual == Y && a.ldr != a.ldc)) return ISOPO_ERR_INVALID_ARG;
  if (!check_ws(workspace, ws_bytes, isopo_linear_workspace(l->n_tokens, l->d_in, l->d_out, l->dtype), &st)) return st;
  a.A = l->X; a.B = l->W; a.bias = l->bias; a.residual = l->residual; a.C = Y; a.Z = Z;
  a.rows = l->n_tokens; a.k = l->d_in; a.n_out = l->d_out;
  a.bf16 = bf16; a.b_rows_are_k = false; a.act = act_of(l->act); a.workspace = static_cast<float*>(workspace);
  return of(launch_linear(a, static_cast<hipStream_t>(stream)));
}

isopo_status isopo_linear_backward(const void* dY, int64_t lddy, const void* W, const void* Z, isopo_dtype dtype, isopo_activation act,
                                   int64_t n_tokens, int32_t d_in, int32_t d_out, void* Delta, void* dX, float* db,
                                   void* workspace, size_t ws_bytes, void* stream) {
  isopo_status st = check_shape(n_tokens, d_in, d_out, dtype);
  if (st != ISOPO_OK) return st;
  if (!enum_in(act, ISOPO_ACT_NONE, ISOPO_ACT_SILU)) return ISOPO_ERR_INVALID_ARG;
  const bool bf16 = dtype == ISOPO_BF16;
  ActBackwardArgs b;
  if (!pitch(lddy, d_out, bf16 ? 8 : 4, &b.ldy)) return ISOPO_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (n_tokens > 0) {
    if (!dY || !aligned16(dY) || !aligned16(Delta) || !aligned16(dX)) return ISOPO_ERR_INVALID_ARG;
    if (act != ISOPO_ACT_NONE && (!Z || !aligned16(Z) || !Delta)) return ISOPO_ERR_INVALID_ARG;
    if (dX && (!W || !aligned16(W) || dX == dY || dX == Delta || dX == Z)) return ISOPO_ERR_INVALID_ARG;
    if (Delta == dY && b.ldy != d_out) return ISOPO_ERR_INVALID_ARG;
    if (!check_ws(workspace, ws_bytes, isopo_linear_backward_workspace(n_tokens, d_in, d_out, dtype), &st)) return st;
  }
  if (!aligned(db, 4)) return ISOPO_ERR_INVALID_ARG;
  if (n_tokens == 0 && !db) return ISOPO_OK;
  b.dY = dY; b.Z = Z; b.Delta = Delta == dY && act == ISOPO_ACT_NONE ? nullptr : Delta; b.db = db;
  b.workspace = static_cast<float*>(workspace); b.rows = n_tokens; b.cols = d_out; b.bf16 = bf16; b.act = act_of(act);
  LinearArgs a;
  if (b.Delta || b.db) {
    st = of(launch_act_backward(b, s, dX ? &a.then : nullptr));
    if (st != ISOPO_OK) return st;
  }
  if (!dX || n_tokens == 0) return ISOPO_OK;
  a.A = Delta ? Delta : dY; a.lda = Delta ? d_out : b.ldy;
  a.B = W; a.bias = nullptr; a.residual = nullptr; a.C = dX; a.Z = nullptr;
  a.rows = n_tokens; a.ldr = 0; a.ldc = d_in; a.k = d_out; a.n_out = d_in;
  a.bf16 = bf16; a.b_rows_are_k = true; a.act = Act::kNone;
  a.workspace = reinterpret_cast<float*>(static_cast<char*>(workspace) + align_up(act_backward_workspace(n_tokens, d_out)));
  return of(launch_linear(a, s));
}

// What both calls ask of the logits; *pitch: elements between rows.
static isopo_status check_logits(const isopo_token_logits* l, const void* dlogits, int64_t ldd, long long* ld, long long* ldo) {
  if (!l) return ISOPO_ERR_INVALID_ARG;
  if (!enum_in(l->dtype, ISOPO_F32, ISOPO_BF16)) return ISOPO_ERR_UNSUPPORTED;
  if (l->n_tokens < 0 || l->vocab <= 0 || !(l->inv_temperature > 0.f) || !(l->inv_temperature < INFINITY)) return ISOPO_ERR_INVALID_ARG;
  if (l->n_tokens > kMaxTokens) return ISOPO_ERR_UNSUPPORTED;
  *ld = l->ld ? l->ld : l->vocab;
  *ldo = ldd ? ldd : l->vocab;
  if (*ld < l->vocab || *ldo < l->vocab) return ISOPO_ERR_INVALID_ARG;
  if (l->n_tokens == 0) return ISOPO_OK;
  const size_t e = l->dtype == ISOPO_BF16 ? 2 : 4;
  if (!l->logits || !l->targets || !aligned(l->logits, e) || !aligned(l->targets, 4) || !aligned(dlogits, e)) return ISOPO_ERR_INVALID_ARG;
  if (dlogits == l->logits && *ld != *ldo) return ISOPO_ERR_INVALID_ARG;
  return ISOPO_OK;
}

isopo_status isopo_token_logprob(const isopo_token_logits* l, float* logp, float* lse, float* entropy, const float* weight, void* dlogits,
                                 int64_t ldd, void* stream) {
  TokenLogprobArgs a;
  isopo_status st = check_logits(l, dlogits, ldd, &a.ld, &a.ldd);
  if (st != ISOPO_OK) return st;
  if ((weight != nullptr) != (dlogits != nullptr)) return ISOPO_ERR_INVALID_ARG;
  if (!aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(weight, 4)) return ISOPO_ERR_INVALID_ARG;
  if (l->n_tokens == 0) return ISOPO_OK;
  a.logits = l->logits; a.bf16 = l->dtype == ISOPO_BF16; a.n_tokens = l->n_tokens; a.vocab = l->vocab; a.targets = l->targets;
  a.inv_temperature = l->inv_temperature; a.logp = logp; a.lse = lse; a.entropy = entropy; a.weight = weight; a.dlogits = dlogits;
  return of(launch_token_logprob(a, static_cast<hipStream_t>(stream)));
}

isopo_status isopo_token_logprob_backward(const isopo_token_logits* l, const float* lse, const float* grad_logp, const float* entropy,
                                          const float* grad_entropy, void* dlogits, int64_t ldd, void* stream) {
  TokenLogprobBackwardArgs a;
  isopo_status st = check_logits(l, dlogits, ldd, &a.ld, &a.ldd);
  if (st != ISOPO_OK) return st;
  if (grad_entropy && !entropy) return ISOPO_ERR_INVALID_ARG;
  if (l->n_tokens == 0) return ISOPO_OK;
  if (!lse || !grad_logp || !dlogits || !aligned(lse, 4) || !aligned(grad_logp, 4) || !aligned(entropy, 4) || !aligned(grad_entropy, 4))
    return ISOPO_ERR_INVALID_ARG;
  a.logits = l->logits; a.bf16 = l->dtype == ISOPO_BF16; a.n_tokens = l->n_tokens; a.vocab = l->vocab; a.targets = l->targets;
  a.inv_temperature = l->inv_temperature; a.lse = lse; a.grad_logp = grad_logp; a.entropy = grad_entropy ? entropy : nullptr;
  a.grad_entropy = grad_entropy; a.dlogits = dlogits;
  return of(launch_token_logprob_backward(a, static_cast<hipStream_t>(stream)));
}

static bool sizes_ok(const isopo_adamw_tensor* t, int32_t n) {
  if (n < 0 || (n > 0 && !t)) return false;
  for (int32_t i = 0; i < n; ++i)
    if (t[i].n < 0 || t[i].n > 0xffffffffLL) return false;
  return true;
}

size_t isopo_grad_norm_workspace(const isopo_adamw_tensor* tensors, int32_t n_tensors) {
  return sizes_ok(tensors, n_tensors) ? grad_norm_workspace(tensors, n_tensors) : 0;
}

isopo_status isopo_grad_norm(const isopo_adamw_tensor* tensors, const void* const* grads, int32_t n_tensors, isopo_dtype grad_dtype,
                             float* norm, void* workspace, size_t ws_bytes, void* stream) {
  if (!enum_in(grad_dtype, ISOPO_F32, ISOPO_BF16)) return ISOPO_ERR_UNSUPPORTED;
  if (!sizes_ok(tensors, n_tensors) || (n_tensors > 0 && !grads) || !norm || !aligned(norm, 4)) return ISOPO_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_tensors; ++i)
    if (tensors[i].n > 0 && (!grads[i] || !aligned16(grads[i]))) return ISOPO_ERR_INVALID_ARG;
  isopo_status st;
  if (!check_ws(workspace, ws_bytes, grad_norm_workspace(tensors, n_tensors), &st)) return st;
  return of(launch_grad_norm(tensors, grads, n_tensors, grad_dtype == ISOPO_BF16, norm, static_cast<double*>(workspace),
                             static_cast<hipStream_t>(stream), nullptr));
}

static isopo_status adamw_args(const isopo_adamw_tensor* tensors, const void* const* grads, int32_t n_tensors, const isopo_adamw_params* q,
                               float* norm, AdamwArgs* a) {
  if (!q) return ISOPO_ERR_INVALID_ARG;
  if (!enum_in(q->param_dtype, ISOPO_F32, ISOPO_BF16) || !enum_in(q->grad_dtype, ISOPO_F32, ISOPO_BF16)) return ISOPO_ERR_UNSUPPORTED;
  if (q->state_bits != 8 && q->state_bits != 32) return ISOPO_ERR_UNSUPPORTED;
  if (!sizes_ok(tensors, n_tensors) || (n_tensors > 0 && !grads) || !aligned(norm, 4)) return ISOPO_ERR_INVALID_ARG;
  const auto fraction = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!fraction(q->beta1) || !fraction(q->beta2) || !(q->eps >= 0.0) || !(q->weight_decay >= 0.0) || q->step < 1 || !(q->lr >= 0.0) || !(q->lr < INFINITY))
    return ISOPO_ERR_INVALID_ARG;
  if (norm && !(q->max_norm > 0.0)) return ISOPO_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const isopo_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    if (!t.param || !grads[i] || !t.m || !t.v || !aligned16(t.param) || !aligned16(grads[i]) || !aligned16(t.m) || !aligned16(t.v) ||
        !aligned16(t.master))
      return ISOPO_ERR_INVALID_ARG;
    if (q->state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))) return ISOPO_ERR_INVALID_ARG;
  }
  a->tensors = tensors; a->grads = grads; a->n_tensors = n_tensors;
  a->param_bf16 = q->param_dtype == ISOPO_BF16; a->grad_bf16 = q->grad_dtype == ISOPO_BF16; a->bits8 = q->state_bits == 8;
  a->maximize = q->maximize != 0;
  a->lr = q->lr; a->beta1 = q->beta1; a->beta2 = q->beta2; a->eps = q->eps; a->weight_decay = q->weight_decay; a->max_norm = q->max_norm;
  a->step = q->step; a->seed = q->seed; a->norm = norm;
  return ISOPO_OK;
}

isopo_status isopo_adamw(const isopo_adamw_tensor* tensors, const void* const* grads, int32_t n_tensors, const isopo_adamw_params* q,
                         const float* norm, void* stream) {
  AdamwArgs a;
  const isopo_status st = adamw_args(tensors, grads, n_tensors, q, const_cast<float*>(norm), &a);        // (is read alone)
  return st == ISOPO_OK ? of(launch_adamw(a, static_cast<hipStream_t>(stream))) : st;
}

isopo_status isopo_adamw_clipped(const isopo_adamw_tensor* tensors, const void* const* grads, int32_t n_tensors, const isopo_adamw_params* q,
                                 float* norm, void* workspace, size_t ws_bytes, void* stream) {
  AdamwArgs a;
  isopo_status st = adamw_args(tensors, grads, n_tensors, q, norm, &a);
  if (st != ISOPO_OK) return st;
  if (!norm) return ISOPO_ERR_INVALID_ARG;
  if (!check_ws(workspace, ws_bytes, grad_norm_workspace(tensors, n_tensors), &st)) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  st = of(launch_grad_norm(tensors, grads, n_tensors, a.grad_bf16, norm, static_cast<double*>(workspace), s, &a.n_norm_parts));
  if (st != ISOPO_OK) return st;
  if (a.n_norm_parts) a.norm_parts = static_cast<const double*>(workspace);
  return of(launch_adamw(a, s));
}

isopo_status isopo_adamw_state(const void* m, const float* m_scale, const void* v, const float* v_scale, int64_t n, isopo_dtype dtype,
                               void* m_out, void* v_out, void* stream) {
  if (!enum_in(dtype, ISOPO_F32, ISOPO_BF16)) return ISOPO_ERR_UNSUPPORTED;
  if (n < 0 || n > (int64_t)1 << 40) return ISOPO_ERR_INVALID_ARG;
  if (n == 0) return ISOPO_OK;
  if (m_out && (!m || !m_scale || !aligned16(m) || !aligned(m_scale, 4) || !aligned16(m_out))) return ISOPO_ERR_INVALID_ARG;
  if (v_out && (!v || !v_scale || !aligned16(v) || !aligned(v_scale, 4) || !aligned16(v_out))) return ISOPO_ERR_INVALID_ARG;
  if (!m_out && !v_out) return ISOPO_OK;
  return of(launch_adamw_state(m, m_scale, v, v_scale, n, dtype == ISOPO_BF16, m_out, v_out, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
