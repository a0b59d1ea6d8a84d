// Replays the host code of the operators around the layer step over small, ordinary and the largest sizes: argument checks,
// workspaces, plans, the cuts into launches, the tables that travel in a launch's arguments.  Built by
// tests/test_policy_sanitizers.py with AddressSanitizer and UndefinedBehaviorSanitizer on the host code; touches no GPU: every launch
// is taken note of and not made.
#include <cstdint>
#include <cstdio>
#include <vector>

#include <hip/hip_runtime.h>

#include "../include/isopo.h"

struct Launch {
  dim3 grid, block;
  size_t lds;
};
static std::vector<Launch> launches;
// What the library's launches call of the runtime: the configuration is kept, and an error keeps the launch itself from being made.
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) {
  launches.push_back({grid, block, lds});
  return hipErrorNotSupported;
}
extern "C" hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

static int failures = 0, calls = 0;
#define EXPECT(cond)                                                                         \
  do {                                                                                       \
    if (!(cond)) { std::printf("FAIL %s:%d %s\n", __FILE__, __LINE__, #cond); ++failures; } \
  } while (0)

static char* const there = reinterpret_cast<char*>((uintptr_t)1 << 40);          // never followed
static float* const f = reinterpret_cast<float*>(there);

static void check_launches(const char* what, long long n, long long a, long long b) {
  ++calls;
  for (const Launch& l : launches) {
    const unsigned long long threads = (unsigned long long)l.grid.x * l.block.x;
    if (!l.grid.x || threads >= 1ull << 32 || l.grid.y > 65535 || l.grid.z != 1 || l.block.x > 1024 || l.lds > 160 * 1024) {
      std::printf("FAIL %s %lld %lld %lld: grid %u x %u, block %u, lds %zu\n", what, n, a, b, l.grid.x, l.grid.y, l.block.x, l.lds);
      ++failures;
    }
  }
}

static void linear(int64_t n, int d_in, int d_out, isopo_dtype dtype, isopo_activation act) {
  size_t need = isopo_linear_workspace(n, d_in, d_out, dtype), parts_launches = 0;
  for (int64_t first = 0; first < n;) {
    isopo_linear_plan_info p{};
    EXPECT(isopo_linear_plan(n, d_in, d_out, dtype, 0, first, &p) == ISOPO_OK);
    EXPECT(p.tokens > 0 && p.tokens <= n - first && p.workspace_end <= need);
    parts_launches += p.parts > 1 ? 2 : 1;
    if (p.tokens <= 0) return;
    first += p.tokens;
  }
  isopo_linear_layer l{};
  l.X = there; l.W = there + 4096; l.bias = there + 2; l.residual = there + (1 << 20); l.dtype = dtype; l.act = act;
  if (dtype == ISOPO_F32) l.bias = there + 4;
  l.n_tokens = n; l.d_in = d_in; l.d_out = d_out;
  launches.clear();
  EXPECT(isopo_linear(&l, there + (1 << 21), there + (1 << 22), need ? there : nullptr, need, nullptr) == ISOPO_OK);
  EXPECT(launches.size() == parts_launches);
  check_launches("linear", n, d_in, d_out);
  need = isopo_linear_backward_workspace(n, d_in, d_out, dtype);
  for (int64_t first = 0; first < n;) {
    isopo_linear_plan_info p{};
    EXPECT(isopo_linear_plan(n, d_in, d_out, dtype, 1, first, &p) == ISOPO_OK && p.tokens > 0 && p.workspace_end <= need);
    if (p.tokens <= 0) return;
    first += p.tokens;
  }
  for (const bool dx : {false, true}) {
    launches.clear();
    EXPECT(isopo_linear_backward(there, 0, there + 4096, there + (1 << 20), dtype, act, n, d_in, d_out, there + (1 << 21), dx ? there + (1 << 22) : nullptr, f,
                                 need ? there : nullptr, need, nullptr) == ISOPO_OK);
    EXPECT(!launches.empty());
    check_launches("linear_backward", n, d_in, d_out);
  }
}

static void logprob(int64_t n, int vocab, isopo_dtype dtype, bool backward_too) {
  isopo_token_logits l{};
  l.logits = there; l.dtype = dtype; l.n_tokens = n; l.vocab = vocab; l.targets = reinterpret_cast<int32_t*>(there); l.inv_temperature = 1.f;
  for (float* const ent : {static_cast<float*>(nullptr), f}) {
    for (const bool grad : {false, true}) {
      launches.clear();
      EXPECT(isopo_token_logprob(&l, f, f, ent, grad ? f : nullptr, grad ? there : nullptr, 0, nullptr) == ISOPO_OK);
      check_launches("token_logprob", n, vocab, grad);
    }
    if (!backward_too) continue;
    launches.clear();
    EXPECT(isopo_token_logprob_backward(&l, f, f, ent, ent, there + 4096, 0, nullptr) == ISOPO_OK);
    check_launches("token_logprob_backward", n, vocab, ent != nullptr);
  }
}

static void adamw(const std::vector<int64_t>& sizes, int bits, bool clip) {
  std::vector<isopo_adamw_tensor> t;
  std::vector<const void*> g;
  long long blocks = 0;
  for (const int64_t n : sizes) {
    t.push_back({there, f, there, there, f, f, n});
    g.push_back(there);
    blocks += (n + 1023) / 1024;
  }
  isopo_adamw_params q{};
  q.param_dtype = ISOPO_BF16; q.grad_dtype = ISOPO_F32; q.state_bits = bits; q.lr = 1e-3; q.beta1 = 0.9; q.beta2 = 0.999; q.eps = 1e-8; q.max_norm = 1.0;
  q.step = 1; q.seed = 1;
  const int32_t n = (int32_t)sizes.size();
  launches.clear();
  const size_t need = isopo_grad_norm_workspace(t.data(), n);
  if (clip) EXPECT(isopo_adamw_clipped(t.data(), g.data(), n, &q, f, need ? there : nullptr, need, nullptr) == ISOPO_OK);
  else EXPECT(isopo_adamw(t.data(), g.data(), n, &q, nullptr, nullptr) == ISOPO_OK);
  check_launches("adamw", n, blocks, clip);
  long long done = 0, norm = 0;
  for (const Launch& l : launches) done += l.grid.x;
  if (clip) {
    launches.clear();
    EXPECT(isopo_grad_norm(t.data(), g.data(), n, ISOPO_F32, f, need ? there : nullptr, need, nullptr) == ISOPO_OK);
    check_launches("grad_norm", n, blocks, bits);
    for (const Launch& l : launches) norm += l.grid.x;
    EXPECT((size_t)(norm - 1) * sizeof(double) == need);              // (the last workgroup joins the parts)
    const bool few = need > 0 && need <= 256 * sizeof(double);        // joined by the update itself
    EXPECT(done == blocks + norm - (few ? 1 : 0));
  } else {
    EXPECT(done == blocks);
  }
  if (!sizes.empty()) {
    launches.clear();
    EXPECT(isopo_adamw_state(there, f, there, f, sizes[0], ISOPO_BF16, there + 4096, there + 8192, nullptr) == ISOPO_OK);
    check_launches("adamw_state", sizes[0], 0, 0);
  }
}

int main() {
  const int widths[][2] = {{64, 128}, {4096, 14336}, {14336, 4096}, {4096, 4096}, {1536, 8960}, {8, 8}, {16384, 64}, {64, 16384}, {520, 264}, {(1 << 22) - 8, 8},
                           {8, (1 << 22) - 8}};
  for (const auto& w : widths)
    for (const isopo_dtype dtype : {ISOPO_F32, ISOPO_BF16}) {
      for (const int backward : {0, 1}) {
        isopo_linear_plan_info p{};
        EXPECT(isopo_linear_plan(0x7fffffff, w[0], w[1], dtype, backward, 0, &p) == ISOPO_OK);
        for (const int64_t more : {-1, 0, 1, 24, 128, 1000})
          if (p.tokens + more <= 0x7fffffff) linear(p.tokens + more, w[0], w[1], dtype, ISOPO_ACT_SILU);
      }
      for (const int64_t n : {1, 2, 24, 64, 129, 1000, 4096, 16384, 100003}) linear(n, w[0], w[1], dtype, n % 2 ? ISOPO_ACT_NONE : ISOPO_ACT_GELU);
      if (w[1] < 1 << 15) linear(0x7fffffff, w[0], w[1], dtype, ISOPO_ACT_RELU);
    }
  for (const isopo_dtype dtype : {ISOPO_F32, ISOPO_BF16}) {
    for (const int vocab : {1, 7, 48, 257, 1000, 8192, 50001, 131072, 152064, 1 << 24, 0x7fffffff})
      for (const int64_t n : {1, 4, 511, 512, 1000}) logprob(n, vocab, dtype, true);
    for (const int vocab : {1, 1000, 131072}) logprob(((int64_t)1 << 21) + 77, vocab, dtype, true);
    logprob(0x7fffffff, 1000, dtype, true);
  }
  for (const int bits : {8, 32})
    for (const bool clip : {false, true}) {
      adamw({}, bits, clip);
      adamw({0, 0}, bits, clip);
      adamw({1}, bits, clip);
      adamw({16384, 0, 5}, bits, clip);
      adamw({4194304, 16384}, bits, clip);
      adamw(std::vector<int64_t>(301, 4097), bits, clip);
      adamw({0xffffffffLL, 0xffffffffLL, 0xffffffffLL, 3}, bits, clip);
    }
  for (const int64_t n : {(int64_t)1, (int64_t)0xffffffff}) EXPECT(isopo_adamw_state(there, f, nullptr, nullptr, n, ISOPO_F32, there, nullptr, nullptr) == ISOPO_OK);
  // values that are none of an enum's: refused, never loaded as the enum; nothing is launched by a call that is refused
  launches.clear();
  for (const int v : {-1, 5, 1 << 30}) {
    isopo_linear_plan_info p{};
    EXPECT(isopo_linear_workspace(64, 64, 64, (isopo_dtype)v) == 0 && isopo_linear_backward_workspace(64, 64, 64, (isopo_dtype)v) == 0);
    EXPECT(isopo_linear_plan(64, 64, 64, (isopo_dtype)v, 0, 0, &p) == ISOPO_ERR_UNSUPPORTED);
    EXPECT(isopo_linear_backward(there, 0, there, there, (isopo_dtype)v, ISOPO_ACT_NONE, 64, 64, 64, there, there, f, there, 1 << 30, nullptr) == ISOPO_ERR_UNSUPPORTED);
    EXPECT(isopo_linear_backward(there, 0, there, there, ISOPO_BF16, (isopo_activation)v, 64, 64, 64, there, there, f, there, 1 << 30, nullptr) ==
           ISOPO_ERR_INVALID_ARG);
    EXPECT(isopo_adamw_state(there, f, there, f, 64, (isopo_dtype)v, there, there, nullptr) == ISOPO_ERR_UNSUPPORTED);
  }
  EXPECT(launches.empty());
  std::printf("calls=%d\ndone failures=%d\n", calls, failures);
  return failures ? 1 : 0;
}
