// AdamW over many tensors in few launches, with states in 32 or 8 bits; the norm of all gradients; the values of 8-bit states.
//
// Bound by HBM: every element is read and written once, 28 bytes (fp32) or 18 (bf16 parameter, fp32 master, 8-bit states,
// fp32 gradient) of it.  218 M elements, fp32: 1.14 ms, 5.3 TB/s, with the norm 1.32; the latter kind 0.72 - 0.82 ms, 4.8 - 5.5 TB/s (a large
// copy: 4.9); the norm before it 0.18 ms, 4.9 TB/s; the states' values as bf16 0.21 ms, 6.2 TB/s.  70 tensors of 4096 elements and so: 12 us in two
// launches, and the host's time, 30 us a step, hides them.  The tensors' addresses travel in the kernel's
// arguments, 83 or 55 a launch: nothing is copied to the device and nothing waits.  A workgroup takes 1024 elements of one tensor, a vector a lane.
//
// 8-bit states: ISOPO_ADAMW_BLOCK = 256 elements share a scale; a wave holds such a block, four elements a lane, so its
// largest magnitude is a reduction over the wave's registers.  The code of x (magnitude over scale) is the fp32 bit pattern of x + C with the low
// 19 bits dropped, counted from C's pattern: 16 codes to an octave, by integer additions alone.  The dropped bits decide with a hash of
// (seed, tensor, element) whether it is rounded up: the sum of both carries into the code with the odds of the remainder.  v is held as its
// root, whose smallest step (2^-20 of the scale) lies well below m's (2^-12): where v is rounded to zero nothing is left of m to be divided by its root.
#include <cmath>
#include <type_traits>

#include "common.h"
#include "policy.h"

namespace isopo {
namespace {

constexpr int kBlock = 256;
constexpr size_t kArgBytes = 4096;       // what a launch's arguments may hold

constexpr float kCm = 1.0625f * 0x1p-8f, kCv = 1.0625f * 0x1p-16f;
constexpr unsigned kCmBits = 0x3b880000u, kCvBits = 0x37880000u;

struct Entry32 {
  void* param;
  float* master;
  const void* grad;
  void* m;
  void* v;
  unsigned n;
  unsigned first;              // the tensor's first workgroup
};
struct Entry8 : Entry32 {
  float* m_scale;
  float* v_scale;
  unsigned key;
};

struct Common {
  int n_tensors;
  float beta1, beta2, g1, g2;  // g = 1 - beta
  float keep, lr;              // keep = 1 - lr weight_decay
  float m_correct, v_correct, eps, max_norm;
  float* norm;
  const double* norm_parts;    // NULL: norm is read;  else these are summed, and it is written
  int n_norm_parts;
};
template <bool BITS8>
struct Params : Common {
  typedef std::conditional_t<BITS8, Entry8, Entry32> Entry;
  static constexpr int kMaxTensors = (int)((kArgBytes - sizeof(Common)) / sizeof(Entry));
  Entry entry[kMaxTensors];
};

__host__ __device__ __forceinline__ unsigned mix(unsigned x) {
  x *= 0x9e3779b1u;            // odd numbers from the golden ratio and the square root of three
  x ^= x >> 15;
  x *= 0xbb67ae85u;
  return x ^ (x >> 16);
}

// The tensor whose workgroup this is: the last one that starts at or before it.
template <class P>
__device__ __forceinline__ int tensor_of(const P& p, unsigned b) {
  int lo = 0, hi = p.n_tensors;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.entry[mid].first <= b) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ float decode(unsigned code, unsigned c_bits, float c) { return __builtin_bit_cast(float, c_bits + (code << 19)) - c; }
__device__ __forceinline__ unsigned encode(float x, float inv, unsigned u, unsigned c_bits, float c, unsigned most) {
  const unsigned code = (__builtin_bit_cast(unsigned, x * inv + c) - c_bits + u) >> 19;
  return code < most ? code : most;
}

// The largest of a wave's magnitudes, by their bit patterns, which rise with them: a NaN's is above all others.
__device__ __forceinline__ unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }
__device__ __forceinline__ float wave_largest(unsigned x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const unsigned y = __shfl_xor(x, o, 64);
    x = y > x ? y : x;
  }
  return __builtin_bit_cast(float, x);
}

template <bool BF16>
__device__ __forceinline__ void load4(const void* p, long long i, float (&x)[4]) {
  if constexpr (BF16) {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const unsigned short*>(p) + i);
    x[0] = __builtin_bit_cast(float, w.x << 16); x[1] = __builtin_bit_cast(float, w.x & 0xffff0000u);
    x[2] = __builtin_bit_cast(float, w.y << 16); x[3] = __builtin_bit_cast(float, w.y & 0xffff0000u);
  } else {
    const f32x4 v = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = v[q];
  }
}
template <bool BF16>
__device__ __forceinline__ void store4(void* p, long long i, const float (&x)[4]) {
  if constexpr (BF16) {
    uint2 w;
    w.x = (unsigned)f32_to_bf16_bits(x[0]) | (unsigned)f32_to_bf16_bits(x[1]) << 16;
    w.y = (unsigned)f32_to_bf16_bits(x[2]) | (unsigned)f32_to_bf16_bits(x[3]) << 16;
    *reinterpret_cast<uint2*>(static_cast<unsigned short*>(p) + i) = w;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(p) + i) = f32x4{x[0], x[1], x[2], x[3]};
  }
}
template <bool BF16>
__device__ __forceinline__ float load1(const void* p, long long i) {
  if constexpr (BF16) return bf16_bits_to_f32(static_cast<const unsigned short*>(p)[i]);
  else return static_cast<const float*>(p)[i];
}
template <bool BF16>
__device__ __forceinline__ void store1(void* p, long long i, float x) {
  if constexpr (BF16) static_cast<unsigned short*>(p)[i] = f32_to_bf16_bits(x);
  else static_cast<float*>(p)[i] = x;
}

// The root of the sum of n parts: every thread's, by the one workgroup of NT threads.  red: NT / 64 doubles.
template <int NT>
__device__ __forceinline__ float norm_of(const double* parts, long long n, double* red) {
  double t = 0.0;
  for (long long i = threadIdx.x; i < n; i += NT) t += parts[i];
  t = wave_sum(t);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
  __syncthreads();
  t = 0.0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t += red[w];
  return (float)sqrt(t);
}
// Up to so many, one a thread, every workgroup of the update sums them itself: no launch between the two (a step of 28 tensors of
// 1000 elements 21.2 -> 15.8 us, the host's time).  With more elements the launch is hidden behind the update's time.
constexpr int kFewParts = 256;

template <bool PB, bool GB, bool BITS8>
__global__ __launch_bounds__(256) void adamw_kernel(Params<BITS8> p) {
  float clip = 1.f;
  if (p.norm) {
    float norm;
    if (p.norm_parts) {
      __shared__ double red[4];
      norm = norm_of<256>(p.norm_parts, p.n_norm_parts, red);
      if (blockIdx.x == 0 && threadIdx.x == 0) *p.norm = norm;
    } else {
      norm = *p.norm;
    }
    if (!(norm < INFINITY)) return;
    clip = fminf(p.max_norm / (norm + 1e-6f), 1.f);
  }
  const int k = __builtin_amdgcn_readfirstlane(tensor_of(p, blockIdx.x));
  const auto& e = p.entry[k];
  const long long i0 = (long long)(blockIdx.x - e.first) * 1024 + threadIdx.x * 4;
  const long long n = e.n;
  const int have = n - i0 >= 4 ? 4 : n > i0 ? (int)(n - i0) : 0;
  const bool whole = have == 4;
  float g[4] = {}, w[4] = {}, m[4] = {}, v[4] = {};
  unsigned mc = 0, vc = 0;
  if (whole) {
    load4<GB>(e.grad, i0, g);
    if (e.master) load4<false>(e.master, i0, w); else load4<PB>(e.param, i0, w);
    if constexpr (BITS8) {
      mc = *reinterpret_cast<const unsigned*>(static_cast<const unsigned char*>(e.m) + i0);
      vc = *reinterpret_cast<const unsigned*>(static_cast<const unsigned char*>(e.v) + i0);
    } else {
      load4<false>(e.m, i0, m);
      load4<false>(e.v, i0, v);
    }
  } else {
    for (int q = 0; q < have; ++q) {
      g[q] = load1<GB>(e.grad, i0 + q);
      w[q] = e.master ? e.master[i0 + q] : load1<PB>(e.param, i0 + q);
      if constexpr (BITS8) {
        mc |= (unsigned)static_cast<const unsigned char*>(e.m)[i0 + q] << (8 * q);
        vc |= (unsigned)static_cast<const unsigned char*>(e.v)[i0 + q] << (8 * q);
      } else {
        m[q] = static_cast<const float*>(e.m)[i0 + q];
        v[q] = static_cast<const float*>(e.v)[i0 + q];
      }
    }
  }
  const long long block = i0 / kBlock;       // one per wave
  if constexpr (BITS8) {
    const bool any = block * kBlock < n;
    const float ms = any ? e.m_scale[block] : 0.f, vs = any ? e.v_scale[block] : 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const unsigned a = mc >> (8 * q) & 255u, b = vc >> (8 * q) & 255u;
      const float x = decode(a & 127u, kCmBits, kCm) * ms, r = decode(b, kCvBits, kCv) * vs;
      m[q] = a & 128u ? -x : x;
      v[q] = r * r;
    }
  }
  float r[4];
  unsigned most_m = 0, most_r = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    g[q] *= clip;
    m[q] = m[q] * p.beta1 + g[q] * p.g1;
    v[q] = v[q] * p.beta2 + g[q] * g[q] * p.g2;
    w[q] = w[q] * p.keep - p.lr * ((m[q] * p.m_correct) / (sqrtf(v[q] * p.v_correct) + p.eps));
    if constexpr (BITS8) {
      if (q >= have) m[q] = v[q] = 0.f;
      r[q] = sqrtf(v[q]);
      most_m = magnitude(m[q]) > most_m ? magnitude(m[q]) : most_m;
      most_r = magnitude(r[q]) > most_r ? magnitude(r[q]) : most_r;
    }
  }
  if constexpr (BITS8) {
    const float top_m = wave_largest(most_m), top_r = wave_largest(most_r);
    const float m_inv = top_m > 0.f ? (1.f - kCm) / top_m : 0.f, v_inv = top_r > 0.f ? (1.f - kCv) / top_r : 0.f;
    mc = vc = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const unsigned h = mix((unsigned)(i0 + q) ^ e.key);
      const unsigned a = encode(fabsf(m[q]), m_inv, (h & 0xffffu) << 3, kCmBits, kCm, 127u) | (m[q] < 0.f ? 128u : 0u);
      const unsigned b = encode(r[q], v_inv, (h >> 16) << 3, kCvBits, kCv, 255u);
      mc |= a << (8 * q);
      vc |= b << (8 * q);
    }
    if ((threadIdx.x & 63) == 0 && block * kBlock < n) {
      e.m_scale[block] = top_m / (1.f - kCm);
      e.v_scale[block] = top_r / (1.f - kCv);
    }
  }
  if (whole) {
    if (e.master) store4<false>(e.master, i0, w);
    store4<PB>(e.param, i0, w);
    if constexpr (BITS8) {
      *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(e.m) + i0) = mc;
      *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(e.v) + i0) = vc;
    } else {
      store4<false>(e.m, i0, m);
      store4<false>(e.v, i0, v);
    }
  } else {
    for (int q = 0; q < have; ++q) {
      if (e.master) e.master[i0 + q] = w[q];
      store1<PB>(e.param, i0 + q, w[q]);
      if constexpr (BITS8) {
        static_cast<unsigned char*>(e.m)[i0 + q] = (unsigned char)(mc >> (8 * q));
        static_cast<unsigned char*>(e.v)[i0 + q] = (unsigned char)(vc >> (8 * q));
      } else {
        static_cast<float*>(e.m)[i0 + q] = m[q];
        static_cast<float*>(e.v)[i0 + q] = v[q];
      }
    }
  }
}

constexpr int kNormTensors = 128;
struct NormParams {
  int n_tensors;
  double* parts;               // one per workgroup of this launch
  struct { const void* grad; long long n; unsigned first; } entry[kNormTensors];
};

constexpr int kNormChunk = 16384;

template <bool GB>
__global__ __launch_bounds__(256) void grad_norm_kernel(NormParams p) {
  __shared__ double red[4];
  const auto& e = p.entry[__builtin_amdgcn_readfirstlane(tensor_of(p, blockIdx.x))];
  const long long i0 = (long long)(blockIdx.x - e.first) * kNormChunk;
  const long long i1 = e.n - i0 > kNormChunk ? i0 + kNormChunk : e.n;
  float t = 0.f;
  for (long long i = i0 + threadIdx.x * 4; i < i1; i += 1024) {
    float g[4] = {};
    if (i + 4 <= i1) load4<GB>(e.grad, i, g);
    else for (int q = 0; q < i1 - i; ++q) g[q] = load1<GB>(e.grad, i + q);
#pragma unroll
    for (int q = 0; q < 4; ++q) t += g[q] * g[q];
  }
  const double d = wave_sum((double)t);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = d;
  __syncthreads();
  if (threadIdx.x == 0) p.parts[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(1024) void grad_norm_finish_kernel(const double* __restrict__ parts, long long n, float* __restrict__ norm) {
  __shared__ double red[16];
  const float t = norm_of<1024>(parts, n, red);
  if (threadIdx.x == 0) *norm = t;
}

// 16 elements a thread, four by four.
template <bool BF16>
__global__ __launch_bounds__(256) void adamw_state_kernel(const unsigned char* __restrict__ m, const float* __restrict__ m_scale,
                                                          const unsigned char* __restrict__ v, const float* __restrict__ v_scale, long long n,
                                                          void* __restrict__ m_out, void* __restrict__ v_out) {
  const long long first = (long long)blockIdx.x * 4096 + threadIdx.x * 4;
  auto four = [&](const unsigned char* code, const float* scale, void* out, auto&& value) {
    unsigned c[4];
    float s[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long i = first + k * 1024;
      c[k] = 0;
      s[k] = i < n ? scale[i / kBlock] : 0.f;
      if (i + 4 <= n) c[k] = *reinterpret_cast<const unsigned*>(code + i);
      else
        for (int q = 0; q < 4 && i + q < n; ++q) c[k] |= (unsigned)code[i + q] << (8 * q);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long i = first + k * 1024;
      float x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = value(c[k] >> (8 * q) & 255u, s[k]);
      if (i + 4 <= n) store4<BF16>(out, i, x);
      else
        for (int q = 0; q < 4 && i + q < n; ++q) store1<BF16>(out, i + q, x[q]);
    }
  };
  if (m_out)
    four(m, m_scale, m_out, [](unsigned c, float s) {
      const float x = decode(c & 127u, kCmBits, kCm) * s;
      return c & 128u ? -x : x;
    });
  if (v_out)
    four(v, v_scale, v_out, [](unsigned c, float s) {
      const float r = decode(c, kCvBits, kCv) * s;
      return r * r;
    });
}

long long norm_blocks(long long n) { return (n + kNormChunk - 1) / kNormChunk; }

}  // namespace

namespace {

template <bool BITS8>
hipError_t launch(const AdamwArgs& a, hipStream_t s) {
  Params<BITS8> p;
  p.beta1 = (float)a.beta1; p.beta2 = (float)a.beta2; p.g1 = (float)(1.0 - a.beta1); p.g2 = (float)(1.0 - a.beta2);
  p.keep = (float)(1.0 - a.lr * a.weight_decay); p.lr = (float)(a.maximize ? -a.lr : a.lr);
  p.m_correct = (float)(1.0 / (1.0 - std::pow(a.beta1, (double)a.step))); p.v_correct = (float)(1.0 / (1.0 - std::pow(a.beta2, (double)a.step)));
  p.eps = (float)a.eps; p.max_norm = (float)a.max_norm;
  p.norm = a.norm; p.norm_parts = a.norm_parts; p.n_norm_parts = a.n_norm_parts;
  const unsigned key = mix(a.seed ^ 0x3c6ef373u);
  for (int t = 0; t < a.n_tensors;) {
    long long blocks = 0;                // a tensor has 2^22 at most; a grid holds 2^32 threads, 2^24 workgroups
    p.n_tensors = 0;
    for (; t < a.n_tensors && p.n_tensors < p.kMaxTensors && blocks < 1 << 23; ++t) {
      const isopo_adamw_tensor& x = a.tensors[t];
      if (x.n <= 0) continue;
      auto& e = p.entry[p.n_tensors++];
      e.param = x.param; e.master = x.master; e.grad = a.grads[t]; e.m = x.m; e.v = x.v;
      e.n = (unsigned)x.n; e.first = (unsigned)blocks;
      if constexpr (BITS8) { e.m_scale = x.m_scale; e.v_scale = x.v_scale; e.key = mix(key + (unsigned)t); }
      blocks += (x.n + 1023) / 1024;
    }
    if (!p.n_tensors) continue;
    const dim3 grid((unsigned)blocks), wg(256);
    auto go = [&](auto pb, auto gb) { hipLaunchKernelGGL((adamw_kernel<decltype(pb)::value, decltype(gb)::value, BITS8>), grid, wg, 0, s, p); };
    auto grads = [&](auto pb) { if (a.grad_bf16) go(pb, std::true_type{}); else go(pb, std::false_type{}); };
    if (a.param_bf16) grads(std::true_type{}); else grads(std::false_type{});
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, hipStream_t s) { return a.bits8 ? launch<true>(a, s) : launch<false>(a, s); }

size_t grad_norm_workspace(const isopo_adamw_tensor* tensors, int n_tensors) {
  long long blocks = 0;
  for (int t = 0; t < n_tensors; ++t) blocks += norm_blocks(tensors[t].n);
  return (size_t)blocks * sizeof(double);
}

hipError_t launch_grad_norm(const isopo_adamw_tensor* tensors, const void* const* grads, int n_tensors, bool bf16, float* norm, double* workspace,
                            hipStream_t s, int* few) {
  NormParams p;
  long long done = 0;
  for (int t = 0; t < n_tensors;) {
    long long blocks = 0;
    p.n_tensors = 0;
    for (; t < n_tensors && p.n_tensors < kNormTensors; ++t) {
      if (tensors[t].n <= 0) continue;
      const long long b = norm_blocks(tensors[t].n);
      if (blocks + b > 0x7fffffffLL) break;
      p.entry[p.n_tensors++] = {grads[t], tensors[t].n, (unsigned)blocks};
      blocks += b;
    }
    if (!p.n_tensors) continue;
    p.parts = workspace + done;
    if (bf16) hipLaunchKernelGGL(grad_norm_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(grad_norm_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, s, p);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    done += blocks;
  }
  if (few) *few = done > 0 && done <= kFewParts ? (int)done : 0;
  if (few && *few) return hipSuccess;
  hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(1024), 0, s, workspace, done, norm);
  return hipGetLastError();
}

hipError_t launch_adamw_state(const void* m, const float* m_scale, const void* v, const float* v_scale, long long n, bool bf16, void* m_out,
                              void* v_out, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  if (n > 4096LL << 23) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((n + 4095) / 4096));
  const auto mb = static_cast<const unsigned char*>(m), vb = static_cast<const unsigned char*>(v);
  if (bf16) hipLaunchKernelGGL(adamw_state_kernel<true>, grid, dim3(256), 0, s, mb, m_scale, vb, v_scale, n, m_out, v_out);
  else hipLaunchKernelGGL(adamw_state_kernel<false>, grid, dim3(256), 0, s, mb, m_scale, vb, v_scale, n, m_out, v_out);
  return hipGetLastError();
}

}  // namespace isopo
