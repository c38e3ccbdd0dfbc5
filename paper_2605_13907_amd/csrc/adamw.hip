// An AdamW step over many tensors in one launch, with moments of 32 or 8 bits.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (wd p + m / c1 / (sqrt(v / c2) + eps)),  c = 1 - b^step
//
// Bound by memory: every array is read once and written once, 28 bytes an element with fp32 arrays and 16.1 with 8-bit moments.
// The tensors' addresses are kernel arguments, so that a call copies nothing to the GPU and can be recorded.  A lane takes eight
// consecutive elements; four lanes have a block of 32 whose 8-bit moments share a scale.
//
// The moments are formed in 64 bits (the GPU's fp64 is as fast as its fp32) and rounded to fp32: which of two 8-bit codes a value
// goes to depends on its last bits.
#include <type_traits>

#include "ais_internal.h"
#include "eights.h"

namespace ais {
namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr int kChunk = 8 * kThreads;             // elements of a workgroup
constexpr int kTensors = 48;                     // of a launch: their addresses are 3.3 of the 4 KiB of kernel arguments

struct Tensor {
  void* p;
  const void* g;
  bf16_t* copy;
  void *m, *v;
  unsigned char *ms, *vs;
  unsigned n, number;
};
struct Batch {
  Tensor t[kTensors];
  unsigned first[kTensors];                      // workgroup that a tensor begins with; past the last tensor: 2^32 - 1
};

struct Rule {
  double b1, b2;
  float lr, eps, decay;
  unsigned seed;
  long long step;
  const float* grad_scale;
  const long long* step_dev;
  const float* lr_dev;
};

__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return x ^ (x >> 16);
}
constexpr uint32_t kPhi = 0x9E3779B1u;

// b^n for n >= 1.
__device__ __forceinline__ double power(double b, long long n) {
  double r = 1.0;
  for (; n > 0; n >>= 1) {
    if (n & 1) r *= b;
    b *= b;
  }
  return r;
}

// The two formats.  kBias: the smallest number with a whole fraction is 2^(1 - kBias) under a scale of 1.  kTop: exponent of the
// block's largest under its scale, one below the format's own, so that a value rounded up still has a code.
struct First {
  static constexpr int kTop = 7, kBias = 7;
  static constexpr uint32_t kMagnitude = 127;
};
struct Second {
  static constexpr int kTop = 15, kBias = 15;
  static constexpr uint32_t kMagnitude = 255;
};

template <typename F>
__device__ __forceinline__ uint32_t scale_byte(float largest) {
  const int e = (int)(__float_as_uint(largest) >> 23) & 255;
  return e == 255 ? 255u : (uint32_t)max(e - F::kTop, F::kTop);
}
// 2^(byte - bias) in fp64: what a code's bits, taken as those of an fp32 from bit 20 on, are to be multiplied by.
template <typename F>
__device__ __forceinline__ double decode_factor(uint32_t byte) {
  if (byte == 255) return __longlong_as_double(0x7ff8000000000000LL);
  return __longlong_as_double((long long)((int)byte - F::kBias + 1023) << 52);
}
template <typename F>
__device__ __forceinline__ double decode(uint32_t code, double factor) {
  const double x = (double)__uint_as_float((code & F::kMagnitude) << 20) * factor;
  return F::kMagnitude == 127 && (code & 128) ? -x : x;
}
// The code of a magnitude (bits of an fp32): 20 bits of fraction are dropped after the random number, 16 bits under the
// code's last, has been added to them.  Below the format's smallest whole exponent the spacing stays that exponent's.
template <typename F>
__device__ __forceinline__ uint32_t encode(uint32_t bits, uint32_t byte, uint32_t random16) {
  const int smallest = (int)byte + 1 - F::kBias;             // its biased fp32 exponent, at least 1
  const int e = (int)(bits >> 23);
  const uint32_t whole = (bits & 0x7fffffu) | (e > 0 ? 0x800000u : 0u);
  const int under = smallest - max(e, 1);
  const uint32_t fixed = under <= 0 ? bits - ((uint32_t)(smallest - 1) << 23) : whole >> min(under, 31);
  return (fixed + (random16 << 4)) >> 20;
}

// Largest of the 32 elements of the four lanes that share a block.
__device__ __forceinline__ float block_max(const float* x) {
  float a = fabsf(x[0]);
  bool bad = x[0] != x[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) {
    a = fmaxf(a, fabsf(x[k]));
    bad |= x[k] != x[k];
  }
  if (bad) a = __builtin_inff();                             // a NaN counts as an infinity: no maximum drops it
  a = fmaxf(a, dpp_move<kDppQuadXor1>(a));
  return fmaxf(a, dpp_move<kDppQuadXor2>(a));
}

__device__ __forceinline__ u32x2 load_codes(const unsigned char* p, int n) {
  if (n == 8) return *reinterpret_cast<const u32x2*>(p);
  u32x2 q = {0u, 0u};
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < n) q[k >> 2] |= (uint32_t)p[k] << (8 * (k & 3));
  return q;
}
__device__ __forceinline__ void store_codes(unsigned char* p, int n, u32x2 q) {
  if (n == 8) {
    *reinterpret_cast<u32x2*>(p) = q;
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < n) p[k] = (unsigned char)(q[k >> 2] >> (8 * (k & 3)));
}
__device__ __forceinline__ uint32_t byte_of(u32x2 q, int k) { return (q[k >> 2] >> (8 * (k & 3))) & 255u; }

template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float* x) {
  if (n == 8) Eight<T>::unpack(Eight<T>::load(p), x);
  else load_some(p, n, x);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float* x) {
  if (n == 8) Eight<T>::store(p, x);
  else store_some(p, n, x);
}

template <typename P, typename G, bool BYTES>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Batch batch, Rule rule) {
  int k = 0;
#pragma unroll
  for (int i = 1; i < kTensors; ++i) k += blockIdx.x >= batch.first[i] ? 1 : 0;
  const Tensor t = batch.t[k];
  const size_t at = (size_t)(blockIdx.x - batch.first[k]) * kChunk + 8 * threadIdx.x;
  if (!BYTES && at >= t.n) return;
  const int n = (int)min((long long)t.n - (long long)min(at, (size_t)t.n), 8LL);    // lanes past the end help with a block's scale
  const long long step = rule.step_dev != nullptr ? *rule.step_dev : rule.step;
  const float lr = rule.lr_dev != nullptr ? *rule.lr_dev : rule.lr;
  const double scale = rule.grad_scale != nullptr ? (double)*rule.grad_scale : 1.0;
  const float c1 = (float)(1.0 / (1.0 - power(rule.b1, step))), c2 = (float)(1.0 / (1.0 - power(rule.b2, step)));
  float p[8], g[8];
  load8(static_cast<const P*>(t.p) + at, n, p);
  load8(static_cast<const G*>(t.g) + at, n, g);
  double m[8] = {}, v[8] = {};
  if constexpr (BYTES) {
    if (n > 0) {
      const u32x2 mc = load_codes(static_cast<const unsigned char*>(t.m) + at, n), vc = load_codes(static_cast<const unsigned char*>(t.v) + at, n);
      const double mf = decode_factor<First>(t.ms[at >> 5]), vf = decode_factor<Second>(t.vs[at >> 5]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = decode<First>(byte_of(mc, j), mf);
        v[j] = decode<Second>(byte_of(vc, j), vf);
      }
    }
  } else {
    float x[8];
    load8(static_cast<const float*>(t.m) + at, n, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] = (double)x[j];
    load8(static_cast<const float*>(t.v) + at, n, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (double)x[j];
  }
  float m1[8], v1[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const double gs = (double)g[j] * scale;
    m1[j] = j < n ? (float)(rule.b1 * m[j] + (1.0 - rule.b1) * gs) : 0.f;
    v1[j] = j < n ? (float)(rule.b2 * v[j] + (1.0 - rule.b2) * (gs * gs)) : 0.f;
    p[j] -= lr * (rule.decay * p[j] + m1[j] * c1 / (sqrtf(v1[j] * c2) + rule.eps));
  }
  if (n > 0) {
    store8(static_cast<P*>(t.p) + at, n, p);
    if (t.copy != nullptr) store8(t.copy + at, n, p);
  }
  if constexpr (BYTES) {
    const uint32_t mb = scale_byte<First>(block_max(m1)), vb = scale_byte<Second>(block_max(v1));
    if (n <= 0) return;
    const uint32_t key = mix(mix(rule.seed ^ (uint32_t)step * kPhi) ^ t.number * kPhi);
    u32x2 mc = {0u, 0u}, vc = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t random = mix(((uint32_t)at + j) * kPhi ^ key);
      const uint32_t mbits = __float_as_uint(m1[j]), vbits = __float_as_uint(v1[j]);
      uint32_t a = encode<First>(mbits & 0x7fffffffu, mb, random & 0xffffu);
      uint32_t b = encode<Second>(vbits, vb, random >> 16);
      if (vbits != 0) b = max(b, 1u);
      a |= mbits >> 31 << 7;
      if (mb == 255) a = 0;
      if (vb == 255) b = 0;
      mc[j >> 2] |= a << (8 * (j & 3));
      vc[j >> 2] |= b << (8 * (j & 3));
    }
    store_codes(static_cast<unsigned char*>(t.m) + at, n, mc);
    store_codes(static_cast<unsigned char*>(t.v) + at, n, vc);
    if ((threadIdx.x & 3) == 0) {
      t.ms[at >> 5] = (unsigned char)mb;
      t.vs[at >> 5] = (unsigned char)vb;
    }
  } else {
    store8(static_cast<float*>(t.m) + at, n, m1);
    store8(static_cast<float*>(t.v) + at, n, v1);
  }
}

template <typename F, typename T>
__global__ __launch_bounds__(kThreads) void adamw_values_kernel(const unsigned char* __restrict__ codes,
                                                                const unsigned char* __restrict__ scales, long long n,
                                                                T* __restrict__ out) {
  const long long at = 8 * ((long long)blockIdx.x * kThreads + threadIdx.x);
  if (at >= n) return;
  const int here = (int)min(n - at, 8LL);
  const u32x2 q = load_codes(codes + at, here);
  const double factor = decode_factor<F>(scales[at >> 5]);
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (float)decode<F>(byte_of(q, j), factor);
  store8(out + at, here, x);
}

}  // namespace

int launch_adamw_step(ais_ctx* ctx, const ais_adamw_tensor* tensors, int n_tensors, const ais_adamw_params& p,
                      const float* grad_scale, const long long* step_dev, const float* lr_dev) {
  ScopedTimer timer(ctx, AIS_K_ADAMW);
  const Rule rule{p.beta1, p.beta2, (float)p.lr, (float)p.eps, (float)p.weight_decay, p.seed, p.step, grad_scale, step_dev, lr_dev};
  hipError_t error = hipSuccess;
  auto run = [&](auto kernel, int param_dtype, int grad_dtype) {
    Batch batch;
    int held = 0;
    unsigned blocks = 0;
    auto flush = [&] {
      if (held == 0) return;
      for (int k = held; k < kTensors; ++k) batch.first[k] = 0xffffffffu;
      kernel<<<dim3(blocks), dim3(kThreads), 0, ctx->stream>>>(batch, rule);
      if (error == hipSuccess) error = hipGetLastError();
      held = 0;
      blocks = 0;
    };
    for (int i = 0; i < n_tensors; ++i) {
      const ais_adamw_tensor& t = tensors[i];
      if (t.n == 0 || t.param_dtype != param_dtype || t.grad_dtype != grad_dtype) continue;
      batch.t[held] = {t.param, t.grad, static_cast<bf16_t*>(t.copy), t.m, t.v, t.m_scale, t.v_scale, (unsigned)t.n, (unsigned)i};
      batch.first[held++] = blocks;
      blocks += (unsigned)((t.n + kChunk - 1) / kChunk);
      if (held == kTensors) flush();
    }
    flush();
  };
  auto types = [&](auto bytes) {
    constexpr bool kBytes = decltype(bytes)::value;
    run(adamw_kernel<float, float, kBytes>, AIS_F32, AIS_F32);
    run(adamw_kernel<float, bf16_t, kBytes>, AIS_F32, AIS_BF16);
    run(adamw_kernel<bf16_t, float, kBytes>, AIS_BF16, AIS_F32);
    run(adamw_kernel<bf16_t, bf16_t, kBytes>, AIS_BF16, AIS_BF16);
  };
  if (p.state_bits == 8) types(std::true_type{});
  else types(std::false_type{});
  return hip_fail(ctx, error);
}

int launch_adamw_values(ais_ctx* ctx, const unsigned char* codes, const unsigned char* scales, long long n, int moment,
                        void* out, ais_dtype dtype) {
  if (n == 0) return AIS_OK;
  ScopedTimer timer(ctx, AIS_K_ADAMW);
  auto run = [&](auto* to, auto format) {
    typedef std::remove_pointer_t<decltype(to)> T;
    adamw_values_kernel<decltype(format), T>
        <<<dim3((unsigned)((n + kChunk - 1) / kChunk)), dim3(kThreads), 0, ctx->stream>>>(codes, scales, n, to);
  };
  auto typed = [&](auto* to) {
    if (moment == 1) run(to, First{});
    else run(to, Second{});
  };
  if (dtype == AIS_BF16) typed(static_cast<bf16_t*>(out));
  else typed(static_cast<float*>(out));
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
