// An AdamW step over many tensors in one launch, with moments of 32 or 8 bits.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (wd p + m / c1 / (sqrt(v / c2) + eps)),  c = 1 - b^step
//
// Bound by memory: every array is read once and written once, 28 bytes an element with fp32 arrays and 16.1 with 8-bit moments.
// The gradients' addresses, which change from step to step, are kernel arguments, so that a call copies nothing to the GPU and can be
// recorded; all else about the tensors lies in a table on the GPU.  A lane takes vectors of four consecutive elements; eight lanes have a
// block of 32 whose 8-bit moments share a scale.
//
// The moments are formed in 64 bits (the GPU's fp64 is as fast as its fp32) and rounded to fp32: which of two 8-bit codes a value
// goes to depends on its last bits.
#include <algorithm>
#include <type_traits>

#include "ais_internal.h"
#include "eights.h"

namespace ais {
namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr int kVector = 4;                       // elements that a lane loads at once: 16 bytes of fp32
// Vectors of a lane, all on their way together: one of 8-bit moments, whose arithmetic is as long as their way, two of fp32.  us with one, two and
// four: 622 million elements with 8-bit moments 1,878, 1,972, 1,977, 150 small tensors 8.3, 9.7, 14; 86 million with fp32 moments 324, 320, 318.
__host__ __device__ constexpr int vectors_of(bool bytes) { return bytes ? 1 : 2; }
__host__ __device__ constexpr int chunk_of(bool bytes) { return kVector * vectors_of(bytes) * kThreads; }     // elements of a workgroup
constexpr int kTensors = 320;                    // of a launch: a gradient's address and a number each, of the 4 KiB of kernel arguments

// What a launch carries: of each tensor where its gradient is, with 1 added if that is bf16, and the workgroup that it begins with.  One that
// is left out begins where the next one does; past the last tensor: 2^32 - 1.
struct Batch {
  uintptr_t grad[kTensors];
  unsigned first[kTensors];
};
static_assert(sizeof(Batch) + 128 <= 4096, "");
// Workgroups of a launch, which may have no more than 2^32 - 1 threads: 2^31 here.  A tensor has 2^22 at most.
constexpr long long kMostBlocks = (1LL << 31) / kThreads;
// Elements whose values a launch gives out.  (Workgroups that go on behind the others take 700 instead of 670 us for 622 million elements.)
constexpr long long kMostValues = 1LL << 31;

struct Rule {
  double b1, b2;
  double c1, c2;                                 // 1 / (1 - b^step); of no meaning with step_dev
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
__host__ __device__ __forceinline__ double power(double b, long long n) {
  double r = 1.0;
  for (; n > 0; n >>= 1) {
    if (n & 1) r *= b;
    b *= b;
  }
  return r;
}

// The rule with what is in device memory.
struct Now {
  long long step;
  double b1, b2, g1, g2;                         // of the moments, of the gradient and its square
  float c2, c2_small, decay, rate;               // v's correction, and times 2^64; lr with the decay, and with m's correction
  __device__ __forceinline__ explicit Now(const Rule& r) : step(r.step), b1(r.b1), b2(r.b2) {
    double c1d = r.c1, c2d = r.c2, scale = 1.0;
    float lr = r.lr;
    if (r.step_dev != nullptr) {                 // uniform, as all of these
      step = *r.step_dev;
      c1d = 1.0 / (1.0 - power(b1, step));
      c2d = 1.0 / (1.0 - power(b2, step));
    }
    if (r.lr_dev != nullptr) lr = *r.lr_dev;
    if (r.grad_scale != nullptr) scale = (double)*r.grad_scale;
    g1 = (1.0 - b1) * scale;
    g2 = (1.0 - b2) * (scale * scale);
    c2 = (float)c2d;
    c2_small = c2 * 0x1p64f;                     // at most 2^53 times that: 1 - b2 is at least 2^-53
    decay = (float)((double)lr * (double)r.decay);
    rate = (float)((double)lr * c1d);
  }
};

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
// What a code's bits, taken as those of an fp32 from bit 20 on, are to be multiplied by: 2^(byte - bias), in fp64.
template <typename F>
__device__ __forceinline__ double decode_factor(uint32_t byte) {
  if (byte == 255) return __longlong_as_double(0x7ff8000000000000LL);
  return __longlong_as_double((long long)((int)byte - F::kBias + 1023) << 52);
}
template <typename F>
__device__ __forceinline__ float code_bits(uint32_t code) {
  const uint32_t magnitude = (code & F::kMagnitude) << 20;
  return __uint_as_float(F::kMagnitude == 127 ? magnitude | (code & 128) << 24 : magnitude);
}
// The code of a magnitude (bits of an fp32): 20 bits of fraction are dropped after the random number, 16 bits under the
// code's last, has been added to them.  Below the format's smallest whole exponent the spacing stays that exponent's.
template <typename F>
__device__ __forceinline__ uint32_t encode(uint32_t bits, uint32_t byte, uint32_t random16) {
  const uint32_t smallest = byte + 1 - F::kBias;             // its biased fp32 exponent, at least 1
  // in units of 2^-23 of that exponent; the multiplication is exact where the number is below 2^23 of them, the conversion cuts
  const uint32_t low = (uint32_t)__builtin_ldexpf(__uint_as_float(bits), 150 - (int)smallest);
  const uint32_t fixed = bits < smallest << 23 ? low : bits - ((smallest - 1) << 23);
  return (fixed + (random16 << 4)) >> 20;
}

// sqrt(v c2) + eps.  The root is the hardware's, which takes subnormal numbers for 0: small squares are scaled before and behind it.
constexpr float kSmall = 0x1p-100f;
__device__ __forceinline__ float root_of(float v, const Now& now, float eps) {
  const bool small = v < kSmall;
  return __builtin_fmaf(__builtin_amdgcn_sqrtf(v * (small ? now.c2_small : now.c2)), small ? 0x1p-32f : 1.f, eps);
}

// Largest of the 32 elements of the eight lanes that share a block; a NaN counts as an infinity, since no maximum drops that.
__device__ __forceinline__ float block_max(const float* x) {
  float a = 0.f;
#pragma unroll
  for (int k = 0; k < kVector; ++k) a = fmaxf(a, x[k] == x[k] ? fabsf(x[k]) : __builtin_inff());
  a = fmaxf(a, dpp_move<kDppQuadXor1>(a));
  a = fmaxf(a, dpp_move<kDppQuadXor2>(a));
  return fmaxf(a, dpp_move<kDppRowHalfMirror>(a));
}

// Vectors of a lane, the last one of a tensor in part.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int n, bool whole, float* x) {
  typedef Pack<T, kVector> P;
  if (whole) {
    P::unpack(__builtin_nontemporal_load(reinterpret_cast<const typename P::Any*>(p)), x);
    return;
  }
#pragma unroll
  for (int k = 0; k < kVector; ++k) x[k] = k < n ? Vec<T>::load1(p + k) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int n, bool whole, const float* x) {
  typedef Pack<T, kVector> P;
  if (whole) {
    __builtin_nontemporal_store((typename P::Any)P::pack(x), reinterpret_cast<typename P::Any*>(p));
    return;
  }
#pragma unroll
  for (int k = 0; k < kVector; ++k)
    if (k < n) Vec<T>::store1(p + k, x[k]);
}
__device__ __forceinline__ uint32_t load_codes(const unsigned char* p, int n, bool whole) {
  if (whole) return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
  uint32_t q = 0;
#pragma unroll
  for (int k = 0; k < kVector; ++k)
    if (k < n) q |= (uint32_t)p[k] << (8 * k);
  return q;
}
__device__ __forceinline__ void store_codes(unsigned char* p, int n, bool whole, uint32_t q) {
  if (whole) {
    __builtin_nontemporal_store(q, reinterpret_cast<uint32_t*>(p));
    return;
  }
#pragma unroll
  for (int k = 0; k < kVector; ++k)
    if (k < n) p[k] = (unsigned char)(q >> (8 * k));
}

// A lane's part of a chunk.  WHOLE: every element of the chunk is there.
template <typename P, typename G, bool BYTES, bool WHOLE>
__device__ __forceinline__ void step_chunk(const ais_adamw_tensor& t, const G* grad, int number, const Rule& rule, size_t base) {
  constexpr int kVectors = vectors_of(BYTES);
  size_t at[kVectors];
  int n[kVectors];
  float p[kVectors][kVector], g[kVectors][kVector], m[kVectors][kVector], v[kVectors][kVector];
  uint32_t mc[kVectors], vc[kVectors], ms[kVectors], vs[kVectors];
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    at[i] = base + kVector * (i * kThreads + threadIdx.x);
    n[i] = WHOLE ? kVector : (int)min(max((long long)t.n - (long long)at[i], 0LL), (long long)kVector);
    const bool whole = WHOLE || n[i] == kVector;
    load4(static_cast<const P*>(t.param) + at[i], n[i], whole, p[i]);
    load4(grad + at[i], n[i], whole, g[i]);
    if constexpr (BYTES) {
      mc[i] = load_codes(static_cast<const unsigned char*>(t.m) + at[i], n[i], whole);
      vc[i] = load_codes(static_cast<const unsigned char*>(t.v) + at[i], n[i], whole);
      ms[i] = WHOLE || n[i] > 0 ? t.m_scale[at[i] >> 5] : 0;
      vs[i] = WHOLE || n[i] > 0 ? t.v_scale[at[i] >> 5] : 0;
    } else {
      load4(static_cast<const float*>(t.m) + at[i], n[i], whole, m[i]);
      load4(static_cast<const float*>(t.v) + at[i], n[i], whole, v[i]);
    }
  }
  const Now now(rule);
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const bool whole = WHOLE || n[i] == kVector;
    double mb = now.b1, vb = now.b2;                         // what the moments' numbers are multiplied by
    if constexpr (BYTES) {
      mb *= decode_factor<First>(ms[i]);
      vb *= decode_factor<Second>(vs[i]);
#pragma unroll
      for (int j = 0; j < kVector; ++j) {
        m[i][j] = code_bits<First>(mc[i] >> (8 * j) & 255u);
        v[i][j] = code_bits<Second>(vc[i] >> (8 * j) & 255u);
      }
    }
#pragma unroll
    for (int j = 0; j < kVector; ++j) {
      const double gs = (double)g[i][j];
      m[i][j] = (float)__builtin_fma(mb, (double)m[i][j], now.g1 * gs);
      v[i][j] = (float)__builtin_fma(vb, (double)v[i][j], now.g2 * (gs * gs));
      if (!WHOLE && j >= n[i]) m[i][j] = v[i][j] = 0.f;
      const float ahead = m[i][j] * __builtin_amdgcn_rcpf(root_of(v[i][j], now, rule.eps));
      p[i][j] -= __builtin_fmaf(now.decay, p[i][j], now.rate * ahead);
    }
    store4(static_cast<P*>(t.param) + at[i], n[i], whole, p[i]);
    if (t.copy != nullptr) store4(static_cast<bf16_t*>(t.copy) + at[i], n[i], whole, p[i]);
    if constexpr (BYTES) {
      const uint32_t mbyte = scale_byte<First>(block_max(m[i])), vbyte = scale_byte<Second>(block_max(v[i]));
      const uint32_t key = mix(mix(rule.seed ^ (uint32_t)now.step * kPhi) ^ (uint32_t)number * kPhi);
      const uint32_t place = (uint32_t)at[i] * kPhi;
      uint32_t a = 0, b = 0;
#pragma unroll
      for (int j = 0; j < kVector; ++j) {
        const uint32_t random = mix((place + j * kPhi) ^ key);
        const uint32_t mbits = __float_as_uint(m[i][j]), vbits = __float_as_uint(v[i][j]);
        const uint32_t first = encode<First>(mbits & 0x7fffffffu, mbyte, random & 0xffffu) | (mbits >> 24 & 128u);
        uint32_t second = encode<Second>(vbits, vbyte, random >> 16);
        if (vbits != 0) second = max(second, 1u);
        a |= first << (8 * j);
        b |= second << (8 * j);
      }
      if (mbyte == 255) a = 0;
      if (vbyte == 255) b = 0;
      store_codes(static_cast<unsigned char*>(t.m) + at[i], n[i], whole, a);
      store_codes(static_cast<unsigned char*>(t.v) + at[i], n[i], whole, b);
      if ((threadIdx.x & 7) == 0 && (WHOLE || n[i] > 0)) {
        t.m_scale[at[i] >> 5] = (unsigned char)mbyte;
        t.v_scale[at[i] >> 5] = (unsigned char)vbyte;
      }
    } else {
      store4(static_cast<float*>(t.m) + at[i], n[i], whole, m[i]);
      store4(static_cast<float*>(t.v) + at[i], n[i], whole, v[i]);
    }
  }
}

// `table`: the tensors from the launch's first on, of which `number` come before.
template <bool BYTES>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Batch batch, const ais_adamw_tensor* __restrict__ table, int number, Rule rule) {
  // every wavefront looks for the workgroup's tensor: the last that begins with it or before it
  int k = -1;
#pragma unroll
  for (int i = 0; i < kTensors; i += 64) k += __popcll(__ballot(batch.first[i + (threadIdx.x & 63)] <= blockIdx.x));
  k = __builtin_amdgcn_readfirstlane(k);
  const ais_adamw_tensor t = table[k];
  const uintptr_t grad = batch.grad[k];
  const size_t base = (size_t)(blockIdx.x - batch.first[k]) * chunk_of(BYTES);
  auto run = [&](auto* param, const auto* g) {
    typedef std::remove_pointer_t<decltype(param)> P;
    typedef std::remove_cv_t<std::remove_pointer_t<decltype(g)>> G;
    if (base + chunk_of(BYTES) <= (size_t)t.n) step_chunk<P, G, BYTES, true>(t, g, number + k, rule, base);
    else step_chunk<P, G, BYTES, false>(t, g, number + k, rule, base);
  };
  auto typed = [&](auto* param) {
    if (grad & 1) run(param, reinterpret_cast<const bf16_t*>(grad - 1));
    else run(param, reinterpret_cast<const float*>(grad));
  };
  if (t.param_dtype == AIS_BF16) typed(static_cast<bf16_t*>(nullptr));
  else typed(static_cast<float*>(nullptr));
}

template <typename F, typename T>
__device__ __forceinline__ void values_of(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                          long long n, T* __restrict__ out) {
  const long long at = 8 * ((long long)blockIdx.x * kThreads + threadIdx.x);
  if (at >= n) return;
  const int here = (int)min(n - at, 8LL);
  const double factor = decode_factor<F>(scales[at >> 5]);
  uint32_t q[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) q[k] = load_codes(codes + at + 4 * k, here - 4 * k, here >= 4 * k + 4);
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (float)((double)code_bits<F>(q[j >> 2] >> (8 * (j & 3)) & 255u) * factor);
  if (here == 8) Eight<T>::store(out + at, x);
  else store_some(out + at, here, x);
}
template <typename T>
__global__ __launch_bounds__(kThreads) void adamw_values_kernel(const unsigned char* m, const unsigned char* m_scale,
                                                                const unsigned char* v, const unsigned char* v_scale, long long n,
                                                                T* m_out, T* v_out) {
  if (blockIdx.y == 0 && m_out != nullptr) values_of<First>(m, m_scale, n, m_out);
  else values_of<Second>(v, v_scale, n, v_out);
}

}  // namespace

int launch_adamw_step(ais_ctx* ctx, const ais_adamw_tensor* tensors, const ais_adamw_tensor* table, int n_tensors,
                      const ais_adamw_params& p, const float* grad_scale, const long long* step_dev, const float* lr_dev) {
  ScopedTimer timer(ctx, AIS_K_ADAMW);
  auto correction = [&](double b) { return step_dev == nullptr ? 1.0 / (1.0 - power(b, p.step)) : 1.0; };
  const Rule rule{p.beta1, p.beta2, correction(p.beta1), correction(p.beta2), (float)p.lr, (float)p.eps, (float)p.weight_decay,
                  p.seed, p.step, grad_scale, step_dev, lr_dev};
  const int chunk = chunk_of(p.state_bits == 8);
  for (int from = 0, behind; from < n_tensors; from = behind) {
    // the tensors before `behind`: as many as a launch has arguments for, whose workgroups it can have
    Batch batch;
    long long blocks = 0;
    behind = n_tensors;
    for (int k = 0; k < kTensors; ++k) {
      batch.first[k] = 0xffffffffu;
      batch.grad[k] = 0;
      if (from + k >= behind) continue;
      const ais_adamw_tensor& t = tensors[from + k];
      const long long here = t.grad != nullptr ? (t.n + chunk - 1) / chunk : 0;
      if (blocks + here > kMostBlocks) {
        behind = from + k;
        continue;
      }
      batch.first[k] = (unsigned)blocks;
      blocks += here;
      if (here > 0) batch.grad[k] = reinterpret_cast<uintptr_t>(t.grad) + (t.grad_dtype == AIS_BF16 ? 1 : 0);
    }
    behind = std::min(behind, from + kTensors);
    if (blocks == 0) continue;
    auto kernel = p.state_bits == 8 ? adamw_kernel<true> : adamw_kernel<false>;
    kernel<<<dim3((unsigned)blocks), dim3(kThreads), 0, ctx->stream>>>(batch, table + from, from, rule);
    const int rc = hip_fail(ctx, hipGetLastError());
    if (rc != AIS_OK) return rc;
  }
  return AIS_OK;
}

int launch_adamw_values(ais_ctx* ctx, const unsigned char* m, const unsigned char* m_scale, const unsigned char* v,
                        const unsigned char* v_scale, long long n, void* m_out, void* v_out, ais_dtype dtype) {
  const unsigned moments = (m_out != nullptr) + (v_out != nullptr);
  if (n == 0 || moments == 0) return AIS_OK;
  ScopedTimer timer(ctx, AIS_K_ADAMW);
  auto run = [&](auto* m_to, auto* v_to) {
    for (long long at = 0; at < n; at += kMostValues) {
      const long long here = std::min(n - at, kMostValues);
      auto from = [&](auto* p, long long behind) { return p != nullptr ? p + behind : p; };
      adamw_values_kernel<<<dim3((unsigned)((here + 8 * kThreads - 1) / (8 * kThreads)), moments), dim3(kThreads), 0, ctx->stream>>>(
          from(m, at), from(m_scale, at / 32), from(v, at), from(v_scale, at / 32), here, from(m_to, at), from(v_to, at));
    }
  };
  if (dtype == AIS_BF16) run(static_cast<bf16_t*>(m_out), static_cast<bf16_t*>(v_out));
  else run(static_cast<float*>(m_out), static_cast<float*>(v_out));
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
