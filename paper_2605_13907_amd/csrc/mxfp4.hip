// Microscaled 4-bit floating point (MXFP4): rows of blocks of 32 E2M1 elements under one E8M0 scale.
#include "ais_internal.h"
#include "device_utils.h"

namespace ais {
namespace {

using namespace dev;

constexpr int kBlock = 32;             // elements under one scale
constexpr int kUnit = 8;               // elements of a lane: four lanes share a block
constexpr int kQuantThreads = 256;

// ---- quantisation ---------------------------------------------------------------------------------------------------
// e = floor(log2 max|x|) - 2 comes from the exponent bits of the largest magnitude, compared as bit patterns: that order has
// infinities and NaN at its top.  x 2^-e is exact, and so is q 2^e in either type, so the only rounding is the one to E2M1.
// A lane holds 8 consecutive elements, and two exchanges inside a quad of lanes find the block's largest.
// Bound by HBM: e R D bytes in, 17 bytes a block out, and e R D bytes where the values are asked for.  151,936 bf16 rows x 4,096
// with values 450 us, 6.3 TB/s; 64 rows 3.4 us, which is the launch.  A lane has one unit: with four, one after the other, these
// were 503 and 4.4.  Rows begin at any element: vectors that lie anywhere cost 151,936 x 1,025 125 us, single elements 392.

template <typename T>
__device__ __forceinline__ void load_unit(const T* p, int left, float* x) {
  typedef typename Unaligned<T>::four Any;
  if (left >= kUnit) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int k = 0; k < kUnit / N; ++k) Vec<T>::unpack(__builtin_nontemporal_load(reinterpret_cast<const Any*>(p + k * N)), x + k * N);
  } else {
#pragma unroll
    for (int k = 0; k < kUnit; ++k) x[k] = k < left ? Vec<T>::load1(p + k) : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ void store_unit(T* p, int left, const float* x) {
  typedef typename Unaligned<T>::four Any;
  if (left >= kUnit) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int k = 0; k < kUnit / N; ++k) __builtin_nontemporal_store((Any)Vec<T>::pack(x + k * N), reinterpret_cast<Any*>(p + k * N));
  } else {
#pragma unroll
    for (int k = 0; k < kUnit; ++k)
      if (k < left) Vec<T>::store1(p + k, x[k]);
  }
}

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppQuadXor1, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppQuadXor2, 0xf, 0xf, true));
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mxfp4_quantize_kernel(
    const T* x, long long row_stride, int width, int row_units, long long n_units, unsigned char* __restrict__ codes,
    long long codes_stride, unsigned char* __restrict__ scales, long long scales_stride, T* values, long long values_stride) {
  const long long first = (long long)blockIdx.x * kQuantThreads;
  const long long row0 = first / row_units;
  if (first + threadIdx.x >= n_units) return;          // units come in fours: a quad of lanes leaves together
  const uint32_t off = (uint32_t)(first - row0 * row_units) + threadIdx.x;
  const uint32_t down = off / (uint32_t)row_units;
  const long long row = row0 + down;
  const int unit = (int)(off - down * (uint32_t)row_units);
  const int left = width - unit * kUnit;               // may be <= 0 in the last block
  float v[kUnit];
  load_unit(x + row * row_stride + (long long)unit * kUnit, left, v);
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kUnit; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = quad_max(top);
  const bool finite = top < 0x7f800000u;
  const int e = max((int)(top >> 23) - 2, 0);          // the scale's byte, exponent + 127
  const float down_scale = __uint_as_float((uint32_t)(254 - e) << 23);
  uint32_t word = 0;
#pragma unroll
  for (int j = 0; j < kUnit; ++j) v[j] *= down_scale;
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0], v[1], 1.f, 0);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2], v[3], 1.f, 1);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4], v[5], 1.f, 2);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6], v[7], 1.f, 3);
  if (!finite) word = 0;
  *reinterpret_cast<uint32_t*>(codes + row * codes_stride + (long long)unit * (kUnit / 2)) = word;
  if ((unit & 3) == 0) scales[row * scales_stride + (unit >> 2)] = finite ? (unsigned char)e : (unsigned char)255;
  if (values != nullptr) {
    const float up = e > 0 ? __uint_as_float((uint32_t)e << 23) : __uint_as_float(1u << 22);   // 2^-127 is subnormal
    const float scale = finite ? up : __builtin_nanf("");
    const f32x2 q0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 0);
    const f32x2 q1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 1);
    const f32x2 q2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 2);
    const f32x2 q3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 3);
    const float out[kUnit] = {q0[0] * scale, q0[1] * scale, q1[0] * scale, q1[1] * scale,
                              q2[0] * scale, q2[1] * scale, q3[0] * scale, q3[1] * scale};
    store_unit(values + row * values_stride + (long long)unit * kUnit, left, out);
  }
}

}  // namespace

int launch_mxfp4_quantize(ais_ctx* ctx, const void* x, ais_dtype dtype, long long n_rows, int width, long long row_stride,
                          unsigned char* codes, long long codes_stride, unsigned char* scales, long long scales_stride,
                          void* values, long long values_stride) {
  if (n_rows == 0) return AIS_OK;
  ScopedTimer timer(ctx, AIS_K_MXFP4_QUANT);
  const int row_units = (width + kBlock - 1) / kBlock * (kBlock / kUnit);
  // no more than 2^31 threads to a launch
  const long long rows_at_once = (1LL << 31) / row_units;
  auto run = [&](auto type) {
    typedef decltype(type) T;
    for (long long r = 0; r < n_rows; r += rows_at_once) {
      const long long n_units = (n_rows - r < rows_at_once ? n_rows - r : rows_at_once) * row_units;
      mxfp4_quantize_kernel<T><<<dim3((unsigned)((n_units + kQuantThreads - 1) / kQuantThreads)), dim3(kQuantThreads), 0, ctx->stream>>>(
          static_cast<const T*>(x) + r * row_stride, row_stride, width, row_units, n_units, codes + r * codes_stride, codes_stride,
          scales + r * scales_stride, scales_stride, values != nullptr ? static_cast<T*>(values) + r * values_stride : nullptr,
          values_stride);
    }
  };
  if (dtype == AIS_BF16) run(bf16_t{});
  else run(float{});
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
