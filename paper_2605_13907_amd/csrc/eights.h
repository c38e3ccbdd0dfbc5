// Groups of consecutive elements of bf16 or fp32 arrays that begin at any element: what a lane loads, computes in fp32 and stores.
#pragma once

#include "device_utils.h"

namespace ais {
namespace dev {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  typedef Unaligned<bf16_t>::four Any;
  struct Raw { u32x4 q; };
  static __device__ __forceinline__ Raw load(const bf16_t* p) {
    return {__builtin_nontemporal_load(reinterpret_cast<const Any*>(p))};
  }
  static __device__ __forceinline__ Raw load_kept(const bf16_t* p) { return {*reinterpret_cast<const Any*>(p)}; }
  static __device__ __forceinline__ Raw zero() { return {u32x4{0u, 0u, 0u, 0u}}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float* x) { Vec<bf16_t>::unpack(r.q, x); }
  static __device__ __forceinline__ void store(bf16_t* p, const float* x) {
    __builtin_nontemporal_store((Any)Vec<bf16_t>::pack(x), reinterpret_cast<Any*>(p));
  }
};
template <> struct Eight<float> {
  typedef Unaligned<float>::four Any;
  struct Raw { u32x4 q[2]; };
  static __device__ __forceinline__ Raw load(const float* p) {
    return {{__builtin_nontemporal_load(reinterpret_cast<const Any*>(p)), __builtin_nontemporal_load(reinterpret_cast<const Any*>(p) + 1)}};
  }
  static __device__ __forceinline__ Raw load_kept(const float* p) {
    return {{*reinterpret_cast<const Any*>(p), *(reinterpret_cast<const Any*>(p) + 1)}};
  }
  static __device__ __forceinline__ Raw zero() { return {{u32x4{0u, 0u, 0u, 0u}, u32x4{0u, 0u, 0u, 0u}}}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float* x) {
    Vec<float>::unpack(r.q[0], x);
    Vec<float>::unpack(r.q[1], x + 4);
  }
  static __device__ __forceinline__ void store(float* p, const float* x) {
    __builtin_nontemporal_store((Any)Vec<float>::pack(x), reinterpret_cast<Any*>(p));
    __builtin_nontemporal_store((Any)Vec<float>::pack(x + 4), reinterpret_cast<Any*>(p) + 1);
  }
};

// N elements that a lane loads and stores at once, from any element on: 16 bytes, or 8 of bf16 beside 16 of fp32.
template <typename T, int N> struct Pack {
  typedef u32x4 Raw;
  typedef typename Unaligned<T>::four Any;
  static __device__ __forceinline__ void unpack(Raw q, float* x) { Vec<T>::unpack(q, x); }
  static __device__ __forceinline__ Raw pack(const float* x) { return Vec<T>::pack(x); }
  static __device__ __forceinline__ Raw zero() { return Raw{0u, 0u, 0u, 0u}; }
};
template <> struct Pack<bf16_t, 4> {
  typedef u32x2 Raw;
  typedef Unaligned<bf16_t>::two Any;
  static __device__ __forceinline__ void unpack(Raw q, float* x) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x[2 * k] = __uint_as_float(q[k] << 16);
      x[2 * k + 1] = __uint_as_float(q[k] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw pack(const float* x) {
    Raw q;
#pragma unroll
    for (int k = 0; k < 2; ++k) q[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * k], x[2 * k + 1]}, bf16x2));
    return q;
  }
  static __device__ __forceinline__ Raw zero() { return Raw{0u, 0u}; }
};

// The first n (1 to 7) of eight elements, the others 0.
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float* x) {
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = k < n ? Vec<T>::load1(p + k) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float* x) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < n) Vec<T>::store1(p + k, x[k]);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off);
  return v;
}

}  // namespace dev
}  // namespace ais
