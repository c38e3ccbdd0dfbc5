// Rows normalised in front of the read-out, and their gradient.
//
//   norm:       y = (x - mean) rstd w + b, mean and variance over the row (or mean 0: root-mean-square norm)
//   norm_grad:  n = (x - mean) rstd, u = dy w:  dx = rstd (u - <u> - n <u n>), dw = sum_r dy n, db = sum_r dy
//
// Bound by memory: a row is read once into registers, its statistics are formed there (the variance from deviations, in a second
// pass over the registers, so that nothing cancels), and it is written once.  A lane holds groups of eight consecutive elements.
#include <algorithm>

#include "ais_internal.h"
#include "eights.h"

namespace ais {
namespace {

using namespace dev;

// Weight or bias of either type; null: the value it stands for.
struct Affine {
  const void* p;
  bool bf16;
  __device__ __forceinline__ void load(int at, float otherwise, float* x) const {
    if (p == nullptr) {                          // uniform
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = otherwise;
    } else if (bf16) {
      Eight<bf16_t>::unpack(Eight<bf16_t>::load_kept(static_cast<const bf16_t*>(p) + at), x);
    } else {
      Eight<float>::unpack(Eight<float>::load_kept(static_cast<const float*>(p) + at), x);
    }
  }
  __device__ __forceinline__ void load_some(int at, int n, float otherwise, float* x) const {
    if (p == nullptr) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = otherwise;
    } else if (bf16) {
      dev::load_some(static_cast<const bf16_t*>(p) + at, n, x);
    } else {
      dev::load_some(static_cast<const float*>(p) + at, n, x);
    }
  }
};

// Sum over the THREADS threads that share a row; `lds` holds a word for each of their wavefronts.
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  v = wave_sum(v);
  if (THREADS == 64) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
  return s;
}

__device__ __forceinline__ float sum8(const float* x) {
  return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}

// Group g of a row of `width` elements: whole, the last one in part, or past the end.
template <typename T>
__device__ __forceinline__ void load_group(const T* row, int g, int width, float* x) {
  const int left = width - 8 * g;
  if (left >= 8) Eight<T>::unpack(Eight<T>::load(row + 8 * g), x);
  else if (left > 0) load_some(row + 8 * g, left, x);
  else {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_group(T* row, int g, int width, const float* x) {
  const int left = width - 8 * g;
  if (left >= 8) Eight<T>::store(row + 8 * g, x);
  else if (left > 0) store_some(row + 8 * g, left, x);
}
__device__ __forceinline__ void load_group(const Affine& a, int g, int width, float otherwise, float* x) {
  const int left = width - 8 * g;
  if (left >= 8) a.load(8 * g, otherwise, x);
  else if (left > 0) a.load_some(8 * g, left, otherwise, x);
}

// A row to each workgroup, NG groups to a thread; NG = 0: any width, the row is read three times.
template <typename T, int THREADS, int NG>
__global__ __launch_bounds__(THREADS) void norm_kernel(const T* x, long long row_stride, int width,
                                                       const unsigned char* __restrict__ valid, Affine weight, Affine bias,
                                                       float eps, int centered, T* y, long long y_stride,
                                                       float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  __shared__ float lds[THREADS / 64];
  const long long row = blockIdx.x;
  const int tid = threadIdx.x, groups = (width - 1) / 8 + 1;
  const T* xr = x + row * row_stride;
  T* yr = y + row * y_stride;
  if (valid != nullptr && valid[row] == 0) {
    const float zero[8] = {};
    for (int g = tid; g < groups; g += THREADS) store_group(yr, g, width, zero);
    if (tid == 0) {
      if (centered) mean_out[row] = 0.f;
      rstd_out[row] = 0.f;
    }
    return;
  }
  const float n = (float)width;
  float mean = 0.f, rstd;
  if constexpr (NG > 0) {
    float v[NG][8];
#pragma unroll
    for (int k = 0; k < NG; ++k) load_group(xr, tid + k * THREADS, width, v[k]);
    if (centered) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NG; ++k) s += sum8(v[k]);
      mean = row_sum<THREADS>(s, lds) / n;
    }
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      float d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // elements past the end do not count
        v[k][j] = 8 * (tid + k * THREADS) + j < width ? v[k][j] - mean : 0.f;
        d[j] = v[k][j] * v[k][j];
      }
      q += sum8(d);
    }
    rstd = 1.f / sqrtf(row_sum<THREADS>(q, lds) / n + eps);
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      const int g = tid + k * THREADS;
      if (g >= groups) break;
      float w[8], b[8];
      load_group(weight, g, width, 1.f, w);
      load_group(bias, g, width, 0.f, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[k][j] = __builtin_fmaf(v[k][j] * rstd, w[j], b[j]);
      store_group(yr, g, width, v[k]);
    }
  } else {
    if (centered) {
      float s = 0.f;
      for (int g = tid; g < groups; g += THREADS) {
        float v[8];
        load_group(xr, g, width, v);
        s += sum8(v);
      }
      mean = row_sum<THREADS>(s, lds) / n;
    }
    float q = 0.f;
    for (int g = tid; g < groups; g += THREADS) {
      float v[8];
      load_group(xr, g, width, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = 8 * (long long)g + j < width ? v[j] - mean : 0.f;
        v[j] = d * d;
      }
      q += sum8(v);
    }
    rstd = 1.f / sqrtf(row_sum<THREADS>(q, lds) / n + eps);
    for (int g = tid; g < groups; g += THREADS) {
      float v[8], w[8], b[8];
      load_group(xr, g, width, v);
      load_group(weight, g, width, 1.f, w);
      load_group(bias, g, width, 0.f, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf((v[j] - mean) * rstd, w[j], b[j]);
      store_group(yr, g, width, v);
    }
  }
  if (tid == 0) {
    if (centered) mean_out[row] = mean;
    rstd_out[row] = rstd;
  }
}

// The gradient.  A workgroup takes every gridDim.x-th row and keeps the weight's and the bias's sums of its own columns in
// registers; they leave as one row of partials each, which norm_grad_sum_kernel adds up in their order.
template <typename T, typename D, int THREADS, int NG>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(const D* dy, long long dy_stride, const T* x, long long row_stride,
                                                            int n_rows, int width, const unsigned char* __restrict__ valid,
                                                            Affine weight, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, T* dx, long long dx_stride,
                                                            float* __restrict__ dweight, float* __restrict__ dbias) {
  __shared__ float lds[2][THREADS / 64];
  const int tid = threadIdx.x, groups = (width - 1) / 8 + 1;
  const float n = (float)width;
  float dw[NG][8] = {}, db[NG][8] = {};
  for (long long row = blockIdx.x; row < n_rows; row += gridDim.x) {
    T* dr = dx + row * dx_stride;
    if (valid != nullptr && valid[row] == 0) {
      const float zero[8] = {};
      for (int g = tid; g < groups; g += THREADS) store_group(dr, g, width, zero);
      continue;
    }
    const float mu = mean != nullptr ? mean[row] : 0.f, rs = rstd[row];
    float v[NG][8], u[NG][8];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      load_group(x + row * row_stride, tid + k * THREADS, width, v[k]);
      load_group(dy + row * dy_stride, tid + k * THREADS, width, u[k]);
    }
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      float w[8], p[8];
      if (tid + k * THREADS >= groups) break;
      load_group(weight, tid + k * THREADS, width, 1.f, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[k][j] = (v[k][j] - mu) * rs;
        db[k][j] += u[k][j];
        dw[k][j] = __builtin_fmaf(u[k][j], v[k][j], dw[k][j]);
        u[k][j] = 8 * (tid + k * THREADS) + j < width ? u[k][j] * w[j] : 0.f;
        p[j] = u[k][j] * v[k][j];
      }
      s1 += sum8(u[k]);
      s2 += sum8(p);
    }
    s1 = mean != nullptr ? row_sum<THREADS>(s1, lds[0]) / n : 0.f;
    s2 = row_sum<THREADS>(s2, lds[1]) / n;
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      if (tid + k * THREADS >= groups) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) u[k][j] = rs * (u[k][j] - s1 - v[k][j] * s2);
      store_group(dr, tid + k * THREADS, width, u[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < NG; ++k) {
    if (dweight != nullptr) store_group(dweight + (size_t)blockIdx.x * width, tid + k * THREADS, width, dw[k]);
    if (dbias != nullptr) store_group(dbias + (size_t)blockIdx.x * width, tid + k * THREADS, width, db[k]);
  }
}

// Rows too wide for that, in two kernels: <u> and <u n> of every row ...
constexpr int kWideThreads = 1024;
template <typename T, typename D>
__global__ __launch_bounds__(kWideThreads) void norm_grad_rows_kernel(const D* __restrict__ dy, long long dy_stride,
                                                                      const T* __restrict__ x, long long row_stride, int width,
                                                                      const unsigned char* __restrict__ valid, Affine weight,
                                                                      const float* __restrict__ mean,
                                                                      const float* __restrict__ rstd, float* __restrict__ sums) {
  __shared__ float lds[2][kWideThreads / 64];
  const long long row = blockIdx.x;
  if (valid != nullptr && valid[row] == 0) return;
  const int tid = threadIdx.x, groups = (width - 1) / 8 + 1;
  const float mu = mean != nullptr ? mean[row] : 0.f, rs = rstd[row];
  float s1 = 0.f, s2 = 0.f;
  for (int g = tid; g < groups; g += kWideThreads) {
    float v[8], u[8], w[8] = {};
    load_group(x + row * row_stride, g, width, v);
    load_group(dy + row * dy_stride, g, width, u);
    load_group(weight, g, width, 1.f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u[j] = 8 * (long long)g + j < width ? u[j] * w[j] : 0.f;
      v[j] = u[j] * ((v[j] - mu) * rs);
    }
    s1 += sum8(u);
    s2 += sum8(v);
  }
  s1 = row_sum<kWideThreads>(s1, lds[0]);
  s2 = row_sum<kWideThreads>(s2, lds[1]);
  if (tid == 0) {
    sums[2 * row] = mean != nullptr ? s1 / (float)width : 0.f;
    sums[2 * row + 1] = s2 / (float)width;
  }
}
// ... and a workgroup for 256 groups of columns and every gridDim.y-th row.
constexpr int kColumnThreads = 256;
template <typename T, typename D>
__global__ __launch_bounds__(kColumnThreads) void norm_grad_columns_kernel(
    const D* dy, long long dy_stride, const T* x, long long row_stride, int n_rows, int width,
    const unsigned char* __restrict__ valid, Affine weight, const float* __restrict__ mean, const float* __restrict__ rstd,
    const float* __restrict__ sums, T* dx, long long dx_stride, float* __restrict__ dweight, float* __restrict__ dbias) {
  const int g = blockIdx.x * kColumnThreads + threadIdx.x;
  if (8 * (long long)g >= width) return;
  float w[8] = {}, dw[8] = {}, db[8] = {};
  load_group(weight, g, width, 1.f, w);
  for (long long row = blockIdx.y; row < n_rows; row += gridDim.y) {
    float v[8], u[8] = {};
    if (valid == nullptr || valid[row] != 0) {
      const float mu = mean != nullptr ? mean[row] : 0.f, rs = rstd[row], s1 = sums[2 * row], s2 = sums[2 * row + 1];
      load_group(x + row * row_stride, g, width, v);
      load_group(dy + row * dy_stride, g, width, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = (v[j] - mu) * rs;
        db[j] += u[j];
        dw[j] = __builtin_fmaf(u[j], v[j], dw[j]);
        u[j] = rs * (u[j] * w[j] - s1 - v[j] * s2);
      }
    }
    store_group(dx + row * dx_stride, g, width, u);
  }
  if (dweight != nullptr) store_group(dweight + (size_t)blockIdx.y * width, g, width, dw);
  if (dbias != nullptr) store_group(dbias + (size_t)blockIdx.y * width, g, width, db);
}

// Sums of the partials of every column, each in the order of the workgroups: 64 columns to a workgroup, whose wavefronts take
// every sixteenth partial.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void norm_grad_sum_kernel(const float* __restrict__ dweight_parts,
                                                                       const float* __restrict__ dbias_parts, int parts,
                                                                       int width, float* __restrict__ dweight,
                                                                       float* __restrict__ dbias) {
  __shared__ float lds[kSumWaves][64];
  const float* from = blockIdx.y == 0 ? dweight_parts : dbias_parts;
  float* to = blockIdx.y == 0 ? dweight : dbias;
  if (to == nullptr) return;                     // uniform
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long d = (long long)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (d < width)
    for (int k = wave; k < parts; k += kSumWaves) s += from[(size_t)k * width + d];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || d >= width) return;
#pragma unroll
  for (int k = 1; k < kSumWaves; ++k) s += lds[k][lane];
  to[d] = s;
}

constexpr int kHeldGroups = 2048;                // groups of the widest row that a workgroup of the gradient holds

template <typename T>
int norm_typed(ais_ctx* ctx, const T* x, int n_rows, int width, long long row_stride, const unsigned char* valid, Affine weight,
               Affine bias, float eps, int centered, T* y, long long y_stride, float* mean, float* rstd) {
  auto run = [&](auto kernel, int threads) {
    kernel<<<dim3((unsigned)n_rows), dim3(threads), 0, ctx->stream>>>(x, row_stride, width, valid, weight, bias, eps, centered, y,
                                                                      y_stride, mean, rstd);
    return hip_fail(ctx, hipGetLastError());
  };
  const int groups = (width - 1) / 8 + 1;
  if (groups <= 64) return run(norm_kernel<T, 64, 1>, 64);
  if (groups <= 256) return run(norm_kernel<T, 256, 1>, 256);
  if (groups <= 512) return run(norm_kernel<T, 256, 2>, 256);
  if (groups <= 1024) return run(norm_kernel<T, 256, 4>, 256);
  if (groups <= 4096) return run(norm_kernel<T, 1024, 4>, 1024);
  return run(norm_kernel<T, 1024, 0>, 1024);
}

template <typename T, typename D>
int norm_grad_typed(ais_ctx* ctx, const D* dy, long long dy_stride, const T* x, long long row_stride, int n_rows, int width,
                    const unsigned char* valid, Affine weight, const float* mean, const float* rstd, T* dx, long long dx_stride,
                    float* dweight, float* dbias) {
  const int parts = norm_grad_parts(n_rows, width, ctx->n_cus);
  float* dw = dweight != nullptr ? static_cast<float*>(ctx->ws) : nullptr;
  float* db = dbias != nullptr ? static_cast<float*>(ctx->ws) + (dweight != nullptr ? (size_t)parts * width : 0) : nullptr;
  const int groups = (width - 1) / 8 + 1;
  if (groups > kHeldGroups) {
    float* sums = static_cast<float*>(ctx->ws) + (size_t)parts * width * ((dweight != nullptr) + (dbias != nullptr));
    norm_grad_rows_kernel<T, D><<<dim3((unsigned)n_rows), dim3(kWideThreads), 0, ctx->stream>>>(dy, dy_stride, x, row_stride, width,
                                                                                             valid, weight, mean, rstd, sums);
    norm_grad_columns_kernel<T, D><<<dim3((unsigned)((groups - 1) / kColumnThreads + 1), (unsigned)parts), dim3(kColumnThreads), 0,
                                     ctx->stream>>>(dy, dy_stride, x, row_stride, n_rows, width, valid, weight, mean, rstd, sums, dx,
                                                    dx_stride, dw, db);
  } else {
    auto run = [&](auto kernel, int threads) {
      kernel<<<dim3((unsigned)parts), dim3(threads), 0, ctx->stream>>>(dy, dy_stride, x, row_stride, n_rows, width, valid, weight,
                                                                       mean, rstd, dx, dx_stride, dw, db);
    };
    if (groups <= 64) run(norm_grad_kernel<T, D, 64, 1>, 64);
    else if (groups <= 256) run(norm_grad_kernel<T, D, 256, 1>, 256);
    else if (groups <= 512) run(norm_grad_kernel<T, D, 256, 2>, 256);
    else if (groups <= 1024) run(norm_grad_kernel<T, D, 512, 2>, 512);
    else run(norm_grad_kernel<T, D, 1024, 2>, 1024);
  }
  if (dweight != nullptr || dbias != nullptr)
    norm_grad_sum_kernel<<<dim3((unsigned)((width - 1) / 64 + 1), 2), dim3(64 * kSumWaves), 0, ctx->stream>>>(dw, db, parts, width,
                                                                                                        dweight, dbias);
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace

// Workgroups that share the rows of the gradient, a row of partials each.
int norm_grad_parts(long long n_rows, long long width, int n_cus) {
  if ((width - 1) / 8 + 1 > kHeldGroups) {
    const long long tiles = ((width - 1) / 8 + 1 + kColumnThreads - 1) / kColumnThreads;
    return (int)std::min(n_rows, std::max(1LL, (8LL * n_cus + tiles - 1) / tiles));
  }
  return (int)std::min(n_rows, 2LL * n_cus);
}

size_t norm_grad_bytes(long long n_rows, long long width, int sums, int n_cus) {
  const size_t rows = (width - 1) / 8 + 1 > kHeldGroups ? 8 * (size_t)n_rows : 0;
  return 4 * (size_t)sums * (size_t)norm_grad_parts(n_rows, width, n_cus) * (size_t)width + rows;
}

int launch_norm_rows(ais_ctx* ctx, const void* x, ais_dtype dtype, long long n_rows, int width, long long row_stride,
                     const unsigned char* valid, const void* weight, const void* bias, ais_dtype param_dtype, float eps,
                     int centered, void* y, long long y_stride, float* mean, float* rstd) {
  if (n_rows == 0) return AIS_OK;
  ScopedTimer timer(ctx, AIS_K_NORM);
  const Affine w{weight, param_dtype == AIS_BF16}, b{bias, param_dtype == AIS_BF16};
  if (dtype == AIS_BF16)
    return norm_typed(ctx, static_cast<const bf16_t*>(x), (int)n_rows, width, row_stride, valid, w, b, eps, centered,
                      static_cast<bf16_t*>(y), y_stride, mean, rstd);
  return norm_typed(ctx, static_cast<const float*>(x), (int)n_rows, width, row_stride, valid, w, b, eps, centered,
                    static_cast<float*>(y), y_stride, mean, rstd);
}

int launch_norm_rows_grad(ais_ctx* ctx, const void* dy, ais_dtype dy_dtype, long long dy_stride, const void* x, ais_dtype dtype,
                          long long n_rows, int width, long long row_stride, const unsigned char* valid, const void* weight,
                          ais_dtype param_dtype, const float* mean, const float* rstd, void* dx, long long dx_stride,
                          float* dweight, float* dbias) {
  ScopedTimer timer(ctx, AIS_K_NORM_GRAD);
  const Affine w{weight, param_dtype == AIS_BF16};
  auto run = [&](const auto* g, auto* out) {
    typedef std::remove_pointer_t<decltype(out)> T;
    return norm_grad_typed(ctx, g, dy_stride, static_cast<const T*>(x), row_stride, (int)n_rows, width, valid, w, mean, rstd, out,
                           dx_stride, dweight, dbias);
  };
  auto typed = [&](auto* out) {
    return dy_dtype == AIS_BF16 ? run(static_cast<const bf16_t*>(dy), out) : run(static_cast<const float*>(dy), out);
  };
  return dtype == AIS_BF16 ? typed(static_cast<bf16_t*>(dx)) : typed(static_cast<float*>(dx));
}

}  // namespace ais
