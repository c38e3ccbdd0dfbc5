// Distillation from a teacher's top logits: the divergence of a row's policy from the teacher's distribution over the tokens
// it lists, and the gradient with respect to the row's logits.
//
//   q = softmax(teacher / T) over the listed tokens,  p = softmax(z / T) over the vocabulary,
//   kl = sum_j q_j (log q_j - log p[id_j]),  dz = weight / T (p - sum_j q_j 1[id_j])
//
// A workgroup owns a row.  Beside the soft-max over the vocabulary, which is all of the traffic, there is little: the listed
// tokens' logits are gathered, and their elements of the gradient are written again once the row is there.  A token that is
// listed twice counts with both entries: a small hash table finds the entries of one token, their q added as fixed-point
// numbers, whose sum does not depend on the order.
#include "ais_internal.h"
#include "device_utils.h"

namespace ais {
namespace {

using namespace dev;

typedef unsigned long long u64;

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kQBits = 62;             // q as a fixed-point number

// What a row's listed tokens need of LDS: dynamic, `slots` (a power of two >= 2 n_top) of the table and n_top entries.
struct Listed {
  u64* mass;                           // [slots] sum of q of the token in the slot
  int* token;                          // [slots] or -1
  float* z;                            // [n_top] logit
  int* slot;                           // [n_top] slot of an entry that writes its token's element, or -1
  static size_t bytes(int n_top, int slots) { return (size_t)slots * 12 + (size_t)n_top * 8; }
  __device__ __forceinline__ Listed(unsigned char* lds, int n_top, int slots) {
    mass = reinterpret_cast<u64*>(lds);
    token = reinterpret_cast<int*>(mass + slots);
    z = reinterpret_cast<float*>(token + slots);
    slot = reinterpret_cast<int*>(z + n_top);
  }
};

struct RowShared {
  float top[kRowWaves];
  double sum[kRowWaves];
  MaxSum soft[kRowWaves];
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float row_max(float v, RowShared& sh) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.top[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) v = fmaxf(v, sh.top[w]);
  return v;
}
__device__ __forceinline__ double row_sum(double v, RowShared& sh) {
  v = wave_sum64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.sum[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh.sum[0];
#pragma unroll
  for (int w = 1; w < kRowWaves; ++w) v += sh.sum[w];
  return v;
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void distill_kernel(
    const T* logits, long long row_stride, int vocab, const int* __restrict__ ids, const float* __restrict__ teacher, int n_top,
    int slots, const unsigned char* __restrict__ valid, const float* __restrict__ weight, float inv_rows, float inv_temperature,
    float* __restrict__ kl_out, T* dlogits, long long dlogits_stride, int* __restrict__ status) {
  constexpr int N = Vec<T>::N;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ RowShared sh;
  const Listed listed(lds, n_top, slots);
  const long long row = blockIdx.x;
  const int tid = threadIdx.x;
  const T* zr = logits + row * row_stride;
  T* dr = dlogits == nullptr ? nullptr : dlogits + row * dlogits_stride;
  const int* id_row = ids + row * n_top;
  const float* t_row = teacher + row * n_top;
  const float c = inv_temperature * kLog2e;

  // ---- the teacher's distribution ----
  float top = -__builtin_inff();
  if (valid == nullptr || valid[row] != 0) {
    for (int j = tid; j < n_top; j += kRowThreads) {
      const int id = id_row[j];
      if (id >= 0 && id < vocab) top = fmaxf(top, t_row[j]);
      else if (id != -1) atomicOr(status, AIS_STATUS_BAD_TOKEN);
    }
    top = row_max(top, sh);
  }
  if (top == -__builtin_inff()) {                      // nothing to learn from: no loss, no gradient
    if (tid == 0) kl_out[row] = 0.f;
    if (dr != nullptr)
      for (int v = tid; v < vocab; v += kRowThreads) Vec<T>::store1(dr + v, 0.f);
    return;
  }
  for (int s = tid; s < slots; s += kRowThreads) {
    listed.token[s] = -1;
    listed.mass[s] = 0;
  }
  double own = 0.0;
  for (int j = tid; j < n_top; j += kRowThreads) {
    const int id = id_row[j];
    if (id >= 0 && id < vocab) own += (double)exp2_fast((t_row[j] - top) * c);
  }
  const double q_sum = row_sum(own, sh);
  const float q_scale = (float)(1.0 / q_sum);
  const bool q_fine = q_sum < 1e30;                    // not where the teacher has a NaN or an infinity

  // ---- the policy's soft-max ----
  // where the gradient lies has no say in the order of the sums
  const int nvec = (reinterpret_cast<uintptr_t>(zr) & 15) == 0 ? vocab / N : 0;
  const bool dr_aligned = (reinterpret_cast<uintptr_t>(dr) & 15) == 0;
  const u32x4* zv = reinterpret_cast<const u32x4*>(zr);
  MaxSum st{kNegHuge, 0.f};
  for (int i = tid; i < nvec; i += kRowThreads) {
    float x[N];
    Vec<T>::unpack(zv[i], x);
    accumulate<N>(x, c, st);
  }
  for (int v = nvec * N + tid; v < vocab; v += kRowThreads) {
    const float x = Vec<T>::load1(zr + v);
    accumulate<1>(&x, c, st);
  }
  st = wave_merge(st);
  if ((tid & 63) == 0) sh.soft[tid >> 6] = st;
  __syncthreads();
  st = sh.soft[0];
#pragma unroll
  for (int w = 1; w < kRowWaves; ++w) st = merge(st, sh.soft[w]);

  // ---- the divergence: log q - log p of every entry, with p = 2^(z c - st.m) / st.s ----
  const double log_ratio = log(q_sum) - log((double)st.s);
  double kl = 0.0;
  for (int j = tid; j < n_top; j += kRowThreads) {
    const int id = id_row[j];
    int slot = -1;
    if (id >= 0 && id < vocab) {
      const float z = Vec<T>::load1(zr + id), t = (t_row[j] - top) * c, q = exp2_fast(t) * q_scale;
      listed.z[j] = z;
      if (!(q <= 0.f)) kl += (double)q * (((double)t - (double)__builtin_fmaf(z, c, -st.m)) * 0.6931471805599453 - log_ratio);
      int s = (int)(((uint32_t)id * 2654435761u) >> 16) & (slots - 1);
      while (true) {
        const int held = atomicCAS(&listed.token[s], -1, id);
        if (held == -1) slot = s;
        if (held == -1 || held == id) break;
        s = (s + 1) & (slots - 1);
      }
      atomicAdd(&listed.mass[s], (u64)ldexp((double)(q_fine ? q : 0.f), kQBits));
    }
    listed.slot[j] = slot;
  }
  kl = row_sum(kl, sh);
  if (tid == 0) kl_out[row] = (float)kl;
  if (dr == nullptr) return;

  // ---- the gradient ----
  const float g = (weight == nullptr ? inv_rows : weight[row]) * inv_temperature;
  const float g_p = g / st.s;
  for (int i = tid; i < nvec; i += kRowThreads) {
    float x[N];
    Vec<T>::unpack(zv[i], x);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = exp2_fast(__builtin_fmaf(x[j], c, -st.m)) * g_p;
    if (dr_aligned) {
      reinterpret_cast<u32x4*>(dr)[i] = Vec<T>::pack(x);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) Vec<T>::store1(dr + i * N + j, x[j]);
    }
  }
  for (int v = nvec * N + tid; v < vocab; v += kRowThreads)
    Vec<T>::store1(dr + v, exp2_fast(__builtin_fmaf(Vec<T>::load1(zr + v), c, -st.m)) * g_p);
  // the listed tokens' elements, once every wavefront's stores have completed
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int j = tid; j < n_top; j += kRowThreads) {
    const int s = listed.slot[j];
    if (s < 0) continue;
    const float q = q_fine ? (float)ldexp((double)listed.mass[s], -kQBits) : __builtin_nanf("");
    const float p = exp2_fast(__builtin_fmaf(listed.z[j], c, -st.m)) / st.s;
    Vec<T>::store1(dr + listed.token[s], g * (p - q));
  }
}

constexpr int kLossThreads = 1024;

// loss = sum_n weight[n] kl[n]: fp64, in a fixed order.
__global__ __launch_bounds__(kLossThreads) void distill_loss_kernel(const float* __restrict__ kl, const float* __restrict__ weight,
                                                                    const unsigned char* __restrict__ valid, long long n_rows,
                                                                    float inv_rows, float* __restrict__ loss) {
  __shared__ double sum[kLossThreads / 64];
  double own = 0.0;
  for (long long n = threadIdx.x; n < n_rows; n += kLossThreads)
    if (valid == nullptr || valid[n] != 0) own += (double)kl[n] * (double)(weight == nullptr ? inv_rows : weight[n]);
  own = wave_sum64(own);
  if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = own;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kLossThreads / 64; ++w) own += sum[w];
  *loss = (float)own;
}

}  // namespace

int launch_distill_topk(ais_ctx* ctx, const void* logits, ais_dtype dtype, long long n_rows, int vocab, long long row_stride,
                        const int* ids, const float* teacher, int n_top, const unsigned char* valid, const float* weight,
                        float inv_temperature, float* kl_out, float* loss_out, void* dlogits, long long dlogits_stride) {
  ScopedTimer timer(ctx, AIS_K_DISTILL);
  const float inv_rows = n_rows > 0 ? (float)(1.0 / (double)n_rows) : 0.f;
  if (n_rows > 0) {
    int slots = 2;
    while (slots < 2 * n_top) slots *= 2;
    auto run = [&](auto type) {
      typedef decltype(type) T;
      distill_kernel<T><<<dim3((unsigned)n_rows), dim3(kRowThreads), Listed::bytes(n_top, slots), ctx->stream>>>(
          static_cast<const T*>(logits), row_stride, vocab, ids, teacher, n_top, slots, valid, weight, inv_rows,
          inv_temperature, kl_out, static_cast<T*>(dlogits), dlogits_stride, ctx->status_dev);
    };
    if (dtype == AIS_BF16) run(bf16_t{});
    else run(float{});
    const int rc = hip_fail(ctx, hipGetLastError());
    if (rc != AIS_OK) return rc;
  }
  distill_loss_kernel<<<dim3(1), dim3(kLossThreads), 0, ctx->stream>>>(kl_out, weight, valid, n_rows, inv_rows, loss_out);
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
