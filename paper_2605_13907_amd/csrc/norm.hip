// Rows normalised in front of the read-out, and their gradient.
//
//   norm:       y = (x - mean) rstd w + b, mean and variance over the row (or mean 0: root-mean-square norm)
//   norm_grad:  n = (x - mean) rstd, u = dy w:  dx = rstd (u - <u> - n <u n>), dw = sum_r dy n, db = sum_r dy
//
// Bound by memory: a row is read once into registers, its statistics are formed there (the variance from deviations, in a second
// pass over the registers, so that nothing cancels), and it is written once.  A lane holds 16-byte vectors, consecutive lanes consecutive
// ones (32 bytes of fp32 to a lane: 5.1 instead of 6.0 TB/s), all of a row's loads go out together, and a row's successor is on its way
// while it is summed and written.  41,643 rows of 4,096 elements: bf16 116 us, 5.9 TB/s; the gradient from an fp32 one 227 us and 5 for
// the sums over the workgroups, 5.9 TB/s (with loads one after the other and no row ahead 133, 346 and 15).
#include <algorithm>
#include <type_traits>

#include "ais_internal.h"
#include "eights.h"

namespace ais {
namespace {

using namespace dev;

constexpr int kWideThreads = 1024;
// Workgroups of a launch, which may have no more than 2^32 - 1 threads; where there are more rows (columns, of the sums), each goes on
// behind the others.  Of more than two million rows a workgroup that holds them has more than two.
constexpr int kMostBlocks = 1 << 20, kMostWideBlocks = 1 << 16;

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
  // N (8 or 4) elements from `at` on; `some`: whether there are any.
  template <int N>
  __device__ __forceinline__ void load_vector(int at, bool some, float otherwise, float* x) const {
    if (p == nullptr || !some) {                 // uniform
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = otherwise;
    } else if constexpr (N == 8) {
      load(at, otherwise, x);
    } else if (bf16) {
      const Unaligned<bf16_t>::two q = *reinterpret_cast<const Unaligned<bf16_t>::two*>(static_cast<const bf16_t*>(p) + at);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        x[2 * k] = __uint_as_float(q[k] << 16);
        x[2 * k + 1] = __uint_as_float(q[k] & 0xffff0000u);
      }
    } else {
      Vec<float>::unpack(*reinterpret_cast<const Unaligned<float>::four*>(static_cast<const float*>(p) + at), x);
    }
  }
  __device__ __forceinline__ float load1(int at, float otherwise) const {
    if (p == nullptr) return otherwise;
    return bf16 ? Vec<bf16_t>::load1(static_cast<const bf16_t*>(p) + at) : static_cast<const float*>(p)[at];
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

template <int N>
__device__ __forceinline__ float sum_of(const float* x) {
  const float a = (x[0] + x[1]) + (x[2] + x[3]);
  if constexpr (N == 4) return a;
  else return a + ((x[4] + x[5]) + (x[6] + x[7]));
}

// How rows are cut into vectors of N elements, which begin at whole words: of bf16 rows that begin in the middle of one the first element
// is left out of them, like those after the last vector.  (The gradient of 28,066 bf16 rows of 2,237 elements, one after the other: 135 us,
// 164 with vectors from their first element on; 20,000 of 4,097: 114, 137.)  Any cut is sound for any row, whatever it costs; a workgroup
// has one for all of its rows.
struct Cut {
  int head, vectors, left;                       // left: elements outside the vectors, those of the head first
  template <typename T, int N>
  __device__ __forceinline__ static Cut of(const T* row, int width) {
    const int head = sizeof(T) == 2 ? (int)(reinterpret_cast<uintptr_t>(row) >> 1 & 1) : 0;
    const int vectors = (width - head) / N;
    return {head, vectors, width - N * vectors};
  }
  // Element that the thread-th of the elements outside is.
  template <int N>
  __device__ __forceinline__ int rest(int thread) const { return thread < head ? thread : N * vectors + thread; }
};

// A row of up to NV vectors of N elements to a thread of the THREADS that share it: those past the row's last repeat it and are left
// out of the sums.  The elements outside are one each of the first threads.  WHOLE: every thread has all of its vectors.
template <typename T, int N, int THREADS, int NV, bool WHOLE>
struct HeldRow {
  typedef Pack<T, N> P;
  typename P::Raw q[NV];
  float rest;
  static __device__ __forceinline__ int thread() { return THREADS == 64 ? threadIdx.x & 63 : threadIdx.x; }
  static __device__ __forceinline__ bool has(int k, int vectors) { return WHOLE || thread() + k * THREADS < vectors; }
  // First element of vector k.
  static __device__ __forceinline__ int element(int k, const Cut& cut) {
    const int g = thread() + k * THREADS;
    return cut.head + N * (WHOLE ? g : max(min(g, cut.vectors - 1), 0));
  }
  __device__ __forceinline__ void load(const T* row, const Cut& cut) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      q[k] = WHOLE || cut.vectors > 0
                 ? (typename P::Raw)__builtin_nontemporal_load(reinterpret_cast<const typename P::Any*>(row + element(k, cut)))
                 : P::zero();
    rest = thread() < cut.left ? Vec<T>::load1(row + cut.rest<N>(thread())) : 0.f;
  }
  // Vector k, 0 where there is none.
  __device__ __forceinline__ void get(int k, int vectors, float* x) const {
    P::unpack(q[k], x);
    if (!has(k, vectors)) {
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = 0.f;
    }
  }
  static __device__ __forceinline__ void store(T* row, int k, const Cut& cut, const float* x) {
    __builtin_nontemporal_store((typename P::Any)P::pack(x),
                                reinterpret_cast<typename P::Any*>(row + cut.head + N * (thread() + k * THREADS)));
  }
};

// Sums of a row's parts over the THREADS threads that share it.  The rows that are summed take turns with two places in LDS, so that one
// barrier a sum is enough: whoever writes a place again has passed the barrier of the row summed in between, which nobody reaches before
// having read this one.  (Masked rows have no barrier: they take no turn.)
template <int THREADS, int SUMS>
struct RowSums {
  float part[2][SUMS][THREADS == 64 ? 1 : THREADS / 64];
  __device__ __forceinline__ void add(int turn, int first, int count, float* v) {
#pragma unroll
    for (int i = 0; i < count; ++i) v[i] = wave_sum(v[i]);
    if constexpr (THREADS > 64) {
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < count; ++i) part[turn][first + i][threadIdx.x >> 6] = v[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < count; ++i) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) s += part[turn][first + i][w];
        v[i] = s;
      }
    }
  }
};

// Rows that a workgroup holds, every gridDim.x-th to each; the next one is on its way while the present one is summed and written.
template <typename T, int THREADS, int NV, bool WHOLE>
__global__ __launch_bounds__(THREADS) void norm_kernel(const T* x, long long row_stride, int n_rows, int width,
                                                       const unsigned char* __restrict__ valid, Affine weight, Affine bias,
                                                       float eps, int centered, T* y, long long y_stride,
                                                       float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  constexpr int N = Vec<T>::N;
  typedef HeldRow<T, N, THREADS, NV, WHOLE> Row;
  __shared__ RowSums<THREADS, 2> sums;
  const int tid = threadIdx.x;
  const Cut cut = Cut::of<T, N>(y + blockIdx.x * y_stride, width);
  const int vectors = cut.vectors, left = cut.left;
  const float n = (float)width;
  float w[NV][N], b[NV][N], w_rest = 1.f, b_rest = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    weight.load_vector<N>(Row::element(k, cut), vectors > 0, 1.f, w[k]);
    bias.load_vector<N>(Row::element(k, cut), vectors > 0, 0.f, b[k]);
  }
  if (tid < left) {
    w_rest = weight.load1(cut.rest<N>(tid), 1.f);
    b_rest = bias.load1(cut.rest<N>(tid), 0.f);
  }
  auto live = [&](long long row) { return valid == nullptr || valid[row] != 0; };
  Row now, next;
  bool here = live(blockIdx.x);
  if (here) now.load(x + blockIdx.x * row_stride, cut);
  int turn = 0;
  for (long long row = blockIdx.x; row < n_rows; row += gridDim.x) {
    const long long after = row + gridDim.x;
    const bool more = after < n_rows && live(after);
    if (more) next.load(x + after * row_stride, cut);
    T* yr = y + row * y_stride;
    float mean = 0.f, rstd = 0.f;
    if (here) {                                  // uniform
      if (centered) {
        float s = now.rest;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          float v[N];
          now.get(k, vectors, v);
          s += sum_of<N>(v);
        }
        sums.add(turn, 0, 1, &s);
        mean = s / n;
      }
      float q = tid < left ? (now.rest - mean) * (now.rest - mean) : 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float v[N];
        now.get(k, vectors, v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          v[j] -= now.has(k, vectors) ? mean : 0.f;
          v[j] *= v[j];
        }
        q += sum_of<N>(v);
      }
      sums.add(turn, 1, 1, &q);
      rstd = 1.f / sqrtf(q / n + eps);
      turn ^= 1;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (!now.has(k, vectors)) break;
      float v[N] = {};
      if (here) {
        Vec<T>::unpack(now.q[k], v);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = __builtin_fmaf((v[j] - mean) * rstd, w[k][j], b[k][j]);
      }
      Row::store(yr, k, cut, v);
    }
    if (tid < left) Vec<T>::store1(yr + cut.rest<N>(tid), here ? __builtin_fmaf((now.rest - mean) * rstd, w_rest, b_rest) : 0.f);
    if (tid == 0) {
      if (centered) mean_out[row] = mean;
      rstd_out[row] = rstd;
    }
    now = next;
    here = more;
  }
}

// Rows of any width, read three times.
template <typename T>
__global__ __launch_bounds__(kWideThreads) void norm_wide_kernel(const T* x, long long row_stride, int n_rows, int width,
                                                                 const unsigned char* __restrict__ valid, Affine weight,
                                                                 Affine bias, float eps, int centered, T* y, long long y_stride,
                                                                 float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  __shared__ float lds[kWideThreads / 64];
  const int tid = threadIdx.x, groups = (width - 1) / 8 + 1;
  for (long long row = blockIdx.x; row < n_rows; row += gridDim.x) {
    const T* xr = x + row * row_stride;
    T* yr = y + row * y_stride;
    const bool here = valid == nullptr || valid[row] != 0;
    float mean = 0.f, rstd = 0.f;
    if (here) {
      const float n = (float)width;
      if (centered) {
        float s = 0.f;
        for (int g = tid; g < groups; g += kWideThreads) {
          float v[8];
          load_group(xr, g, width, v);
          s += sum8(v);
        }
        mean = row_sum<kWideThreads>(s, lds) / n;
      }
      float q = 0.f;
      for (int g = tid; g < groups; g += kWideThreads) {
        float v[8];
        load_group(xr, g, width, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = 8 * (long long)g + j < width ? v[j] - mean : 0.f;
          v[j] = d * d;
        }
        q += sum8(v);
      }
      rstd = 1.f / sqrtf(row_sum<kWideThreads>(q, lds) / n + eps);
    }
    for (int g = tid; g < groups; g += kWideThreads) {
      float v[8] = {}, w[8] = {}, b[8] = {};
      if (here) {
        load_group(xr, g, width, v);
        load_group(weight, g, width, 1.f, w);
        load_group(bias, g, width, 0.f, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf((v[j] - mean) * rstd, w[j], b[j]);
      }
      store_group(yr, g, width, v);
    }
    if (tid == 0) {
      if (centered) mean_out[row] = mean;
      rstd_out[row] = rstd;
    }
  }
}

// The gradient.  TEAMS teams of THREADS threads of a workgroup take a row each, with the next one on its way, and keep the weight's and
// the bias's sums of their own columns in registers; a workgroup's leave as one row of partials, which norm_grad_sum_kernel adds up in
// their order.
template <typename T, typename D, int THREADS, int TEAMS, int NV, int WHOLE>
__global__ __launch_bounds__(THREADS * TEAMS) void norm_grad_kernel(
    const D* dy, long long dy_stride, const T* x, long long row_stride, int n_rows, int width,
    const unsigned char* __restrict__ valid, Affine weight, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
    long long dx_stride, float* __restrict__ dweight, float* __restrict__ dbias) {
  static_assert(TEAMS == 1 || THREADS == 64, "a barrier inside a row is the whole workgroup's");
  constexpr int N = sizeof(T) == 2 && sizeof(D) == 2 ? 8 : 4;
  typedef HeldRow<T, N, THREADS, NV, WHOLE != 0> Row;
  typedef HeldRow<D, N, THREADS, NV, WHOLE != 0> Grad;
  __shared__ RowSums<THREADS, 2> sums;
  const int thread = Row::thread(), team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The teams' sums meet column by column, with one cut for all of them: where rows may begin differently, theirs are a multiple of the
  // workgroups' number apart, which is even.
  constexpr bool kAlike = sizeof(T) == 4 || WHOLE == 2;
  long long row = kAlike ? (long long)blockIdx.x * TEAMS + team : blockIdx.x + (long long)gridDim.x * team;
  const Cut cut = WHOLE == 2 ? Cut{0, THREADS * NV, 0} : Cut::of<T, N>(dx + blockIdx.x * dx_stride, width);
  const int vectors = cut.vectors, left = cut.left;
  const float n = (float)width;
  float w[NV][N], w_rest = 1.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) weight.load_vector<N>(Row::element(k, cut), vectors > 0, 1.f, w[k]);
  if (thread < left) w_rest = weight.load1(cut.rest<N>(thread), 1.f);
  float dw[NV][N] = {}, db[NV][N] = {}, dw_rest = 0.f, db_rest = 0.f;
  struct Held {
    Row x;
    Grad dy;
    float mu, rs;
    bool here;
  } now, next;
  auto load = [&](Held& h, long long row) {
    h.here = row < n_rows && (valid == nullptr || valid[row] != 0);
    if (!h.here) return;
    h.x.load(x + row * row_stride, cut);
    h.dy.load(dy + row * dy_stride, cut);
    h.mu = mean != nullptr ? mean[row] : 0.f;
    h.rs = rstd[row];
  };
  const long long stride = (long long)gridDim.x * TEAMS;
  load(now, row);
  int turn = 0;
  for (; row < n_rows; row += stride) {
    load(next, row + stride);
    T* dr = dx + row * dx_stride;
    float v[NV][N], u[NV][N], v_rest = 0.f, u_rest = 0.f, s[2] = {0.f, 0.f};
    const float rs = now.here ? now.rs : 0.f;
    if (now.here) {                              // uniform
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        now.x.get(k, vectors, v[k]);
        now.dy.get(k, vectors, u[k]);
        float p[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          v[k][j] = (v[k][j] - now.mu) * rs;
          db[k][j] += u[k][j];
          dw[k][j] = __builtin_fmaf(u[k][j], v[k][j], dw[k][j]);
          u[k][j] *= w[k][j];
          p[j] = u[k][j] * v[k][j];
        }
        s[0] += sum_of<N>(u[k]);
        s[1] += sum_of<N>(p);
      }
      if (thread < left) {
        v_rest = (now.x.rest - now.mu) * rs;
        u_rest = now.dy.rest;
        db_rest += u_rest;
        dw_rest = __builtin_fmaf(u_rest, v_rest, dw_rest);
        u_rest *= w_rest;
        s[0] += u_rest;
        s[1] += u_rest * v_rest;
      }
      sums.add(turn, 0, 2, s);
      turn ^= 1;
      s[0] = mean != nullptr ? s[0] / n : 0.f;
      s[1] /= n;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (!Row::has(k, vectors)) break;
#pragma unroll
      for (int j = 0; j < N; ++j) u[k][j] = now.here ? rs * (u[k][j] - s[0] - v[k][j] * s[1]) : 0.f;
      Row::store(dr, k, cut, u[k]);
    }
    if (thread < left) Vec<T>::store1(dr + cut.rest<N>(thread), now.here ? rs * (u_rest - s[0] - v_rest * s[1]) : 0.f);
    now = next;
  }
  // the teams' sums, added up in their order
  __shared__ float other[TEAMS == 1 ? 1 : TEAMS - 1][64];
  auto all = [&](float a) {
    if constexpr (TEAMS > 1) {
      __syncthreads();
      if (team > 0) other[team - 1][thread] = a;
      __syncthreads();
#pragma unroll
      for (int t = 0; t < TEAMS - 1; ++t) a += other[t][thread];
    }
    return a;
  };
  auto leave = [&](float (&sum)[NV][N], float rest, float* to) {
    if (to == nullptr) return;                   // uniform
    to += (size_t)blockIdx.x * width;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < N; ++j) sum[k][j] = all(sum[k][j]);
      if (team != 0 || !Row::has(k, vectors)) continue;
      float* at = to + cut.head + N * (thread + k * THREADS);
#pragma unroll
      for (int j = 0; j < N; j += 4) *reinterpret_cast<Unaligned<float>::four*>(at + j) = Vec<float>::pack(sum[k] + j);
    }
    rest = all(rest);
    if (team == 0 && thread < left) to[cut.rest<N>(thread)] = rest;
  };
  leave(dw, dw_rest, dweight);
  leave(db, db_rest, dbias);
}

// Rows too wide for that, in two kernels: <u> and <u n> of every row ...
template <typename T, typename D>
__global__ __launch_bounds__(kWideThreads) void norm_grad_rows_kernel(const D* __restrict__ dy, long long dy_stride,
                                                                      const T* __restrict__ x, long long row_stride, int n_rows, int width,
                                                                      const unsigned char* __restrict__ valid, Affine weight,
                                                                      const float* __restrict__ mean,
                                                                      const float* __restrict__ rstd, float* __restrict__ sums) {
  __shared__ float lds[2][kWideThreads / 64];
  const int tid = threadIdx.x, groups = (width - 1) / 8 + 1;
  for (long long row = blockIdx.x; row < n_rows; row += gridDim.x) {
    if (valid != nullptr && valid[row] == 0) continue;             // uniform
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

// Sums of the partials of every column, each in the order of the workgroups: 64 columns to a workgroup, whose wavefronts take every
// sixteenth partial, eight of them on their way at once.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void norm_grad_sum_kernel(const float* __restrict__ dweight_parts,
                                                                       const float* __restrict__ dbias_parts, int parts,
                                                                       int width, float* __restrict__ dweight,
                                                                       float* __restrict__ dbias) {
  __shared__ float lds[kSumWaves][64];
  const bool first = blockIdx.y == 0 && dweight != nullptr;
  const float* from = first ? dweight_parts : dbias_parts;
  float* to = first ? dweight : dbias;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long at = 64LL * blockIdx.x; at < width; at += 64LL * gridDim.x) {
    const long long d = min(at + lane, (long long)width - 1);
    float s = 0.f;
    for (int k = wave; k < parts; k += 8 * kSumWaves) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = from[(size_t)min(k + i * kSumWaves, parts - 1) * width + d];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += k + i * kSumWaves < parts ? v[i] : 0.f;
    }
    if (at != 64LL * blockIdx.x) __syncthreads();            // the first wavefront has read the columns before
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int k = 1; k < kSumWaves; ++k) s += lds[k][lane];
      if (at + lane < width) to[d] = s;
    }
  }
}

// Whether bf16 rows all begin at whole words.
bool at_words(const void* rows, long long stride) { return ((reinterpret_cast<uintptr_t>(rows) / 2 | (uintptr_t)stride) & 1) == 0; }

// 1: every row is `most` vectors of n elements, however it is cut; 2: and has no element outside them; 0: neither.
template <typename T>
int whole_rows(const T* rows, long long stride, int width, int n, int most) {
  const bool odd = sizeof(T) == 2 && !at_words(rows, stride);
  if (width / n != most || (odd && (width - 1) / n != most)) return 0;
  return !odd && width % n == 0 ? 2 : 1;
}

template <typename T>
int norm_typed(ais_ctx* ctx, const T* x, int n_rows, int width, long long row_stride, const unsigned char* valid, Affine weight,
               Affine bias, float eps, int centered, T* y, long long y_stride, float* mean, float* rstd) {
  const int vectors = width / Vec<T>::N;
  // Two rows to a workgroup, so that the second is read while the first is written and the weight is loaded for both; one each where there
  // are few.  41,643 rows of 4,096 bf16 elements, us with one, two, four rows each, and with as many workgroups as there is room for: 146,
  // 116, 118 to 122, 124.
  // (An even number of workgroups: rows of one begin alike.)
  const unsigned grid = (unsigned)(n_rows <= 8 * ctx->n_cus ? n_rows : std::min(n_rows / 4 * 2 + 2, kMostBlocks));
  auto held = [&](auto threads, auto most) {
    constexpr int kThreads = decltype(threads)::value, kMost = decltype(most)::value;
    auto kernel = whole_rows(y, y_stride, width, Vec<T>::N, kThreads * kMost) ? norm_kernel<T, kThreads, kMost, true>
                                                                              : norm_kernel<T, kThreads, kMost, false>;
    kernel<<<dim3(grid), dim3(kThreads), 0, ctx->stream>>>(x, row_stride, n_rows, width, valid, weight, bias, eps, centered, y,
                                                           y_stride, mean, rstd);
    return hip_fail(ctx, hipGetLastError());
  };
  // Threads and vectors of each that hold a row with few of them idle; us with these and with half or twice as many threads, rows of 1.4 GB in all:
  // bf16, 1,024 elements 33, 36; 2,048 61, 61, 77; 4,096 116, 118, 131; 5,120 (as 192 x 4, 320 x 2, 256 x 4) 139, 142, 155; 8,192 120, 133, 157;
  // 2,240 (28,066 rows of them, as 64 x 5, 128 x 3, 256 x 2) 61, 66, 81;
  // fp32, 1,024 57, 58; 4,096 (512 x 2, 256 x 4, 128 x 8) 222, 227, 226; 5,120 222, 230; 8,192 (512 x 4, 256 x 8, 1,024 x 2) 224, 232, 268.
#define AIS_NORM_CASE(THREADS, NV)                                                                                     \
  if (vectors <= THREADS * NV) return held(std::integral_constant<int, THREADS>{}, std::integral_constant<int, NV>{});
  AIS_NORM_CASE(64, 1)
  AIS_NORM_CASE(64, 2)
  AIS_NORM_CASE(64, 3)
  AIS_NORM_CASE(64, 4)
  AIS_NORM_CASE(64, 5)
  AIS_NORM_CASE(128, 3)
  AIS_NORM_CASE(256, 2)
  AIS_NORM_CASE(192, 4)
  AIS_NORM_CASE(256, 4)
  AIS_NORM_CASE(320, 4)
  AIS_NORM_CASE(384, 4)
  AIS_NORM_CASE(512, 4)
  if constexpr (sizeof(T) == 4) {                // of bf16, eight vectors, weight and bias are more than a thread has registers for
    AIS_NORM_CASE(384, 8)
    AIS_NORM_CASE(512, 8)
  }
#undef AIS_NORM_CASE
  norm_wide_kernel<T><<<dim3((unsigned)std::min(n_rows, kMostWideBlocks)), dim3(kWideThreads), 0, ctx->stream>>>(
      x, row_stride, n_rows, width, valid, weight, bias, eps, centered, y, y_stride, mean, rstd);
  return hip_fail(ctx, hipGetLastError());
}

template <typename T, typename D>
int norm_grad_typed(ais_ctx* ctx, const D* dy, long long dy_stride, const T* x, long long row_stride, int n_rows, int width,
                    const unsigned char* valid, Affine weight, const float* mean, const float* rstd, T* dx, long long dx_stride,
                    float* dweight, float* dbias) {
  const NormGradPlan plan = norm_grad_plan(n_rows, width, sizeof(T) + sizeof(D), dx, dx_stride, ctx->n_cus);
  const size_t all = (size_t)plan.parts * width;
  float* at = static_cast<float*>(ctx->ws);
  float *dw = nullptr, *db = nullptr;
  if (dweight != nullptr) dw = at, at += all;
  if (dbias != nullptr) db = at, at += all;
  if (plan.teams == 0) {
    norm_grad_rows_kernel<T, D><<<dim3((unsigned)std::min(n_rows, kMostWideBlocks)), dim3(kWideThreads), 0, ctx->stream>>>(
        dy, dy_stride, x, row_stride, n_rows, width, valid, weight, mean, rstd, at);
    norm_grad_columns_kernel<T, D><<<dim3((unsigned)((width - 1) / (8 * kColumnThreads) + 1), (unsigned)plan.parts), dim3(kColumnThreads),
                                     0, ctx->stream>>>(dy, dy_stride, x, row_stride, n_rows, width, valid, weight, mean, rstd, at, dx,
                                                       dx_stride, dw, db);
  } else {
    auto held = [&](auto threads, auto teams, auto most) {
      constexpr int kThreads = decltype(threads)::value, kTeams = decltype(teams)::value, kMost = decltype(most)::value;
      constexpr int kN = sizeof(T) == 2 && sizeof(D) == 2 ? 8 : 4;
      const int whole = whole_rows(dx, dx_stride, width, kN, kThreads * kMost);
      auto kernel = whole == 2   ? norm_grad_kernel<T, D, kThreads, kTeams, kMost, 2>
                    : whole == 1 ? norm_grad_kernel<T, D, kThreads, kTeams, kMost, 1>
                                 : norm_grad_kernel<T, D, kThreads, kTeams, kMost, 0>;
      kernel<<<dim3((unsigned)plan.parts), dim3(kThreads * kTeams), 0, ctx->stream>>>(dy, dy_stride, x, row_stride, n_rows, width,
                                                                                      valid, weight, mean, rstd, dx, dx_stride, dw, db);
    };
#define AIS_GRAD_CASE(THREADS, TEAMS, NV)                                                                            \
  if (plan.threads == THREADS && plan.vectors == NV)                                                                 \
    held(std::integral_constant<int, THREADS>{}, std::integral_constant<int, TEAMS>{}, std::integral_constant<int, NV>{});
    AIS_GRAD_CASE(64, 4, 1)
    AIS_GRAD_CASE(64, 4, 2)
    AIS_GRAD_CASE(64, 4, 4)
    AIS_GRAD_CASE(256, 1, 2)
    AIS_GRAD_CASE(256, 1, 3)
    if constexpr (sizeof(T) == 2 && sizeof(D) == 2) {
      AIS_GRAD_CASE(64, 4, 3)
      AIS_GRAD_CASE(128, 1, 2)
      AIS_GRAD_CASE(128, 1, 3)
      AIS_GRAD_CASE(256, 1, 4)
      AIS_GRAD_CASE(1024, 1, 1)
    } else {
      AIS_GRAD_CASE(64, 4, 5)
      AIS_GRAD_CASE(512, 1, 2)
      AIS_GRAD_CASE(1024, 1, 2)
    }
#undef AIS_GRAD_CASE
  }
  const unsigned sums = (dweight != nullptr) + (dbias != nullptr);
  if (sums > 0)
    norm_grad_sum_kernel<<<dim3((unsigned)std::min((width - 1) / 64 + 1, kMostBlocks), sums), dim3(64 * kSumWaves), 0, ctx->stream>>>(
        dw, db, plan.parts, width, dweight, dbias);
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace

// Threads and vectors that hold a row with few of them idle, and as many workgroups as a compute unit has room for, each with six rows at
// least where there is more than one of them to a unit: their partial sums have to be written and read.  us, in turns with other choices:
//   bf16 with an fp32 gradient: 41,643 rows of 4,096 elements, two, three, four workgroups 230, 254, 236 (256 threads with four vectors each
//     232, 246; 1,024 with one 249); 28,066 of 2,240 91, with 512 threads and two vectors 112; 41,643 of 1,024, a wavefront to a row, which has
//     no barrier in it, 64, 256 threads 68;
//   fp32: 41,643 of 4,096 334, 341 with four workgroups; 5,001 of 1,100 22.0, 256 threads 24.1;
//   bf16: 28,066 of 2,240 80, with 256 threads and two vectors 103; 30,000 of 3,500 139, two workgroups 156; 25,000 of 5,000 138, with 256
//     threads and four vectors 236; 72,000 of 1,600 132, a wavefront with four vectors 176; 1,000 of 4,096 15.1, two workgroups 19.4.
//   Four vectors of eight a thread leave registers for two workgroups to a unit only where no element lies outside them: there (60,000 of
//     2,048 128, 14,000 of 8,192 126) they are ahead of 128 threads with two (138) and 1,024 with one (136), elsewhere (the same rows,
//     beginning in the middle of a word) behind them: 203 and 200, 147 and 157 with those.
NormGradPlan norm_grad_plan(long long n_rows, long long width, int bytes, const void* dx, long long dx_stride, int n_cus) {
  const bool bf16 = bytes == 4, words = at_words(dx, dx_stride);
  const long long vectors = width / (bf16 ? 8 : 4);
  NormGradPlan p{0, 0, 0, 0};
  auto held = [&](int threads, int teams, int most, int of_a_cu) {
    if (p.teams != 0 || vectors > threads * most) return;
    const long long each = (n_rows + teams - 1) / teams, even = teams > 1 ? (each + 1) / 2 * 2 : each;
    const long long parts = std::max((long long)n_cus, std::min((long long)of_a_cu * n_cus, n_rows / 6));
    p = {threads, teams, most, (int)std::min(even, (parts + 1) / 2 * 2)};
  };
  held(64, 4, 1, 2);
  held(64, 4, 2, 2);
  if (bf16) {
    held(64, 4, 3, 2);
    if (words && width == 8 * 256) held(64, 4, 4, 1);
    held(128, 1, 2, 6);
    held(128, 1, 3, 4);
    held(256, 1, 2, 3);
    held(256, 1, 3, 2);
    if (words && width == 8 * 1024) held(256, 1, 4, 2);
    held(1024, 1, 1, 1);
  } else {
    held(64, 4, 4, 2);
    held(64, 4, 5, 2);
    held(256, 1, 2, bytes == 6 ? 3 : 2);
    held(256, 1, 3, bytes == 6 ? 3 : 2);
    held(512, 1, 2, 2);
    held(1024, 1, 2, 1);
  }
  if (p.teams == 0) {
    const long long tiles = (width - 1) / (8 * kColumnThreads) + 1;
    p.parts = (int)std::min(n_rows, std::max(1LL, (8LL * n_cus + tiles - 1) / tiles));
  }
  return p;
}

size_t norm_grad_bytes(long long n_rows, long long width, int bytes, const void* dx, long long dx_stride, int sums, int n_cus) {
  const NormGradPlan p = norm_grad_plan(n_rows, width, bytes, dx, dx_stride, n_cus);
  return 4 * (size_t)sums * (size_t)p.parts * (size_t)width + (p.teams == 0 ? 8 * (size_t)n_rows : 0);
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
