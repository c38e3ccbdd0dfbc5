// The next token of every row under temperature, top-k, top-p and min-p, from given Exp(1) random numbers.
//
// With t = z / temperature and independent E ~ Exp(1), the arg-max of t - log E over a set of tokens is a draw from softmax(t)
// restricted to that set: no normalisation, no running sum over the vocabulary whose rounding decides the token, and random
// numbers are read for the kept tokens alone.  The kept tokens are a prefix of the ranking by (logit, index), so what a limit
// asks for is the place of a cut in that ranking: after k tokens, or where the mass before a token reaches its share.
//
// A workgroup owns a row.  A row without limits takes one pass over logits and random numbers.  Otherwise one pass finds the
// largest logit, the sum of the exponentials, and each thread's own largest logit, of which a wavefront then makes a bound
// that leaves little more than the kept tokens:
//   top-k   the k-th largest of the threads' own: at least k logits are no smaller;
//   top-p   where the masses of the threads' own alone reach the share;
//   min-p   is a bound itself.
// A second pass collects what is no smaller in LDS.  Up to 64 tokens are sorted, summed and drawn from by one wavefront in its
// registers, up to 2,048 by the workgroup.  Where there is no such bound (flat rows, or more tokens than threads), tokens and
// their masses are counted in 2,048 ranges of the exponent, and the range in which the cut lies is sorted.
// Masses are summed as fixed-point numbers, so no result depends on the order in which threads arrive.
#include "ais_internal.h"
#include "device_utils.h"

#include <type_traits>

namespace ais {
namespace {

using namespace dev;

typedef unsigned long long u64;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kCap = 2048;             // candidates that LDS holds; two for each thread
constexpr u64 kNoLimit = ~0ull;

// Numbers whose unsigned order is that of the floats (-0 is made +0 first).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}

struct Best {
  float score;
  int token;
};
__device__ __forceinline__ Best better(Best a, Best b) {
  return b.score > a.score || (b.score == a.score && b.token < a.token) ? b : a;
}

struct SampleShared {
  u64 mass[kBins];
  u64 keys[kCap];
  uint32_t count[kBins];
  float own_top[kThreads];
  u64 wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  float wave_max[kWaves];
  MaxSum wave_sum[kWaves];
  Best wave_best[kWaves];
  float least;
  int bounded;
  uint32_t n;
  int bin;                             // the range that holds the cut, -1: none does
  uint32_t bin_count;                  // its tokens
  u64 above_mass;                      // of the tokens before it
  uint32_t above_count;
};

// Element j of a vector.
template <typename T>
__device__ __forceinline__ float element(u32x4 q, int j) {
  const int w = j * (int)sizeof(T) / 4;
  const uint32_t word = w < 2 ? (w == 0 ? q[0] : q[1]) : (w == 2 ? q[2] : q[3]);
  if constexpr (sizeof(T) == 4) return __uint_as_float(word);
  return __uint_as_float((j & 1) ? word & 0xffff0000u : word << 16);
}

// A row and how its tokens are ranked.
template <typename T>
struct Row {
  const T* z;
  int vocab, head, nvec, rest;
  int index_bits;
  float top, c;                        // largest logit, log2(e) / temperature
  int mass_bits;
  __device__ __forceinline__ float exponent(float x) const { return (x - top) * c; }      // log2 of its mass
  __device__ __forceinline__ u64 mass(float x) const {
    return (u64)ldexpf(exp2_fast(exponent(x)), mass_bits);
  }
  __device__ __forceinline__ u64 key(float x, int v) const { return (u64)(~ordered(x)) << index_bits | (u64)v; }
  __device__ __forceinline__ float value(u64 key) const { return from_ordered(~(uint32_t)(key >> index_bits)); }
  __device__ __forceinline__ int token(u64 key) const { return (int)(key & ((1ull << index_bits) - 1)); }

  // f(logits, first index) of every kUnroll vectors, their logits one after the other, and g(logit, index) of every element outside
  // them.  In f the logits of vector u begin at u N and have the index v + u kThreads N.
  template <int kUnroll, typename F, typename F1, typename G>
  __device__ __forceinline__ void visit(F f, F1 f1, G g) const {
    constexpr int N = Vec<T>::N;
    const u32x4* zv = reinterpret_cast<const u32x4*>(z + head);
    int i = threadIdx.x;
    for (; i + (kUnroll - 1) * kThreads < nvec; i += kUnroll * kThreads) {
      u32x4 q[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) q[u] = zv[i + u * kThreads];
      f(q, head + i * N);
    }
    for (; i < nvec; i += kThreads) f1(zv[i], head + i * N);
    const int r = threadIdx.x;
    if (r < rest) {
      const int v = r < head ? r : nvec * N + r;
      g(Vec<T>::load1(z + v), v);
    }
  }
  // f(logit, index) of every element that is no smaller than `least`.
  template <typename F>
  __device__ __forceinline__ void visit_from(float least, F f) const {
    constexpr int N = Vec<T>::N;
    auto one = [&](u32x4 q, int v) {
      float x[N];
      Vec<T>::unpack(q, x);
      float m = x[0];
#pragma unroll
      for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
      if (m >= least) {
        uint32_t found = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) found |= (uint32_t)(x[j] >= least) << j;
        while (found != 0) {                           // one copy of f, whatever the vector holds
          const int j = __builtin_ctz(found);
          found &= found - 1;
          f(element<T>(q, j), v + j);
        }
      }
    };
    visit<4>(
        [&](const u32x4* q, int v) {
#pragma unroll
          for (int u = 0; u < 4; ++u) one(q[u], v + u * kThreads * N);
        },
        one,
        [&](float x, int v) {
          if (x >= least) f(x, v);
        });
  }
};

__device__ __forceinline__ float clamped_noise(float e) { return fmaxf(fminf(e, 3.0e38f), 1.17549435e-38f); }

__device__ __forceinline__ Best wave_best(Best b) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) b = better(b, Best{__shfl_xor(b.score, d), __shfl_xor(b.token, d)});
  return b;
}
__device__ __forceinline__ Best block_best(Best b, SampleShared& sh) {
  b = wave_best(b);
  if ((threadIdx.x & 63) == 0) sh.wave_best[threadIdx.x >> 6] = b;
  __syncthreads();
  b = sh.wave_best[0];
  for (int w = 1; w < kWaves; ++w) b = better(b, sh.wave_best[w]);
  return b;
}

// Sums of count and mass over the threads before this one, and over all.
struct Before {
  uint32_t count, all_count;
  u64 mass, all_mass;
};
__device__ __forceinline__ Before scan(uint32_t count, u64 mass, SampleShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t c = count;
  u64 m = mass;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t pc = __shfl_up(c, d);
    const u64 pm = __shfl_up(m, d);
    if (lane >= d) {
      c += pc;
      m += pm;
    }
  }
  __syncthreads();
  if (lane == 63) {
    sh.wave_count[wave] = c;
    sh.wave_mass[wave] = m;
  }
  __syncthreads();
  Before b{c - count, 0, m - mass, 0};
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) {
      b.count += sh.wave_count[w];
      b.mass += sh.wave_mass[w];
    }
    b.all_count += sh.wave_count[w];
    b.all_mass += sh.wave_mass[w];
  }
  return b;
}

// Sorts sh.keys[0 .. n) in ascending order; what lies beyond, up to the next power of two, is overwritten.
__device__ __forceinline__ void sort_keys(uint32_t n, SampleShared& sh) {
  uint32_t size = 2;
  while (size < n) size <<= 1;
  for (uint32_t i = n + threadIdx.x; i < size; i += kThreads) sh.keys[i] = ~0ull;
  __syncthreads();
  for (uint32_t run = 2; run <= size; run <<= 1) {
    for (uint32_t d = run >> 1; d > 0; d >>= 1) {
      for (uint32_t p = threadIdx.x; p < size / 2; p += kThreads) {
        const uint32_t i = 2 * p - (p & (d - 1)), j = i + d;
        const u64 a = sh.keys[i], b = sh.keys[j];
        if ((a > b) == ((i & run) == 0)) {
          sh.keys[i] = b;
          sh.keys[j] = a;
        }
      }
      __syncthreads();
    }
  }
}

// Where the kept tokens end: those whose key is less than `key` are kept.
struct Cut {
  u64 key;
  uint32_t count;
  u64 mass;
};

// The cut among the sorted keys of LDS, before which `above` tokens rank: the first that is the limit_count-th or has
// limit_mass before it.  All threads get it.
template <typename T>
__device__ Cut cut_sorted(const Row<T>& row, uint32_t n, uint32_t above_count, u64 above_mass, uint32_t limit_count,
                          u64 limit_mass, u64 end_key, SampleShared& sh) {
  const uint32_t i = 2 * threadIdx.x;
  const u64 k0 = i < n ? sh.keys[i] : 0, k1 = i + 1 < n ? sh.keys[i + 1] : 0;
  const u64 m0 = i < n ? row.mass(row.value(k0)) : 0, m1 = i + 1 < n ? row.mass(row.value(k1)) : 0;
  const Before b = scan((i < n) + (i + 1 < n), m0 + m1, sh);
  const u64 before0 = above_mass + b.mass, before1 = before0 + m0;
  const bool kept0 = i < n && above_count + i < limit_count && before0 < limit_mass;
  const bool kept1 = i + 1 < n && above_count + i + 1 < limit_count && before1 < limit_mass;
  const Before kept = scan((uint32_t)kept0 + (uint32_t)kept1, (kept0 ? m0 : 0) + (kept1 ? m1 : 0), sh);
  Cut cut{end_key, above_count + kept.all_count, above_mass + kept.all_mass};
  if (kept.all_count < n) cut.key = sh.keys[kept.all_count];
  return cut;
}

// The cut of the whole row: the tokens no smaller than `least`, and of those that `depth` (in log2 of the mass) below the largest
// or deeper only the last range knows.
template <typename T>
__device__ Cut cut_row(const Row<T>& row, float least, float depth, uint32_t limit_count, u64 limit_mass, bool by_mass,
                       SampleShared& sh) {
  const float per_range = (float)kBins / depth;
  auto range_of = [&](float x) { return (int)fminf(-row.exponent(x) * per_range, (float)(kBins - 1)); };
  int within = -1;                                     // the range that the ones below are parts of
  uint32_t above_count = 0;
  u64 above_mass = 0, lo = 0, hi = kNoLimit;
  while (true) {
    int shift = 0;
    if (within >= 0)
      while (((hi - lo - 1) >> shift) >= (u64)kBins) ++shift;
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
      sh.count[b] = 0;
      sh.mass[b] = 0;
    }
    if (threadIdx.x == 0) {
      sh.bin = -1;
      sh.n = 0;
    }
    __syncthreads();
    auto add = [&](uint32_t bin, float x) {
      atomicAdd(&sh.count[bin], 1u);
      if (by_mass) atomicAdd(&sh.mass[bin], row.mass(x));
    };
    if (within < 0) {
      row.visit_from(least, [&](float x, int) { add((uint32_t)range_of(x), x); });
    } else {
      row.visit_from(least, [&](float x, int v) {
        if (range_of(x) != within) return;
        const u64 k = row.key(x, v);
        if (k >= lo && k < hi) add((uint32_t)((k - lo) >> shift), x);
      });
    }
    __syncthreads();
    const int b0 = 2 * threadIdx.x;
    const uint32_t c0 = sh.count[b0], c1 = sh.count[b0 + 1];
    const u64 m0 = sh.mass[b0], m1 = sh.mass[b0 + 1];
    const Before before = scan(c0 + c1, m0 + m1, sh);
    // the cut lies in the first range after which a limit is reached
    auto look = [&](int b, uint32_t cb, u64 mb, uint32_t c, u64 m) {
      const bool inside = above_count + cb < limit_count && above_mass + mb < limit_mass;
      const bool after = above_count + cb + c >= limit_count || above_mass + mb + m >= limit_mass;
      if (c > 0 && inside && after) {
        sh.bin = b;
        sh.bin_count = c;
        sh.above_count = above_count + cb;
        sh.above_mass = above_mass + mb;
      }
    };
    look(b0, before.count, before.mass, c0, m0);
    look(b0 + 1, before.count + c0, before.mass + m0, c1, m1);
    __syncthreads();
    const int bin = sh.bin;
    if (bin < 0) return Cut{hi, above_count + before.all_count, above_mass + before.all_mass};
    if (within < 0) {
      // the keys of the range's logits, with room for the rounding of their exponents
      within = bin;
      const float upper = row.top - (float)bin / per_range / row.c, lower = row.top - (float)(bin + 1) / per_range / row.c;
      const float room = 1e-5f * (fabsf(row.top) + fabsf(lower));
      lo = row.key(fminf(upper + room, row.top), 0);
      hi = row.key(bin == kBins - 1 ? -3.4028235e38f : fmaxf(lower - room, -3.4028235e38f), row.vocab - 1) + 1;
    } else {
      const u64 width = 1ull << shift;
      const u64 start = lo + ((u64)bin << shift);
      hi = hi - start < width ? hi : start + width;
      lo = start;
    }
    above_count = sh.above_count;
    above_mass = sh.above_mass;
    const uint32_t n = sh.bin_count;
    if (n > (uint32_t)kCap) continue;
    row.visit_from(least, [&](float x, int v) {
      if (range_of(x) != within) return;
      const u64 k = row.key(x, v);
      if (k >= lo && k < hi) sh.keys[atomicAdd(&sh.n, 1u)] = k;
    });
    __syncthreads();
    sort_keys(n, sh);
    return cut_sorted(row, n, above_count, above_mass, limit_count, limit_mass, hi, sh);
  }
}

// What a row's limits ask for.
struct Limits {
  bool by_count, by_mass, by_share;
  uint32_t count;
  float top_p, share;                  // share: log2 of min-p
  u64 mass;                            // that top-p without top-k ends at
  __device__ __forceinline__ u64 part_of(double m) const { return (u64)fmax((double)top_p * m, 1.0); }
};

// A bound on the kept logits from the threads' own largest, by one wavefront; false if they allow none.
template <typename T>
__device__ bool bound(const Row<T>& row, const Limits& lim, float total, const float* own_top, float* least) {
  constexpr int kOwn = kThreads / 64;
  const int lane = threadIdx.x & 63;
  float v[kOwn];
#pragma unroll
  for (int j = 0; j < kOwn; ++j) v[j] = own_top[j * 64 + lane];
  if (lim.by_count) {
    auto count = [&](float from) {
      uint32_t c = 0;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) c += (uint32_t)__builtin_popcountll(__ballot(v[j] >= from));
      return c;
    };
    const float lowest = -3.4028235e38f;
    if (count(lowest) < lim.count) return false;
    uint32_t lo = ordered(lowest), hi = ordered(row.top);
    const uint32_t enough = lim.count + (lim.count >> 3) + 2;
    while (hi - lo > 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const uint32_t c = count(from_ordered(mid));
      if (c < lim.count) {
        hi = mid;
      } else {
        lo = mid;
        if (c <= enough) break;
      }
    }
    *least = from_ordered(lo);
    return true;
  }
  float p[kOwn];
#pragma unroll
  for (int j = 0; j < kOwn; ++j) p[j] = exp2_fast(row.exponent(v[j]));
  auto mass = [&](float from) {
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) m += v[j] >= from ? p[j] : 0.f;
    return wave_sum(m);
  };
  // rounding of the sums must not cost a token that the fixed-point sums keep
  const float wanted = lim.top_p * total * 1.00001f;
  float hi = row.top, lo = row.top - 32.f / row.c;
  if (!(mass(lo) >= wanted)) return false;
  for (int k = 0; k < 13; ++k) {
    const float mid = 0.5f * (lo + hi);
    if (mass(mid) >= wanted) lo = mid;
    else hi = mid;
  }
  *least = lo;
  return true;
}

struct Drawn {
  Best best;
  u64 kept_mass;
};

// Up to 64 candidates, by one wavefront: sorted by exchanges between its lanes, lane i then has the i-th.
template <typename T, typename S>
__device__ Drawn draw_from_few(const Row<T>& row, const Limits& lim, uint32_t n, const u64* keys, S scored) {
  const uint32_t i = threadIdx.x & 63;
  u64 key = i < n ? keys[i] : kNoLimit;
#pragma unroll
  for (uint32_t run = 2; run <= 64; run <<= 1)
#pragma unroll
    for (uint32_t d = run >> 1; d > 0; d >>= 1) {
      const u64 other = __shfl_xor(key, (int)d);
      const bool keep_less = ((i & d) == 0) == ((i & run) == 0);
      key = (other < key) == keep_less ? other : key;
    }
  const float x = i < n ? row.value(key) : row.top;
  const u64 m = i < n ? row.mass(x) : 0;
  auto sum_to = [&](u64 own) {
    u64 s = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const u64 p = __shfl_up(s, d);
      if ((int)i >= d) s += p;
    }
    return s;
  };
  const u64 upto = sum_to(m);
  u64 limit = lim.mass;
  if (lim.by_count && lim.by_mass) limit = lim.part_of((double)__shfl(upto, (int)min(n, lim.count) - 1));
  const bool kept = i < n && i < lim.count && upto - m < limit && row.exponent(x) >= lim.share;
  Drawn d{{-__builtin_inff(), row.vocab}, __shfl(sum_to(kept ? m : 0), 63)};
  if (kept) d.best = scored(x, row.token(key));
  d.best = wave_best(d.best);
  return d;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const T* __restrict__ logits, long long row_stride, int vocab,
                                                          const float* __restrict__ noise, long long noise_stride,
                                                          const unsigned char* __restrict__ valid, SampleLimits limits,
                                                          int* __restrict__ token_out, float* __restrict__ logp_out,
                                                          float* __restrict__ full_out, int* __restrict__ status) {
  constexpr int N = Vec<T>::N;
  __shared__ SampleShared sh;
  const long long r = blockIdx.x;
  const int tid = threadIdx.x;
  auto answer = [&](int token, float logp, float full) {
    if (tid != 0) return;
    token_out[r] = token;
    logp_out[r] = logp;
    if (full_out != nullptr) full_out[r] = full;
  };
  if (valid != nullptr && valid[r] == 0) {
    answer(-1, 0.f, 0.f);
    return;
  }
  const float temperature = limits.temperature != nullptr ? limits.temperature[r] : 1.f;
  const float min_p = limits.min_p != nullptr ? limits.min_p[r] : 0.f;
  int k = limits.top_k != nullptr ? limits.top_k[r] : 0;
  Limits lim;
  lim.top_p = limits.top_p != nullptr ? limits.top_p[r] : 1.f;
  auto refuse = [&] {
    if (tid == 0) atomicOr(status, AIS_STATUS_BAD_ROW);
    answer(-1, 0.f, 0.f);
  };
  const bool greedy = temperature == 0.f;
  if (!(temperature >= 0.f) || temperature > 3.0e38f || lim.top_p != lim.top_p || min_p != min_p) {
    refuse();
    return;
  }
  if (greedy || lim.top_p <= 0.f || min_p > 1.f) k = 1;
  lim.by_count = k > 0 && k < vocab;
  lim.by_mass = lim.top_p < 1.f;
  lim.by_share = min_p > 0.f;
  lim.count = lim.by_count ? (uint32_t)k : 0xffffffffu;
  lim.share = lim.by_share ? log2_fast(min_p) : -__builtin_inff();
  lim.mass = kNoLimit;

  Row<T> row;
  row.z = logits + r * row_stride;
  row.vocab = vocab;
  row.head = (reinterpret_cast<uintptr_t>(row.z) & 15) == 0 ? 0 : head_elements(row.z, vocab);
  row.nvec = (vocab - row.head) / N;
  row.rest = vocab - row.nvec * N;
  row.index_bits = vocab > 1 ? 32 - __builtin_clz((unsigned)(vocab - 1)) : 1;
  row.mass_bits = min(40, 62 - row.index_bits);
  row.c = greedy ? kLog2e : kLog2e / temperature;
  const float* e = noise + r * noise_stride;
  const bool open = k != 1 && !lim.by_count && !lim.by_mass && !lim.by_share;

  // ---- the largest logit and the sum of the exponentials; without limits the draw as well ----
  MaxSum st{kNegHuge, 0.f};
  float top = -__builtin_inff();
  Best best{-__builtin_inff(), vocab};
  auto fold = [&](const float* x, auto count) {
    constexpr int n = decltype(count)::value;
    accumulate<n>(x, row.c, st);
#pragma unroll
    for (int j = 0; j < n; ++j) top = fmaxf(top, x[j]);
  };
  if (open) {
    // indices rise, so that an equal score does not take a lower one's place; the threads' best are scored again below, relative
    // to the largest logit
    auto race = [&](float x, float noise_of, int v) {
      const float score = __builtin_fmaf(x, row.c, -log2_fast(clamped_noise(noise_of)));
      if (score > best.score) best = Best{score, v};
    };
    auto one = [&](u32x4 q, int v) {
      float x[N], w[N];
      Vec<T>::unpack(q, x);
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = __builtin_nontemporal_load(e + v + j);
      fold(x, std::integral_constant<int, N>{});
#pragma unroll
      for (int j = 0; j < N; ++j) race(x[j], w[j], v + j);
    };
    row.template visit<2>(
        [&](const u32x4* q, int v) {
          float x[2 * N], w[2 * N];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) w[u * N + j] = __builtin_nontemporal_load(e + v + u * kThreads * N + j);
#pragma unroll
          for (int u = 0; u < 2; ++u) Vec<T>::unpack(q[u], x + u * N);
          fold(x, std::integral_constant<int, 2 * N>{});
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) race(x[u * N + j], w[u * N + j], v + u * kThreads * N + j);
        },
        one,
        [&](float x, int v) {
          fold(&x, std::integral_constant<int, 1>{});
          const float score = __builtin_fmaf(x, row.c, -log2_fast(clamped_noise(e[v])));
          best = better(best, Best{score, v});
        });
  } else {
    row.template visit<4>(
        [&](const u32x4* q, int) {
          float x[4 * N];
#pragma unroll
          for (int u = 0; u < 4; ++u) Vec<T>::unpack(q[u], x + u * N);
          fold(x, std::integral_constant<int, 4 * N>{});
        },
        [&](u32x4 q, int) {
          float x[N];
          Vec<T>::unpack(q, x);
          fold(x, std::integral_constant<int, N>{});
        },
        [&](float x, int) { fold(&x, std::integral_constant<int, 1>{}); });
    sh.own_top[tid] = top;
  }
  st = wave_merge(st);
  top = wave_max(top);
  if ((tid & 63) == 0) {
    sh.wave_sum[tid >> 6] = st;
    sh.wave_max[tid >> 6] = top;
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  st = sh.wave_sum[0];
  for (int w = 0; w < kWaves; ++w) {
    if (w > 0) st = merge(st, sh.wave_sum[w]);
    top = fmaxf(top, sh.wave_max[w]);
  }
  row.top = top;
  // a NaN or +inf makes the sum NaN; nothing but -inf leaves no largest
  if (!(st.s > 0.f) || !(st.m < 3.4e38f) || !(top > -3.4e38f)) {
    refuse();
    return;
  }
  // the sum relative to the largest logit's exponential: st.m is the rounded product top * c
  const float total = st.s * exp2_fast(-__builtin_fmaf(top, row.c, -st.m));
  auto scored = [&](float x, int v) { return Best{row.exponent(x) - log2_fast(clamped_noise(e[v])), v}; };
  auto finish = [&](int token, u64 kept_mass) {
    if (tid != 0) return;
    if (token >= vocab) {                              // not reached: the first ranked token is always kept
      answer(-1, 0.f, 0.f);
      return;
    }
    const double at = (double)row.exponent(Vec<T>::load1(row.z + token)) * 0.6931471805599453;
    const double full = at - log((double)total);
    answer(token, (float)(kept_mass > 0 ? at - log(ldexp((double)kept_mass, -row.mass_bits)) : full), (float)full);
  };
  if (k == 1) {
    best = Best{-__builtin_inff(), vocab};
    row.visit_from(top, [&](float, int v) { best = better(best, Best{0.f, v}); });
    best = block_best(best, sh);
    answer(best.token, 0.f, greedy ? 0.f : (float)-log((double)total));
    return;
  }
  if (open) {
    if (best.token < vocab) best = scored(Vec<T>::load1(row.z + best.token), best.token);
    finish(block_best(best, sh).token, 0);
    return;
  }
  if (lim.by_mass && !lim.by_count) lim.mass = lim.part_of(ldexp((double)total, row.mass_bits));
  // (x - top) c >= the least exponent, with room for its rounding: the condition itself is looked at again
  auto from_exponent = [&](float low) { return top + low / row.c - 1e-5f * (fabsf(top) + fabsf(low / row.c)); };
  const float lowest = -3.4028235e38f;
  float least = lim.by_share && !lim.by_count ? fmaxf(from_exponent(lim.share), lowest) : lowest;
  u64 kept_mass = 0, end_key = kNoLimit;
  auto look = [&](float x, u64 key) {
    if (key >= end_key || row.exponent(x) < lim.share) return;
    kept_mass += row.mass(x);
    best = better(best, scored(x, row.token(key)));
  };
  if (lim.by_count || lim.by_mass) {
    // ---- candidates ----
    if (tid < 64) {
      float bounded = lowest;
      const bool some = bound(row, lim, total, sh.own_top, &bounded);
      if (tid == 0) {
        sh.bounded = some;
        sh.least = bounded;
      }
    }
    __syncthreads();
    uint32_t n = 0xffffffffu;
    if (sh.bounded) {
      const float from = fmaxf(least, sh.least);
      row.visit_from(from, [&](float x, int v) {
        const uint32_t at = atomicAdd(&sh.n, 1u);
        if (at < (uint32_t)kCap) sh.keys[at] = row.key(x, v);
      });
      __syncthreads();
      n = sh.n;
    }
    if (n <= 64) {
      if (tid >= 64) return;
      const Drawn d = draw_from_few(row, lim, n, sh.keys, scored);
      finish(d.best.token, d.kept_mass);
      return;
    }
    Cut cut;
    if (n <= (uint32_t)kCap) {
      sort_keys(n, sh);
      cut = cut_sorted(row, n, 0, 0, lim.count, lim.mass, kNoLimit, sh);
      if (lim.by_count && lim.by_mass) cut = cut_sorted(row, n, 0, 0, lim.count, lim.part_of((double)cut.mass), kNoLimit, sh);
      end_key = cut.key;
      for (uint32_t i = tid; i < n; i += kThreads) look(row.value(sh.keys[i]), sh.keys[i]);
      best = block_best(best, sh);
      kept_mass = scan(0, kept_mass, sh).all_mass;
      finish(best.token, kept_mass);
      return;
    }
    // tokens of at most (1 - top_p) / vocab of the mass each hold no more than 1 - top_p together
    float depth = 64.f;
    if (!lim.by_count) {
      const float low = fmaxf(lim.share, log2_fast((1.f - lim.top_p) * total / (float)vocab) - 0.01f);
      least = fmaxf(least, from_exponent(low));
      depth = fmaxf(-low, 1.f);
    }
    // with both limits the first cut, by count, tells the mass that top-p is a share of
    u64 limit_mass = lim.mass;
    for (int pass = lim.by_count && lim.by_mass ? 0 : 1; pass < 2; ++pass) {
      cut = cut_row(row, least, depth, lim.count, limit_mass, lim.by_mass, sh);
      limit_mass = lim.part_of((double)cut.mass);
    }
    end_key = cut.key;
  }
  // ---- the draw from the row itself ----
  row.visit_from(least, [&](float x, int v) { look(x, row.key(x, v)); });
  best = block_best(best, sh);
  kept_mass = scan(0, kept_mass, sh).all_mass;
  finish(best.token, kept_mass);
}

}  // namespace

int launch_sample_tokens(ais_ctx* ctx, const void* logits, ais_dtype dtype, long long n_rows, int vocab, long long row_stride,
                         const float* noise, long long noise_stride, const unsigned char* valid, const SampleLimits& limits,
                         int* token_out, float* logp_out, float* logp_full_out) {
  if (n_rows == 0) return AIS_OK;
  ScopedTimer timer(ctx, AIS_K_SAMPLE);
  const dim3 grid((unsigned)n_rows), block(kThreads);
  if (dtype == AIS_BF16)
    sample_kernel<bf16_t><<<grid, block, 0, ctx->stream>>>(static_cast<const bf16_t*>(logits), row_stride, vocab, noise,
                                                           noise_stride, valid, limits, token_out, logp_out, logp_full_out,
                                                           ctx->status_dev);
  else
    sample_kernel<float><<<grid, block, 0, ctx->stream>>>(static_cast<const float*>(logits), row_stride, vocab, noise,
                                                          noise_stride, valid, limits, token_out, logp_out, logp_full_out,
                                                          ctx->status_dev);
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
