// The next token of every row under temperature, top-k, top-p and min-p, from given Exp(1) random numbers.
//
// With t = z / temperature and independent E ~ Exp(1), the arg-max of t - log E over a set of tokens is a draw from softmax(t)
// restricted to that set: no normalisation, no running sum over the vocabulary whose rounding decides the token, and random
// numbers are read for the kept tokens alone.  The kept tokens are a prefix of the ranking by (logit, index), so what a limit
// asks for is the place of a cut in that ranking: after k tokens, or where the mass before a token reaches its share.
//
// A workgroup owns a row.  One pass finds the largest logit and the sum of the exponentials.  A bound from it leaves a few
// candidates of the ranking's head:
//   top-k   the k-th largest of the threads' own maxima: at least k logits are no smaller;
//   top-p   tokens of at most (1 - top_p) / vocab of the mass each hold no more than 1 - top_p together;
//   min-p   its own condition.
// A second pass collects them in LDS, where they are sorted and their masses summed.  If there are more than LDS holds, passes
// that count tokens and mass in 2,048 ranges of the ranking narrow the cut down to one range until it does.
// Masses are summed as fixed-point numbers, so no result depends on the order in which threads arrive.
#include "ais_internal.h"
#include "device_utils.h"

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
  u64 wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  float wave_max[kWaves];
  MaxSum wave_sum[kWaves];
  Best wave_best[kWaves];
  uint32_t n;
  int bin;                             // the range that holds the cut, -1: none does
  uint32_t bin_count;                  // its tokens
  u64 above_mass;                      // of the tokens before it
  uint32_t above_count;
  u64 total;
};

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

  // f(logits, first index) of every vector and g(logit, index) of every element outside the vectors.
  template <typename F, typename G>
  __device__ __forceinline__ void visit(F f, G g) const {
    constexpr int N = Vec<T>::N;
    const u32x4* zv = reinterpret_cast<const u32x4*>(z + head);
    for (int i = threadIdx.x; i < nvec; i += kThreads) {
      float x[N];
      Vec<T>::unpack(zv[i], x);
      f(x, head + i * N);
    }
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
    visit(
        [&](const float* x, int v) {
          float m = x[0];
#pragma unroll
          for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
          if (m >= least) {
#pragma unroll
            for (int j = 0; j < N; ++j)
              if (x[j] >= least) f(x[j], v + j);
          }
        },
        [&](float x, int v) {
          if (x >= least) f(x, v);
        });
  }
};

__device__ __forceinline__ float clamped_noise(float e) { return fmaxf(fminf(e, 3.0e38f), 1.17549435e-38f); }

__device__ __forceinline__ Best block_best(Best b, SampleShared& sh) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) b = better(b, Best{__shfl_xor(b.score, d), __shfl_xor(b.token, d)});
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

// The cut among the tokens whose keys lie in [lo, hi) and whose logits are no smaller than `least`, before which none is
// left out.
template <typename T>
__device__ Cut cut_row(const Row<T>& row, float least, u64 lo, u64 hi, uint32_t limit_count, u64 limit_mass,
                       SampleShared& sh) {
  uint32_t above_count = 0;
  u64 above_mass = 0;
  while (true) {
    int shift = 0;
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
    row.visit_from(least, [&](float x, int v) {
      const u64 k = row.key(x, v);
      if (k >= lo && k < hi) {
        const uint32_t bin = (uint32_t)((k - lo) >> shift);
        atomicAdd(&sh.count[bin], 1u);
        atomicAdd(&sh.mass[bin], row.mass(x));
      }
    });
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
    if (sh.bin < 0) return Cut{hi, above_count + before.all_count, above_mass + before.all_mass};
    const u64 width = 1ull << shift;
    const u64 start = lo + ((u64)sh.bin << shift);
    hi = hi - start < width ? hi : start + width;
    lo = start;
    above_count = sh.above_count;
    above_mass = sh.above_mass;
    const uint32_t n = sh.bin_count;
    if (n > (uint32_t)kCap) continue;
    row.visit_from(least, [&](float x, int v) {
      const u64 k = row.key(x, v);
      if (k >= lo && k < hi) sh.keys[atomicAdd(&sh.n, 1u)] = k;
    });
    __syncthreads();
    sort_keys(n, sh);
    return cut_sorted(row, n, above_count, above_mass, limit_count, limit_mass, hi, sh);
  }
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
  const float top_p = limits.top_p != nullptr ? limits.top_p[r] : 1.f;
  const float min_p = limits.min_p != nullptr ? limits.min_p[r] : 0.f;
  int k = limits.top_k != nullptr ? limits.top_k[r] : 0;
  auto refuse = [&] {
    if (tid == 0) atomicOr(status, AIS_STATUS_BAD_ROW);
    answer(-1, 0.f, 0.f);
  };
  const bool greedy = temperature == 0.f;
  if (!(temperature >= 0.f) || temperature > 3.0e38f || top_p != top_p || min_p != min_p) {
    refuse();
    return;
  }
  if (greedy || top_p <= 0.f || min_p > 1.f) k = 1;
  const bool by_count = k > 0 && k < vocab, by_mass = top_p < 1.f && k != 1, by_share = min_p > 0.f && k != 1;

  Row<T> row;
  row.z = logits + r * row_stride;
  row.vocab = vocab;
  row.head = (reinterpret_cast<uintptr_t>(row.z) & 15) == 0 ? 0 : head_elements(row.z, vocab);
  row.nvec = (vocab - row.head) / N;
  row.rest = vocab - row.nvec * N;
  row.index_bits = vocab > 1 ? 32 - __builtin_clz((unsigned)(vocab - 1)) : 1;
  row.mass_bits = min(40, 62 - row.index_bits);
  row.c = greedy ? kLog2e : kLog2e / temperature;

  // ---- the largest logit and the sum of the exponentials ----
  MaxSum st{kNegHuge, 0.f};
  float top = -__builtin_inff();
  row.visit(
      [&](const float* x, int) {
        accumulate<N>(x, row.c, st);
#pragma unroll
        for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
      },
      [&](float x, int) {
        accumulate<1>(&x, row.c, st);
        top = fmaxf(top, x);
      });
  const float own_top = top;
  st = wave_merge(st);
  top = wave_max(top);
  if ((tid & 63) == 0) {
    sh.wave_sum[tid >> 6] = st;
    sh.wave_max[tid >> 6] = top;
  }
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
  const float* e = noise + r * noise_stride;
  auto scored = [&](float x, int v) { return Best{row.exponent(x) - log2_fast(clamped_noise(e[v])), v}; };
  Best best{-__builtin_inff(), vocab};
  u64 kept_mass = 0;
  if (k == 1) {
    row.visit_from(top, [&](float x, int v) { best = better(best, Best{0.f, v}); });
    best = block_best(best, sh);
    answer(best.token, 0.f, greedy ? 0.f : (float)-log((double)total));
    return;
  }
  if (!by_count && !by_mass && !by_share) {
    row.visit_from(-3.4028235e38f, [&](float x, int v) { best = better(best, scored(x, v)); });
  } else {
    // ---- a bound on the logits that can be kept ----
    float least = -3.4028235e38f;
    float share = -__builtin_inff();                   // log2 of the least mass, by min-p
    if (by_share) share = log2_fast(min_p);
    if (by_count && k <= kThreads) {
      sh.keys[tid] = (u64)(~ordered(own_top));
      sort_keys(kThreads, sh);
      const float pivot = from_ordered(~(uint32_t)sh.keys[k - 1]);
      least = fmaxf(least, pivot);
      __syncthreads();
    }
    if (!by_count) {
      float low = share;
      if (by_mass) low = fmaxf(low, log2_fast((1.f - top_p) * total / (float)vocab) - 0.01f);
      // (x - top) c >= low, with room for its rounding: the condition itself is looked at again
      least = fmaxf(least, top + low / row.c - 1e-5f * (fabsf(top) + fabsf(low / row.c)));
    }
    if (tid == 0) sh.n = 0;
    __syncthreads();
    row.visit_from(least, [&](float x, int v) {
      if (!by_count && row.exponent(x) < share) return;
      const uint32_t at = atomicAdd(&sh.n, 1u);
      if (at < (uint32_t)kCap) sh.keys[at] = row.key(x, v);
    });
    __syncthreads();
    const uint32_t n = sh.n;
    const uint32_t limit_count = by_count ? (uint32_t)k : 0xffffffffu;
    const u64 end_key = kNoLimit;
    auto share_of = [&](double mass) { return (u64)fmax((double)top_p * mass, 1.0); };
    const u64 limit_mass = by_mass && !by_count ? share_of(ldexp((double)total, row.mass_bits)) : kNoLimit;
    Cut cut;
    const bool listed = n <= (uint32_t)kCap;
    if (listed) {
      sort_keys(n, sh);
      cut = cut_sorted(row, n, 0, 0, limit_count, limit_mass, end_key, sh);
      if (by_count && by_mass) cut = cut_sorted(row, n, 0, 0, limit_count, share_of((double)cut.mass), end_key, sh);
    } else {
      const u64 lo = row.key(top, 0), hi = row.key(least, vocab - 1) + 1;
      cut = cut_row(row, least, lo, hi, limit_count, limit_mass, sh);
      if (by_count && by_mass) cut = cut_row(row, least, lo, hi, limit_count, share_of((double)cut.mass), sh);
    }
    // ---- the draw ----
    // min-p beside top-k, or beside a list that was not made by it, ends the prefix earlier; its tokens' mass is summed here
    auto look = [&](float x, u64 key) {
      if (key >= cut.key || row.exponent(x) < share) return;
      kept_mass += row.mass(x);
      best = better(best, scored(x, row.token(key)));
    };
    if (listed) {
      for (uint32_t i = tid; i < n; i += kThreads) look(row.value(sh.keys[i]), sh.keys[i]);
    } else {
      row.visit_from(least, [&](float x, int v) { look(x, row.key(x, v)); });
    }
    const Before sum = scan(0, kept_mass, sh);
    kept_mass = sum.all_mass;
  }
  best = block_best(best, sh);
  if (tid != 0) return;
  if (best.token >= vocab) {                           // not reached: the first ranked token is always kept
    answer(-1, 0.f, 0.f);
    return;
  }
  const double at = (double)row.exponent(Vec<T>::load1(row.z + best.token)) * 0.6931471805599453;
  const double full = at - log((double)total);
  answer(best.token, (float)(kept_mass > 0 ? at - log(ldexp((double)kept_mass, -row.mass_bits)) : full), (float)full);
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
