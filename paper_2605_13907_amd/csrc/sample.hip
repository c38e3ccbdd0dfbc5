// The next token of every row under temperature, top-k, top-p and min-p, from given Exp(1) random numbers.
//
// With t = z / temperature and independent E ~ Exp(1), the arg-max of t - log E over a set of tokens is a draw from softmax(t)
// restricted to that set: no normalisation, no running sum over the vocabulary whose rounding decides the token.  Random numbers
// are read for the kept tokens alone, except where the draw passes over the row itself, which reads them all.  The kept tokens are a prefix of the ranking by (logit, index), so what a limit
// asks for is the place of a cut in that ranking: after k tokens, or where the mass before a token reaches its share.
//
// A workgroup owns a row.  A row without limits takes one pass over logits and random numbers.  Otherwise one pass finds the
// largest logit, the sum of the exponentials, and the largest logit of each of four parts of every thread's, which make a bound
// that leaves little more than the kept tokens:
//   top-k   the k-th largest of the parts' own: at least k logits are no smaller;
//   top-p   where the masses of the parts' own alone reach the share;
//   min-p   is a bound itself.
// A second pass collects what is no smaller in LDS.  Up to 64 tokens are sorted, summed and drawn from by one wavefront in its
// registers.  Up to 4,096, tokens and masses are counted in 2,048 ranges of the exponent, and the range in which the cut lies is
// sorted.  Where there is no such bound (flat rows, more tokens than parts) the same is done to the row itself; of a bf16 row the
// tokens of every value are counted instead, whose masses follow from their number, so that a token costs one addition in LDS.
// The tokens that share the cut's value are found by the draw, which passes over such a row sixteen tokens at a time.
// Masses are summed as fixed-point numbers, so no result depends on the order in which threads arrive.
//
// Measured, us a call, logits in the cache of a step that made them: bf16 rows of 151,936 without limits 18 (1 row), 21 (64) and
// 45 (256: 233 MB, 5.2 TB/s); of 64 such rows with limits 35 (top-k), 17 (min-p), 67 (top-p over flat rows, all of whose tokens
// pass the bound).  64 rows with limits of their own take as long as the slowest of them: of 60 batches 32 took 22 to 27, where no row
// has many candidates, 21 took 30 to 55, and 7 with a row that keeps 8,000 tokens or more 61 to 89.  Few rows are bound by one compute unit's exponentials and reading of its row and the barriers between the passes,
// many without limits by memory.  A kernel of 1,024 threads has 128 registers to each: what the compiler would compute early and keep
// (indices, addresses, widened numbers) went to scratch memory, and with it 64 rows under top-k took 46 us and 256 without limits 52.
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
constexpr int kCap = 4096;             // candidates that LDS holds
constexpr int kMembers = 2048;         // tokens of a range that are sorted; two for each thread
constexpr int kParts = 4;              // of a thread's logits
constexpr u64 kNoLimit = ~0ull;
constexpr float kLowest = -3.4028235e38f, kHighest = 3.4028235e38f;

// Numbers whose unsigned order is that of the floats (-0 is made +0 first).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}

// A number that all lanes have as a wider one, here and not earlier.
__device__ __forceinline__ double widened(float x) {
  asm volatile("" : "+s"(x));
  return (double)x;
}
// What another lane of the wavefront has, the lane's index modulo 64.
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_ds_bpermute(lane << 2, (int)x); }
__device__ __forceinline__ u64 from_lane(u64 x, int lane) {
  return (u64)from_lane((uint32_t)(x >> 32), lane) << 32 | from_lane((uint32_t)x, lane);
}
// A number that all lanes have, as one of the wavefront.
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

struct Best {
  float score;
  int token;
};
__device__ __forceinline__ Best better(Best a, Best b) {
  return b.score > a.score || (b.score == a.score && b.token < a.token) ? b : a;
}

// Values of bf16 that are told apart: magnitudes of 64 octaves from 2^-32 on, of either sign; smaller ones count as zero.
constexpr int kValues = 16384, kValueLow = 95 << 7;

struct SampleShared {
  union {
    struct {
      u64 mass[kBins];                 // of the ranges, later the sorted tokens of one
      uint32_t count[kBins];
      u64 keys[kCap];
    };
    uint32_t value_count[kValues];
  };
  u64 wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  float wave_max[kWaves];
  MaxSum wave_sum[kWaves];
  Best wave_best[kWaves];
  float vote_count[2][kWaves], vote_mass[2][kWaves];
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
    int i = fresh_thread();
    const int r = i;
    for (; i + (kUnroll - 1) * kThreads < nvec; i += kUnroll * kThreads) {
      u32x4 q[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) q[u] = zv[i + u * kThreads];
      f(q, head + i * N);
    }
    for (; i < nvec; i += kThreads) f1(zv[i], head + i * N);
    if (r < rest) {
      const int v = r < head ? r : nvec * N + r;
      g(Vec<T>::load1(z + v), v);
    }
  }
  // f(logit) of every element from `least` on, where that is most of them.
  template <typename F>
  __device__ __forceinline__ void visit_most(float least, F f) const {
    constexpr int N = Vec<T>::N;
    auto one = [&](u32x4 q, int) {
      float x[N];
      Vec<T>::unpack(q, x);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (x[j] >= least) f(x[j]);
    };
    visit<16 / N>(
        [&](const u32x4* q, int) {
#pragma unroll
          for (int u = 0; u < 16 / N; ++u) one(q[u], 0);
        },
        one,
        [&](float x, int) {
          if (x >= least) f(x);
        });
  }
  // f(logit, index) of every element in [least, most].
  template <typename F>
  __device__ __forceinline__ void visit_between(float least, float most, F f) const {
    constexpr int N = Vec<T>::N;
    auto one = [&](u32x4 q, int v) {
      float x[N];
      Vec<T>::unpack(q, x);
      uint32_t found = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) found |= (uint32_t)(x[j] >= least && x[j] <= most) << j;
      while (found != 0) {                             // one copy of f, whatever the vector holds
        const int j = __builtin_ctz(found);
        found &= found - 1;
        f(element<T>(q, j), v + j);
      }
    };
    visit<4>(
        [&](const u32x4* q, int v) {
#pragma unroll
          for (int u = 0; u < 4; ++u) one(q[u], v + u * kThreads * N);
        },
        one,
        [&](float x, int v) {
          if (x >= least && x <= most) f(x, v);
        });
  }
  template <typename F>
  __device__ __forceinline__ void visit_from(float least, F f) const {
    visit_between(least, kHighest, f);
  }
};

// N random numbers from p on, which lies at any multiple of four bytes.
template <int N>
__device__ __forceinline__ void load_noise(const float* p, float* w) {
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int j = 0; j < N; j += 4) {
    const f32x4_any q = *reinterpret_cast<const f32x4_any*>(p + j);
#pragma unroll
    for (int k = 0; k < 4; ++k) w[j + k] = q[k];
  }
}
// Between 2^-126 and 3e38, compared as whole numbers, whose order has negative numbers below and NaN above.
__device__ __forceinline__ float clamped_noise(float e) {
  return __int_as_float(min(max(__float_as_int(e), 0x00800000), 0x7f61b1e6));
}

// Folds n logits, the largest of which is `most`, into the running sum.
template <int n>
__device__ __forceinline__ void add_to(const float* x, float most, float scale, MaxSum& st) {
  const float mn = fmaxf(st.m, most * scale);
  float acc0 = st.s * exp2_fast(st.m - mn), acc1 = 0.f;
#pragma unroll
  for (int k = 0; k < n; k += 2) {
    acc0 += exp2_fast(__builtin_fmaf(x[k], scale, -mn));
    acc1 += exp2_fast(__builtin_fmaf(x[k + 1], scale, -mn));
  }
  st.m = mn;
  st.s = acc0 + acc1;
}

__device__ __forceinline__ Best wave_best(Best b) {
  const int tid = fresh_thread();
#pragma unroll
  for (int d = 1; d < 64; d <<= 1)
    b = better(b, Best{__uint_as_float(from_lane(__float_as_uint(b.score), tid ^ d)), (int)from_lane((uint32_t)b.token, tid ^ d)});
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
  const int tid = fresh_thread();
  const int lane = tid & 63, wave = tid >> 6;
  uint32_t c = count;
  u64 m = mass;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t pc = from_lane(c, lane - d);
    const u64 pm = from_lane(m, lane - d);
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

// A wavefront's keys in ascending order, by exchanges between its lanes.
__device__ __forceinline__ u64 wave_sorted(u64 key) {
  const uint32_t i = fresh_thread() & 63;
#pragma unroll
  for (uint32_t run = 2; run <= 64; run <<= 1)
#pragma unroll
    for (uint32_t d = run >> 1; d > 0; d >>= 1) {
      const u64 other = from_lane(key, (int)(i ^ d));
      const bool keep_less = ((i & d) == 0) == ((i & run) == 0);
      key = (other < key) == keep_less ? other : key;
    }
  return key;
}

// Sorts keys[0 .. n), n <= kMembers, in ascending order; what lies beyond, up to the next power of two, is overwritten.
__device__ __forceinline__ void sort_keys(uint32_t n, u64* keys) {
  const int tid = fresh_thread();
  if (n <= 64) {
    if (tid < 64) {
      const u64 key = wave_sorted(tid < n ? keys[tid] : kNoLimit);
      if (tid < n) keys[tid] = key;
    }
    __syncthreads();
    return;
  }
  uint32_t size = 128;
  while (size < n) size <<= 1;
  for (uint32_t i = n + tid; i < size; i += kThreads) keys[i] = kNoLimit;
  __syncthreads();
  for (uint32_t run = 2; run <= size; run <<= 1) {
    for (uint32_t d = run >> 1; d > 0; d >>= 1) {
      for (uint32_t p = tid; p < size / 2; p += kThreads) {
        const uint32_t i = 2 * p - (p & (d - 1)), j = i + d;
        const u64 a = keys[i], b = keys[j];
        if ((a > b) == ((i & run) == 0)) {
          keys[i] = b;
          keys[j] = a;
        }
      }
      __syncthreads();
    }
  }
}

// Where the kept tokens end: those whose key is less than `key` are kept, and of those of the logit `edge`, if take > 0, the first
// `take`, whose keys are not less.
struct Cut {
  u64 key;
  u64 mass;
  uint32_t take = 0;
  float edge = 0.f;
};

// Tokens among which the cut lies: their keys are in [lo, hi), `above` tokens rank before them.
struct Span {
  u64 lo, hi;
  uint32_t n, above_count;
  u64 above_mass;
};

// The cut among n sorted keys: the first that is the limit_count-th or has limit_mass before it.  All threads get it.
template <typename T>
__device__ __forceinline__ Cut cut_sorted(const Row<T>& row, const Span& s, uint32_t limit_count, u64 limit_mass, const u64* keys,
                          SampleShared& sh) {
  const int tid = fresh_thread();
  const uint32_t n = s.n;
  if (n <= 64) {                                       // one wavefront looks at them and tells the others
    __syncthreads();
    if (tid < 64) {
      const uint32_t i = tid;
      const u64 m = i < n ? row.mass(row.value(keys[i])) : 0;
      u64 upto = m;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const u64 p = from_lane(upto, (int)i - d);
        if ((int)i >= d) upto += p;
      }
      const bool kept = i < n && s.above_count + i < limit_count && s.above_mass + upto - m < limit_mass;
      const uint32_t all = (uint32_t)__builtin_popcountll(__ballot(kept));
      const u64 mass = from_lane(upto, (int)max(all, 1u) - 1);
      if (i == 0) {
        sh.wave_count[0] = all;
        sh.wave_mass[0] = all > 0 ? mass : 0;
      }
    }
    __syncthreads();
    const uint32_t all = sh.wave_count[0];
    return Cut{all < n ? keys[all] : keys[n - 1] + 1, s.above_mass + sh.wave_mass[0]};
  }
  const uint32_t i = 2 * tid;
  const u64 k0 = i < n ? keys[i] : 0, k1 = i + 1 < n ? keys[i + 1] : 0;
  const u64 m0 = i < n ? row.mass(row.value(k0)) : 0, m1 = i + 1 < n ? row.mass(row.value(k1)) : 0;
  const Before b = scan((i < n) + (i + 1 < n), m0 + m1, sh);
  const u64 before0 = s.above_mass + b.mass, before1 = before0 + m0;
  const bool kept0 = i < n && s.above_count + i < limit_count && before0 < limit_mass;
  const bool kept1 = i + 1 < n && s.above_count + i + 1 < limit_count && before1 < limit_mass;
  const Before kept = scan((uint32_t)kept0 + (uint32_t)kept1, (kept0 ? m0 : 0) + (kept1 ? m1 : 0), sh);
  // behind the last of them where all are kept, not at the span's end, which may reach over others
  const u64 end = kept.all_count < n ? keys[kept.all_count] : keys[n - 1] + 1;
  return Cut{end, s.above_mass + kept.all_mass};
}

// Where the cut lies among ranges of which each thread has kOwn: in the first one after which a limit is reached.  held(k, f) calls
// f(tokens, mass) with what the thread's k-th holds.  Sets sh.bin and what belongs to it; the sums over all ranges are returned.
template <int kOwn, typename Held>
__device__ __forceinline__ Before find_range(Held held, const Span& s, uint32_t limit_count, u64 limit_mass, SampleShared& sh) {
  const int tid = fresh_thread();
  uint32_t c = 0;
  u64 m = 0;
#pragma unroll 2
  for (int k = 0; k < kOwn; ++k)
    held(k, [&](uint32_t count, u64 mass) {
      c += count;
      m += mass;
    });
  const Before before = scan(c, m, sh);
  uint32_t above_count = s.above_count + before.count;
  u64 above_mass = s.above_mass + before.mass;
  // one thread at most has it among its own
  if (above_count < limit_count && above_mass < limit_mass && (above_count + c >= limit_count || above_mass + m >= limit_mass)) {
    for (int k = 0; k < kOwn; ++k)
      held(k, [&](uint32_t count, u64 mass) {
        const bool inside = above_count < limit_count && above_mass < limit_mass;
        const bool after = above_count + count >= limit_count || above_mass + mass >= limit_mass;
        if (count > 0 && inside && after) {
          sh.bin = kOwn * tid + k;
          sh.bin_count = count;
          sh.above_count = above_count;
          sh.above_mass = above_mass;
        }
        above_count += count;
        above_mass += mass;
      });
  }
  __syncthreads();
  return before;
}

// Counts what `each` gives to add(range, logit) in kBins ranges and finds the one with the cut; false if there is none, with the
// cut behind everything.
template <typename T, typename Each>
__device__ __forceinline__ bool narrow(const Row<T>& row, Each each, bool by_mass, uint32_t limit_count, u64 limit_mass, Span* s, Cut* cut,
                       SampleShared& sh) {
  const int tid = fresh_thread();
  __syncthreads();
  for (int b = tid; b < kBins; b += kThreads) {
    sh.count[b] = 0;
    sh.mass[b] = 0;
  }
  if (tid == 0) sh.bin = -1;
  __syncthreads();
  each([&](uint32_t bin, float x) {
    atomicAdd(&sh.count[bin], 1u);
    if (by_mass) atomicAdd(&sh.mass[bin], row.mass(x));
  });
  __syncthreads();
  constexpr int kOwn = kBins / kThreads;
  const Before all = find_range<kOwn>(
      [&](int k, auto f) { f(sh.count[kOwn * tid + k], sh.mass[kOwn * tid + k]); }, *s, limit_count, limit_mass, sh);
  if (sh.bin < 0) {
    *cut = Cut{s->hi, s->above_mass + all.all_mass};
    return false;
  }
  s->n = sh.bin_count;
  s->above_count = sh.above_count;
  s->above_mass = sh.above_mass;
  return true;
}

// The cut inside a span whose tokens are those of `each`: further ranges while there are more than can be sorted.
template <typename T, typename Each>
__device__ __forceinline__ Cut finish_cut(const Row<T>& row, Each each, Span s, bool by_mass, uint32_t limit_count, u64 limit_mass,
                          SampleShared& sh) {
  const int tid = fresh_thread();
  while (s.n > (uint32_t)kMembers) {
    int shift = 0;
    while (((s.hi - s.lo - 1) >> shift) >= (u64)kBins) ++shift;
    Cut cut;
    const bool some = narrow(
        row,
        [&](auto add) {
          each([&](float x, u64 key) {
            if (key >= s.lo && key < s.hi) add((uint32_t)((key - s.lo) >> shift), x);
          });
        },
        by_mass, limit_count, limit_mass, &s, &cut, sh);
    if (!some) return cut;
    const u64 start = s.lo + ((u64)sh.bin << shift), width = 1ull << shift;
    s.hi = s.hi - start < width ? s.hi : start + width;
    s.lo = start;
  }
  __syncthreads();                                     // the ranges have been read: their place is for the tokens now
  if (tid == 0) sh.n = 0;
  __syncthreads();
  each([&](float x, u64 key) {
    if (key < s.lo || key >= s.hi) return;
    const uint32_t at = atomicAdd(&sh.n, 1u);          // as many as were counted
    if (at < (uint32_t)kMembers) sh.mass[at] = key;
  });
  __syncthreads();
  sort_keys(s.n, sh.mass);
  return cut_sorted(row, s, limit_count, limit_mass, sh.mass, sh);
}

// The cut among the tokens whose logits all(f) gives to f, and each(f, least, most), those between two logits, with their keys: by
// ranges of the exponent down to `depth` (in log2 of the mass) below the largest logit's; what lies deeper is in the last one.
template <typename T, typename All, typename Each>
__device__ __forceinline__ Cut cut_by_exponent(const Row<T>& row, All all, Each each, float depth, bool by_mass, uint32_t limit_count, u64 limit_mass,
                               SampleShared& sh) {
  const float per_range = (float)kBins / depth;
  auto range_of = [&](float x) { return (int)fminf(-row.exponent(x) * per_range, (float)(kBins - 1)); };
  Span s{0, kNoLimit, 0, 0, 0};
  Cut cut;
  if (!narrow(
          row, [&](auto add) { all([&](float x) { add((uint32_t)range_of(x), x); }); }, by_mass, limit_count,
          limit_mass, &s, &cut, sh))
    return cut;
  // the keys of the range's logits, with room for the rounding of their exponents
  const int bin = sh.bin;
  const float upper = row.top - (float)bin / per_range / row.c, lower = row.top - (float)(bin + 1) / per_range / row.c;
  const float room = 1e-5f * (fabsf(row.top) + fabsf(lower));
  const float most = fminf(upper + room, row.top), least = bin == kBins - 1 ? kLowest : fmaxf(lower - room, kLowest);
  s.lo = row.key(most, 0);
  s.hi = row.key(least, row.vocab - 1) + 1;
  auto inside = [&](auto f) {
    each(
        [&](float x, u64 key) {
          if (range_of(x) == bin) f(x, key);
        },
        least, most);
  };
  return finish_cut(row, inside, s, by_mass, limit_count, limit_mass, sh);
}

// Place of a bf16 value, given as fp32, among those that are told apart, the largest first.
__device__ __forceinline__ int value_place(float x) {
  const int bits = __float_as_int(x + 0.f);            // a negative zero is a zero
  const int m = min(max((int)((uint32_t)bits >> 16 & 0x7fffu) - kValueLow, 0), kValues / 2 - 1);
  return kValues / 2 - 1 - (m ^ (bits >> 31));         // half + m where negative
}

// The cut among the tokens of a bf16 row that are no smaller than `least`: the tokens of every value are counted.
__device__ __forceinline__ Cut cut_by_value(const Row<bf16_t>& row, float least, uint32_t limit_count, u64 limit_mass, SampleShared& sh) {
  constexpr int kOwn = kValues / kThreads;
  const int tid = fresh_thread();
  __syncthreads();
  u32x4* counts = reinterpret_cast<u32x4*>(sh.value_count);
  for (int b = tid; b < kValues / 4; b += kThreads) counts[b] = u32x4{0, 0, 0, 0};
  if (tid == 0) sh.bin = -1;
  __syncthreads();
  auto add = [&](float x) {
    if (x >= least) atomicAdd(&sh.value_count[value_place(x)], 1u);
  };
  auto one = [&](u32x4 q, int) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      add(__uint_as_float(q[w] << 16));
      add(__uint_as_float(q[w] & 0xffff0000u));
    }
  };
  row.template visit<4>(
      [&](const u32x4* q, int v) {
#pragma unroll
        for (int u = 0; u < 4; ++u) one(q[u], v);
      },
      one, [&](float x, int) { add(x); });
  __syncthreads();
  auto value_of = [&](int place) {
    const int m = place >= kValues / 2 ? place - kValues / 2 : kValues / 2 - 1 - place;
    const float x = m == 0 ? 0.f : __uint_as_float((uint32_t)(m + kValueLow) << 16);
    return place >= kValues / 2 ? -x : x;
  };
  Span s{0, kNoLimit, 0, 0, 0};
  u32x4 own[kOwn / 4];
#pragma unroll
  for (int k = 0; k < kOwn / 4; ++k) own[k] = counts[kOwn / 4 * tid + k];
  const Before all = find_range<kOwn>(
      [&](int k, auto f) {
        uint32_t c = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) c = j == k ? own[j / 4][j % 4] : c;
        if (c > 0) f(c, c * row.mass(value_of(kOwn * tid + k)));
      },
      s, limit_count, limit_mass, sh);
  if (sh.bin < 0) return Cut{kNoLimit, all.all_mass};
  const int bin = sh.bin;
  s.n = sh.bin_count;
  s.above_count = sh.above_count;
  s.above_mass = sh.above_mass;
  // one value, or, at the ends of what is told apart, several
  const int from_zero = bin >= kValues / 2 ? bin - kValues / 2 : kValues / 2 - 1 - bin;
  const float x = value_of(bin), small = __uint_as_float((uint32_t)kValueLow << 16);
  float upper = x, lower = x;
  if (from_zero == 0) {
    upper = bin < kValues / 2 ? small : 0.f;
    lower = bin < kValues / 2 ? 0.f : -small;
  }
  if (bin == 0) upper = row.top;
  if (bin == kValues - 1) lower = kLowest;
  if (upper == lower && s.n <= (uint32_t)kMembers) {   // as many of them as the limits allow: the draw finds the first ones
    const u64 each = row.mass(x);
    u64 take = min(s.n, limit_count - s.above_count);
    if (each > 0 && limit_mass != kNoLimit) take = min(take, (limit_mass - s.above_mass + each - 1) / each);
    if (tid == 0) sh.n = 0;
    __syncthreads();
    return Cut{row.key(x, 0), s.above_mass + take * each, (uint32_t)take, x};
  }
  lower = uniform(fmaxf(lower, least));                       // several values may lie on both sides of the bound: those counted
  s.lo = row.key(upper, 0);
  s.hi = row.key(lower, row.vocab - 1) + 1;
  auto inside = [&](auto f) {
    row.visit_between(lower, upper, [&](float x, int v) {
      if (value_place(x) == bin) f(x, row.key(x, v));
    });
  };
  return finish_cut(row, inside, s, true, limit_count, limit_mass, sh);
}

// What a row's limits ask for.
struct Limits {
  bool by_count, by_mass, by_share;
  uint32_t count;
  float top_p, share;                  // share: log2 of min-p
  u64 mass;                            // that top-p without top-k ends at
  __device__ __forceinline__ u64 part_of(double m) const { return (u64)fmax(widened(top_p) * m, 1.0); }
};

// Sum of the wavefronts' votes, in every lane: exchanges inside rows of 16 lanes, one for each wavefront.
__device__ __forceinline__ float votes_of(const float* votes) {
  const int tid = fresh_thread();
  static_assert(kWaves == 16, "");
  float v = votes[tid & 15];
  v += dpp_move<kDppQuadXor1>(v);
  v += dpp_move<kDppQuadXor2>(v);
  v += dpp_move<kDppRowHalfMirror>(v);
  return v + dpp_move<kDppRowMirror>(v);
}

// A bound on the kept logits from the largest of the parts of every thread's logits; false if they allow none.
template <typename T>
__device__ __forceinline__ bool bound(const Row<T>& row, const Limits& lim, float total, const float* own_top, float* least, SampleShared& sh) {
  const int tid = fresh_thread();
  const int lane = tid & 63, wave = tid >> 6;
  int turn = 0;
  // one barrier for each question: the answers of the one before are read while those of the next are written
  auto count = [&](float from) {
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < kParts; ++j) c += (uint32_t)__builtin_popcountll(__ballot(own_top[j] >= from));
    float* votes = sh.vote_count[turn ^= 1];           // at most 4,096: exact
    if (lane == 0) votes[wave] = (float)c;
    __syncthreads();
    return (uint32_t)votes_of(votes);
  };
  float lo = row.top - 32.f / row.c, hi = row.top;
  if (lim.by_count) {
    if (lim.count > (uint32_t)(kParts * kThreads) || count(kLowest) < lim.count) return false;
    const uint32_t enough = lim.count + (lim.count >> 3) + 2;
    if (count(lo) >= lim.count) {
      for (int k = 0; k < 14; ++k) {
        const float mid = 0.5f * (lo + hi);
        const uint32_t c = count(mid);
        if (c < lim.count) {
          hi = mid;
        } else {
          lo = mid;
          if (c <= enough) break;
        }
      }
      *least = lo;
      return true;
    }
    // far below the largest, masked tokens perhaps: by the numbers' own order
    uint32_t a = ordered(kLowest), b = ordered(lo);
    while (b - a > 1) {
      const uint32_t mid = a + (b - a) / 2, c = count(from_ordered(mid));
      if (c < lim.count) {
        b = mid;
      } else {
        a = mid;
        if (c <= enough) break;
      }
    }
    *least = from_ordered(a);
    return true;
  }
  float p[kParts];
#pragma unroll
  for (int j = 0; j < kParts; ++j) p[j] = exp2_fast(row.exponent(own_top[j]));
  uint32_t parts = 0;                                  // as large as the last question's
  auto mass = [&](float from) {
    float m = 0.f;
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < kParts; ++j) {
      m += own_top[j] >= from ? p[j] : 0.f;
      c += (uint32_t)__builtin_popcountll(__ballot(own_top[j] >= from));
    }
    m = wave_sum(m);
    turn ^= 1;
    if (lane == 0) {
      sh.vote_mass[turn][wave] = m;
      sh.vote_count[turn][wave] = (float)c;
    }
    __syncthreads();
    parts = (uint32_t)votes_of(sh.vote_count[turn]);
    return votes_of(sh.vote_mass[turn]);
  };
  // rounding of the sums must not cost a token that the fixed-point sums keep
  const float wanted = lim.top_p * total * 1.00001f;
  if (!(mass(lo) >= wanted)) return false;
  // until few enough for one wavefront are left, most likely
  for (int k = 0; k < 12 && parts > 32; ++k) {
    const float mid = 0.5f * (lo + hi);
    const uint32_t before = parts;
    if (mass(mid) >= wanted) {
      lo = mid;
    } else {
      hi = mid;
      parts = before;
    }
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
__device__ __forceinline__ Drawn draw_from_few(const Row<T>& row, const Limits& lim, uint32_t n, const u64* keys, S scored) {
  const int tid = fresh_thread();
  const uint32_t i = tid & 63;
  const u64 key = wave_sorted(i < n ? keys[i] : kNoLimit);
  const float x = i < n ? row.value(key) : row.top;
  const u64 m = i < n ? row.mass(x) : 0;
  auto sum_to = [&](u64 own) {
    u64 s = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const u64 p = from_lane(s, (int)i - d);
      if ((int)i >= d) s += p;
    }
    return s;
  };
  const u64 upto = sum_to(m);
  u64 limit = lim.mass;
  if (lim.by_count && lim.by_mass) limit = lim.part_of((double)from_lane(upto, (int)min(n, lim.count) - 1));
  const bool kept = i < n && i < lim.count && upto - m < limit && row.exponent(x) >= lim.share;
  Drawn d{{-__builtin_inff(), row.vocab}, from_lane(sum_to(kept ? m : 0), 63)};
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
  lim.top_p = uniform(limits.top_p != nullptr ? limits.top_p[r] : 1.f);
  auto refuse = [&] {
    if (tid == 0) atomicOr(status, AIS_STATUS_BAD_ROW);
    answer(-1, 0.f, 0.f);
  };
  const bool greedy = temperature == 0.f;
  if (!(temperature >= 0.f) || temperature > kHighest || lim.top_p != lim.top_p || min_p != min_p) {
    refuse();
    return;
  }
  if (greedy || lim.top_p <= 0.f || min_p > 1.f) k = 1;
  lim.by_count = k > 0 && k < vocab;
  lim.by_mass = lim.top_p < 1.f;
  lim.by_share = min_p > 0.f;
  lim.count = lim.by_count ? (uint32_t)k : 0xffffffffu;
  lim.share = uniform(lim.by_share ? log2_fast(min_p) : -__builtin_inff());
  lim.mass = kNoLimit;

  Row<T> row;
  row.z = logits + r * row_stride;
  row.vocab = vocab;
  row.head = (reinterpret_cast<uintptr_t>(row.z) & 15) == 0 ? 0 : head_elements(row.z, vocab);
  row.nvec = (vocab - row.head) / N;
  row.rest = vocab - row.nvec * N;
  row.index_bits = vocab > 1 ? 32 - __builtin_clz((unsigned)(vocab - 1)) : 1;
  row.mass_bits = min(40, 62 - row.index_bits);
  row.c = uniform(greedy ? kLog2e : fminf(kLog2e / temperature, 3e38f));
  const float* e = noise + r * noise_stride;
  const bool open = k != 1 && !lim.by_count && !lim.by_mass && !lim.by_share;

  // ---- the largest logit and the sum of the exponentials; without limits the draw as well ----
  MaxSum st{kNegHuge, 0.f};
  float top = -__builtin_inff();
  Best best{-__builtin_inff(), vocab};
  float best_score = -__builtin_inff(), second_score = best_score;             // without limits: of a thread's vectors,
  int best_at = -1, best_many = 0;                     // where the best begin, and how many they are
  auto largest = [](const float* x) {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
    return m;
  };
  float own_top[kParts];                               // of a thread's first, second, ... vectors of four, and the rest
#pragma unroll
  for (int j = 0; j < kParts; ++j) own_top[j] = top;
  if (open) {
    // Sixteen logits and their random numbers at a time, of which only the best score is looked at; a thread keeps where its best
    // ones are and the second best of them.  What lies near the workgroup's best is read and scored again below, relative to the
    // largest logit.  (If every thread does that for its own best, it is as much to read as the row: 256 rows x 151,936 52 and
    // 68 us.)
    constexpr int kOpen = 16 / N;
    const u32x4* zv = reinterpret_cast<const u32x4*>(row.z + row.head);
    auto scores = [&](const float* x, const float* w, float* score, auto count) {
#pragma unroll
      for (int j = 0; j < decltype(count)::value; ++j)
        score[j] = __builtin_fmaf(x[j], row.c, -log2_fast(clamped_noise(w[j])));
    };
    auto race = [&](const float* score, int i, int many) {
      float m = score[0];
#pragma unroll
      for (int j = 1; j < N; ++j) m = fmaxf(m, score[j]);
      if (many > 1) {
#pragma unroll
        for (int j = N; j < 16; ++j) m = fmaxf(m, score[j]);
      }
      second_score = fmaxf(second_score, fminf(m, best_score));
      if (m > best_score) {
        best_score = m;
        best_at = i;
        best_many = many;
      }
    };
    int i = tid;
    for (; i + (kOpen - 1) * kThreads < row.nvec; i += kOpen * kThreads) {
      u32x4 q[kOpen];
      float x[16], w[16], score[16];
#pragma unroll
      for (int u = 0; u < kOpen; ++u) q[u] = zv[i + u * kThreads];
#pragma unroll
      for (int u = 0; u < kOpen; ++u) load_noise<N>(e + row.head + (i + u * kThreads) * N, w + u * N);
      float most = -__builtin_inff();
#pragma unroll
      for (int u = 0; u < kOpen; ++u) {
        Vec<T>::unpack(q[u], x + u * N);
        most = fmaxf(most, largest(x + u * N));
      }
      add_to<16>(x, most, row.c, st);
      top = fmaxf(top, most);
      scores(x, w, score, std::integral_constant<int, 16>{});
      race(score, i, kOpen);
    }
    for (; i < row.nvec; i += kThreads) {
      float x[N];
      Vec<T>::unpack(zv[i], x);
      const float most = largest(x);
      add_to<N>(x, most, row.c, st);
      top = fmaxf(top, most);
      float w[N], score[N];
      load_noise<N>(e + row.head + i * N, w);
      scores(x, w, score, std::integral_constant<int, N>{});
      race(score, i, 1);
    }
    if (tid < row.rest) {
      const int v = tid < row.head ? tid : row.nvec * N + tid;
      const float x = Vec<T>::load1(row.z + v);
      accumulate<1>(&x, row.c, st);
      top = fmaxf(top, x);
      best = Best{__builtin_fmaf(x, row.c, -log2_fast(clamped_noise(e[v]))), v};
    }
  } else {
    int single = 0;
    row.template visit<kParts>(
        [&](const u32x4* q, int) {
          float x[kParts * N];
#pragma unroll
          for (int u = 0; u < kParts; ++u) Vec<T>::unpack(q[u], x + u * N);
          float most = -__builtin_inff();
#pragma unroll
          for (int u = 0; u < kParts; ++u) {
            const float m = largest(x + u * N);
            most = fmaxf(most, m);
            own_top[u] = fmaxf(own_top[u], m);
          }
          add_to<kParts * N>(x, most, row.c, st);
        },
        [&](u32x4 q, int) {
          float x[N];
          Vec<T>::unpack(q, x);
          const float m = largest(x);
          add_to<N>(x, m, row.c, st);
#pragma unroll
          for (int u = 0; u < kParts; ++u) own_top[u] = u == single ? fmaxf(own_top[u], m) : own_top[u];
          ++single;                                    // at most three of them
        },
        [&](float x, int) {
          accumulate<1>(&x, row.c, st);
          own_top[kParts - 1] = fmaxf(own_top[kParts - 1], x);
        });
#pragma unroll
    for (int j = 0; j < kParts; ++j) top = fmaxf(top, own_top[j]);
  }
  st = wave_merge(st);
  top = wave_max(top);
  const float wave_score = open ? wave_max(fmaxf(best_score, best.score)) : 0.f;
  if ((tid & 63) == 0) {
    sh.wave_sum[tid >> 6] = st;
    sh.wave_max[tid >> 6] = top;
    sh.vote_mass[0][tid >> 6] = wave_score;
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  st = sh.wave_sum[0];
  for (int w = 0; w < kWaves; ++w) {
    if (w > 0) st = merge(st, sh.wave_sum[w]);
    top = fmaxf(top, sh.wave_max[w]);
  }
  top = uniform(top);
  row.top = top;
  // the sum relative to the largest logit's exponential: st.m is the rounded product top * c
  float total = st.s * exp2_fast(-__builtin_fmaf(top, row.c, -st.m));
  // Far from zero products are rounded to whole numbers or do not fit.  If the largest logit's is, or if a thread that has nothing but the
  // type's lowest value made the sum something else than a number, it is taken again.
  const bool far = !(fabsf(top * row.c) < 1e9f);
  if (far || !(total > 0.5f) || !(total < kHighest)) {
    float own = 0.f;
    if (fabsf(top) <= kHighest) {
      for (uint32_t v = tid; v < (uint32_t)vocab; v += kThreads) own += exp2_fast(row.exponent(Vec<T>::load1(row.z + v)));
    }
    own = wave_sum(own);
    __syncthreads();
    if ((tid & 63) == 0) sh.vote_mass[1][tid >> 6] = own;
    __syncthreads();
    total = 0.f;
    for (int w = 0; w < kWaves; ++w) total += sh.vote_mass[1][w];
    __syncthreads();                                   // the bound's questions write there again
  }
  total = uniform(total);
  // none of +inf, NaN and nothing but -inf has a sum of 1 or more
  if (!(total > 0.5f) || !(total < kHighest)) {
    refuse();
    return;
  }
  auto scored = [&](float x, int v) { return Best{row.exponent(x) - log2_fast(clamped_noise(e[v])), v}; };
  auto finish = [&](int token, u64 kept_mass) {
    if (tid != 0) return;
    if (token >= vocab) {                              // not reached: the first ranked token is always kept
      answer(-1, 0.f, 0.f);
      return;
    }
    const double at = (double)row.exponent(Vec<T>::load1(row.z + token)) * 0.6931471805599453;
    const double full = at - log(widened(total));
    answer(token, (float)(kept_mass > 0 ? at - log(ldexp((double)kept_mass, -row.mass_bits)) : full), (float)full);
  };
  // Scores the best vectors, or all vectors, of the threads that ask for it once more, the wavefront for each of them together.
  auto look_again = [&](bool ask, bool all, auto score) {
    for (u64 who = __ballot(ask); who != 0; who &= who - 1) {
      const int lane = __builtin_ctzll(who);
      const bool every = __shfl((int)all, lane) != 0;
      const int from = every ? (tid & ~63) + lane : __shfl(best_at, lane);
      const int n = (every ? (row.nvec - from + kThreads - 1) / kThreads : __shfl(best_many, lane)) * N;
      for (int j = tid & 63; j < n; j += 64) best = better(best, score(row.head + (from + j / N * kThreads) * N + j % N));
    }
  };
  if (k == 1) {
    best = Best{-__builtin_inff(), vocab};
    row.visit_from(top, [&](float, int v) { best = better(best, Best{0.f, v}); });
    best = block_best(best, sh);
    answer(best.token, 0.f, greedy ? 0.f : (float)-log(widened(total)));
    return;
  }
  if (open) {
    float near = sh.vote_mass[0][0];
    for (int w = 1; w < kWaves; ++w) near = fmaxf(near, sh.vote_mass[0][w]);
    near -= 1e-6f * (fabsf(near) + fabsf(top * row.c) + 300.f);                // some times what the scores are rounded by
    if (far) best.token = tid < row.rest ? (tid < row.head ? tid : row.nvec * N + tid) : vocab;
    best = (far || best.score >= near) && best.token < vocab ? scored(Vec<T>::load1(row.z + best.token), best.token)
                                                             : Best{-__builtin_inff(), vocab};
    // all of a thread's vectors: rare, except at very large logits over the temperature
    look_again(far || best_score >= near, far || second_score >= near, [&](int v) { return scored(Vec<T>::load1(row.z + v), v); });
    finish(block_best(best, sh).token, 0);
    return;
  }
  best = Best{-__builtin_inff(), vocab};
  if (lim.by_mass && !lim.by_count) lim.mass = lim.part_of(ldexp(widened(total), row.mass_bits));
  // (x - top) c >= the least exponent, with room for its rounding: the condition itself is looked at again
  auto from_exponent = [&](float low) { return top + low / row.c - 1e-5f * (fabsf(top) + fabsf(low / row.c)); };
  float least = lim.by_share && !lim.by_count ? fmaxf(from_exponent(lim.share), kLowest) : kLowest;
  u64 kept_mass = 0;
  Cut cut{kNoLimit, 0};
  const bool sum_mass = !lim.by_mass || lim.by_share;  // of the kept tokens; otherwise the cut tells it
  // ---- candidates ----
  float bounded = kLowest;
  const bool cuts = lim.by_count || lim.by_mass;        // min-p is a bound by itself
  const bool some = !cuts || bound(row, lim, total, own_top, &bounded, sh);
  if (some) least = fmaxf(least, bounded);
  uint32_t n = 0xffffffffu;
  if (some) {
    // a part whose largest logit is smaller has none
    const u32x4* zv = reinterpret_cast<const u32x4*>(row.z + row.head);
    auto keep = [&](uint32_t at, float x, int v) {
      if (at < (uint32_t)kCap) sh.keys[at] = row.key(x, v);
    };
#pragma unroll
    for (int u = 0; u < kParts; ++u) {
      if (own_top[u] < least) continue;
      constexpr int kAhead = 5;
      for (int i = tid + u * kThreads; i < row.nvec; i += kAhead * kParts * kThreads) {
        u32x4 q[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) q[a] = zv[min(i + a * kParts * kThreads, row.nvec - 1)];
        u64 found = 0;
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          float x[N];
          Vec<T>::unpack(q[a], x);
          uint32_t here = 0;
#pragma unroll
          for (int j = 0; j < N; ++j) here |= (uint32_t)(x[j] >= least) << j;
          if (i + a * kParts * kThreads < row.nvec) found |= (u64)here << (a * N);
        }
        if (found == 0) continue;
        uint32_t at = atomicAdd(&sh.n, (uint32_t)__popcll(found));
        for (; found != 0 && at < (uint32_t)kCap; found &= found - 1) {        // read again: they are few, or counted only
          const int j = __builtin_ctzll(found);
          const int v = row.head + (i + j / N * (kParts * kThreads)) * N + j % N;
          keep(at++, Vec<T>::load1(row.z + v), v);
        }
      }
      if (u == kParts - 1 && tid < row.rest) {
        const int v = tid < row.head ? tid : row.nvec * N + tid;
        const float x = Vec<T>::load1(row.z + v);
        if (x >= least) keep(atomicAdd(&sh.n, 1u), x, v);
      }
    }
    __syncthreads();
    n = sh.n;
  }
  if (n <= 64) {
    if (tid >= 64) return;
    const Drawn d = draw_from_few(row, lim, n, sh.keys, scored);
    finish(d.best.token, d.kept_mass);
    return;
  }
  const bool listed = n <= (uint32_t)kCap;
  if (cuts) {
    // log2 of the least mass that a token can be kept with, by the candidates' bound; without one, tokens of at most
    // (1 - top_p) / vocab of the mass each hold no more than 1 - top_p together
    float low = row.exponent(least);
    if (!some && !lim.by_count) {
      low = fmaxf(lim.share, log2_fast((1.f - lim.top_p) * total / (float)vocab) - 0.01f);
      least = fmaxf(least, from_exponent(low));
    }
    const float depth = fminf(fmaxf(-low, 1.f), 64.f);
    // with both limits the first cut, by count, tells the mass that top-p is a share of
    u64 limit_mass = lim.mass;
    for (int pass = lim.by_count && lim.by_mass ? 0 : 1; pass < 2; ++pass) {
      // nothing that follows from these is computed before the loop and kept
      asm volatile("" : "+s"(row.top), "+s"(row.c), "+s"(row.mass_bits), "+s"(row.index_bits));
      if (listed) {
        auto each = [&](auto f, float, float) {
          for (uint32_t i = tid; i < n; i += kThreads) f(row.value(sh.keys[i]), sh.keys[i]);
        };
        auto all = [&](auto f) {
          for (uint32_t i = tid; i < n; i += kThreads) f(row.value(sh.keys[i]));
        };
        cut = cut_by_exponent(row, all, each, depth, lim.by_mass, lim.count, limit_mass, sh);
      } else {
        bool done = false;
        if constexpr (sizeof(T) == 2) {
          // what counts as zero has the same mass but for 2^-32 c < 2^-20 of the exponent; the last value and what lies beyond, almost
          // 2^31 below the largest logit and more, none
          if (fabsf(top) < 2147483648.f && row.c < 4096.f && row.c > 3.1e-8f) {
            cut = cut_by_value(row, least, lim.count, limit_mass, sh);
            done = true;
          }
        }
        if (!done) {
          auto each = [&](auto f, float from, float to) {
            row.visit_between(fmaxf(from, least), to, [&](float x, int v) { f(x, row.key(x, v)); });
          };
          auto all = [&](auto f) { row.visit_most(least, f); };
          cut = cut_by_exponent(row, all, each, depth, lim.by_mass, lim.count, limit_mass, sh);
        }
      }
      limit_mass = lim.part_of((double)cut.mass);
    }
    if (!sum_mass) kept_mass = cut.mass;
  }
  if (listed) {
    for (uint32_t i = tid; i < n; i += kThreads) {
      const float x = row.value(sh.keys[i]);
      if (sh.keys[i] >= cut.key || row.exponent(x) < lim.share) continue;
      if (sum_mass) kept_mass += row.mass(x);
      best = better(best, scored(x, row.token(sh.keys[i])));
    }
    best = block_best(best, sh);
    if (sum_mass) kept_mass = scan(0, kept_mass, sh).all_mass;
    finish(best.token, kept_mass);
    return;
  }
  // ---- the draw from the row itself: sixteen logits at a time, of which only the best score is looked at, as above; all of the
  // row's random numbers are read, at the same time as its logits.
  const float last = uniform(cut.key == kNoLimit ? least : fmaxf(least, row.value(cut.key)));
  // of the tokens of that logit; all of them where the cut is the next smaller one's, of which zero's next is a zero too
  const int end = __builtin_amdgcn_readfirstlane(
      cut.key >> row.index_bits == row.key(last, 0) >> row.index_bits ? row.token(cut.key) : vocab);
  const uint32_t take = __builtin_amdgcn_readfirstlane(cut.take);
  const float edge = uniform(cut.edge);
  constexpr int kOpen = 16 / N;
  const int head = __builtin_amdgcn_readfirstlane(row.head), nvec = __builtin_amdgcn_readfirstlane(row.nvec);
  const u32x4* zv = reinterpret_cast<const u32x4*>(logits + r * row_stride + head);
  const float* ev = noise + r * noise_stride + head;
  const float share = uniform(lim.share), scale = uniform(row.c), origin = uniform(row.top);
  best_score = -__builtin_inff();
  best_at = -1;
  best_many = 0;
  auto full_score = [&](float x, float noise_of) { return (x - origin) * scale - log2_fast(clamped_noise(noise_of)); };
  auto score_of = [&](float x, float noise_of, int v) {
    float score = full_score(x, noise_of);
    asm volatile("" : "+v"(score));                    // a choice of two numbers, no branch for each token
    const bool kept = ((x > last) | ((x == last) & (v < end))) & ((x - origin) * scale >= share);
    return kept ? score : -__builtin_inff();
  };
  auto at_edge = [&](float x, int v) {                 // no more than there is room for
    sh.mass[atomicAdd(&sh.n, 1u)] = (u64)v << 32 | __float_as_uint(full_score(x, ev[v - head]));
  };
  auto race = [&](auto many, int i) {
    constexpr int kMany = decltype(many)::value;
    u32x4 q[kMany];
    float x[kMany * N], w[kMany * N];
#pragma unroll
    for (int u = 0; u < kMany; ++u) q[u] = zv[i + u * kThreads];
#pragma unroll
    for (int u = 0; u < kMany; ++u) load_noise<N>(ev + (i + u * kThreads) * N, w + u * N);
#pragma unroll
    for (int u = 0; u < kMany; ++u) Vec<T>::unpack(q[u], x + u * N);
#pragma unroll
    for (int j = 0; j < kMany * N; ++j) w[j] = score_of(x[j], w[j], head + (i + j / N * kThreads) * N + j % N);
    float m = w[0];
#pragma unroll
    for (int j = 1; j < kMany * N; ++j) m = fmaxf(m, w[j]);
    auto each = [&](uint32_t found, auto f) {          // f(logit, index): few of them, mostly
      for (; found != 0; found &= found - 1) {
        const int j = __builtin_ctz(found), v = head + (i + j / N * kThreads) * N + j % N;
        f(Vec<T>::load1(row.z + v), v);
      }
    };
    if (sum_mass && m > -__builtin_inff()) {
      uint32_t found = 0;
#pragma unroll
      for (int j = 0; j < kMany * N; ++j) found |= (uint32_t)(w[j] > -__builtin_inff()) << j;
      each(found, [&](float z, int) { kept_mass += row.mass(z); });
    }
    if (take > 0) {
      uint32_t found = 0;
#pragma unroll
      for (int j = 0; j < kMany * N; ++j) found |= (uint32_t)(x[j] == edge) << j;
      each(found, at_edge);
    }
    if (m > best_score) {
      best_score = m;
      best_at = i;
      best_many = kMany;
    }
  };
  int i = fresh_thread();
  for (; i + (kOpen - 1) * kThreads < nvec; i += kOpen * kThreads) race(std::integral_constant<int, kOpen>{}, i);
  for (; i < nvec; i += kThreads) race(std::integral_constant<int, 1>{}, i);
  best = Best{-__builtin_inff(), vocab};
  if (tid < row.rest) {
    const int v = tid < head ? tid : nvec * N + tid;
    const float x = Vec<T>::load1(row.z + v);
    best.score = score_of(x, e[v], v);
    if (best.score > -__builtin_inff()) {
      best.token = v;
      if (sum_mass) kept_mass += row.mass(x);
    }
    if (take > 0 && x == edge) at_edge(x, v);
  }
  const float won = wave_max(fmaxf(best_score, best.score));
  if ((tid & 63) == 0) sh.vote_mass[0][tid >> 6] = won;
  __syncthreads();
  float first = sh.vote_mass[0][0];
  for (int w = 1; w < kWaves; ++w) first = fmaxf(first, sh.vote_mass[0][w]);
  look_again(best_score >= first, false, [&](int v) { return Best{score_of(Vec<T>::load1(row.z + v), e[v], v), v}; });
  if (take > 0 && row.exponent(edge) >= share) {
    sort_keys(sh.n, sh.mass);
    for (uint32_t j = tid; j < take; j += kThreads) {
      if (sum_mass) kept_mass += row.mass(edge);
      best = better(best, Best{__uint_as_float((uint32_t)sh.mass[j]), (int)(sh.mass[j] >> 32)});
    }
  }
  best = block_best(best, sh);
  if (sum_mass) kept_mass = scan(0, kept_mass, sh).all_mass;
  finish(best.token, kept_mass);
}

}  // namespace

int launch_sample_tokens(ais_ctx* ctx, const void* logits, ais_dtype dtype, long long n_rows, int vocab, long long row_stride,
                         const float* noise, long long noise_stride, const unsigned char* valid, const SampleLimits& limits,
                         int* token_out, float* logp_out, float* logp_full_out) {
  if (n_rows == 0) return AIS_OK;
  ScopedTimer timer(ctx, AIS_K_SAMPLE);
  auto run = [&](auto type) {
    typedef decltype(type) T;
    constexpr long long kMostRows = (1LL << 31) / kThreads;                    // of a launch
    auto from = [](auto* p, long long r) { return p != nullptr ? p + r : nullptr; };
    for (long long r = 0; r < n_rows; r += kMostRows)
      sample_kernel<T><<<dim3((unsigned)(n_rows - r < kMostRows ? n_rows - r : kMostRows)), dim3(kThreads), 0, ctx->stream>>>(
          static_cast<const T*>(logits) + r * row_stride, row_stride, vocab, noise + r * noise_stride, noise_stride, from(valid, r),
          SampleLimits{from(limits.temperature, r), from(limits.top_k, r), from(limits.top_p, r), from(limits.min_p, r)},
          token_out + r, logp_out + r, from(logp_full_out, r), ctx->status_dev);
  };
  if (dtype == AIS_BF16) run(bf16_t{});
  else run(float{});
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
