// Distillation from a teacher's top logits: the divergence of a row's policy from the teacher's distribution over the tokens
// it lists, and the gradient with respect to the row's logits.
//
//   q = softmax(teacher / T) over the listed tokens,  p = softmax(z / T) over the vocabulary,
//   kl = sum_j q_j (log q_j - log p[id_j]),  dz = weight / T (p - sum_j q_j 1[id_j])
//
// A workgroup owns a row.  Beside the soft-max over the vocabulary, which is all of the traffic, there is little: the listed
// tokens' logits are gathered, and their elements of the gradient differ from the others'.  A token that is listed twice counts
// with both entries: a small hash table finds the entries of one token, their q added as fixed-point numbers, whose sum does
// not depend on the order.
//
// Rows that fit are held by one compute unit, in registers and, beyond 20 vectors a lane, in LDS: one read and one write of the
// row.  The loads of a row are all on their way before the teacher's part begins, which they hide; a listed token's element is
// written again by the thread that wrote it, so that nobody waits for the row's stores.
// 8,192 bf16 rows x 151,936 with 64 listed tokens 1,014 us: 4.98 GB at 4.91 TB/s (a copy 5.15); 3,001 x 50,257 with 200 listed, 0.6 of the
// rows valid, 109 us; 512 fp32 rows x 1,024 6.5 us and the loss 1.8.  The other kernel reads a row twice, or once for the loss alone:
// 2,048 fp32 rows x 151,936 754 us, 3.73 GB at 4.95 TB/s; the loss of 8,192 bf16 rows 363.
#include "ais_internal.h"
#include "device_utils.h"

namespace ais {
namespace {

using namespace dev;

typedef unsigned long long u64;

// q as a fixed-point number: a token's is off by 2^-62 at most, which shows in the gradient only where p and q are below some 1e-14.
constexpr int kQBits = 62;
constexpr float kLowest = -3.4028235e38f;

// What a row's listed tokens need of LDS: `slots` (a power of two >= 2 n_top) of the table and n_top entries.
struct Listed {
  u64* mass;                           // [slots] sum of q of the token in the slot
  int* token;                          // [slots] or -1
  float* t;                            // [n_top] the teacher's logit; -inf where there is no entry
  float* z;                            // [n_top] the policy's
  int* next;                           // [n_top] next entry of the same thread's row elements, or -1
  int* slot;                           // [n_top] of an entry that stands for its token, else -1
  static size_t bytes(int n_top, int slots) { return (size_t)slots * 12 + (size_t)n_top * 16; }
  __device__ __forceinline__ Listed(unsigned char* lds, int n_top, int slots) {
    mass = reinterpret_cast<u64*>(lds);
    token = reinterpret_cast<int*>(mass + slots);
    t = reinterpret_cast<float*>(token + slots);
    z = t + n_top;
    next = reinterpret_cast<int*>(z + n_top);
    slot = next + n_top;
  }
};

// A largest logit, as it is, and the sum of 2^((t - largest) c).  Lists are padded with numbers far below zero, whose products with c are
// rounded by more than an exponent holds: differences are taken before they are multiplied.
struct TopSum {
  float top, s;
};

template <int THREADS>
struct RowShared {
  TopSum teacher[THREADS / 64];
  MaxSum policy[THREADS / 64];
  double kl[THREADS / 64];
  int first[THREADS];                  // first entry of each thread's row elements, or -1
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
// The wavefronts' parts as one, in every lane: a few exchanges inside rows of 16 lanes.  (One after the other by every thread they
// took 2 us of the 30 that a compute unit spends on a row of 151,936 logits.)
template <int WAVES>
__device__ __forceinline__ MaxSum merge_all(const MaxSum* part) {
  MaxSum st = part[threadIdx.x & (WAVES - 1)];
  if constexpr (WAVES > 1) st = merge_dpp<kDppQuadXor1>(st);
  if constexpr (WAVES > 2) st = merge_dpp<kDppQuadXor2>(st);
  if constexpr (WAVES > 4) st = merge_dpp<kDppRowHalfMirror>(st);
  if constexpr (WAVES > 8) st = merge_dpp<kDppRowMirror>(st);
  return st;
}

template <int WAVES, typename Op>
__device__ __forceinline__ float fold_all(float v, Op op) {
  if constexpr (WAVES > 1) v = op(v, dpp_move<kDppQuadXor1>(v));
  if constexpr (WAVES > 2) v = op(v, dpp_move<kDppQuadXor2>(v));
  if constexpr (WAVES > 4) v = op(v, dpp_move<kDppRowHalfMirror>(v));
  if constexpr (WAVES > 8) v = op(v, dpp_move<kDppRowMirror>(v));
  return v;
}
template <int WAVES>
__device__ __forceinline__ TopSum join_all(const TopSum* part, float c) {
  const TopSum own = part[threadIdx.x & (WAVES - 1)];
  const float top = fold_all<WAVES>(own.top, [](float a, float b) { return fmaxf(a, b); });
  return {top, fold_all<WAVES>(own.s * exp2_fast((own.top - top) * c), [](float a, float b) { return a + b; })};
}

// The arguments of a row's kernels.
template <typename T>
struct DistillArgs {
  const T* logits;
  long long row_stride;
  int vocab;
  const int* ids;
  const float* teacher;
  int n_top, slots;
  const unsigned char* valid;
  const float* weight;
  float inv_rows, inv_temperature;
  double exact;                        // what the fp32 factor of the exponents is off by (see exact_exponents)
  float* kl;
  T* dlogits;
  long long dlogits_stride;
  int* status;
};

// The teacher's side of a row, in steps that its kernel places among its own.
template <typename T, int THREADS>
struct Teacher {
  const Listed listed;
  RowShared<THREADS>& sh;
  const DistillArgs<T>& a;
  const long long row;
  const float c;
  TopSum all;
  __device__ __forceinline__ Teacher(unsigned char* lds, RowShared<THREADS>& sh, const DistillArgs<T>& a, long long row)
      : listed(lds, a.n_top, a.slots), sh(sh), a(a), row(row), c(a.inv_temperature * kLog2e) {}
  __device__ __forceinline__ bool entry(int id) const { return id >= 0 && id < a.vocab; }

  // f(entry) of this thread's entries.  A thousand threads have one each, and no loop: what is asked for from memory inside one
  // would be waited for together with everything on its way, the whole row.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if constexpr (THREADS >= 1024) {
      if ((int)threadIdx.x < a.n_top) f((int)threadIdx.x);
    } else {
      for (int j = threadIdx.x; j < a.n_top; j += THREADS) f(j);
    }
  }
  // The thread's first entry, further ones when they are needed.
  int id0 = -1;
  float t0 = kMasked;
  T z0{};
  bool bad = false;                    // an id that is neither of the vocabulary nor -1
  // Asks for the first entry.  Neither this nor the loads of the policy's logits branch: where paths with and without a load
  // meet, the compiler waits for everything on its way, the whole row.
  __device__ __forceinline__ void fetch() {
    const long long at = row * a.n_top + min((int)threadIdx.x, a.n_top - 1);
    id0 = a.ids[at];
    t0 = a.teacher[at];
  }
  __device__ __forceinline__ bool first(int j) const { return THREADS >= 1024 || j < THREADS; }
  __device__ __forceinline__ int id(int j) const {
    if (first(j)) return id0;
    return a.ids[row * a.n_top + j];
  }

  // Entries to LDS, their sum to the workgroup; empties the table.  No barrier.
  __device__ __forceinline__ void read() {
    const int tid = threadIdx.x;
    TopSum st{kLowest, 0.f};                           // finite also where there is no entry
    each([&](int j) {
      float t = t0;
      if (!first(j)) t = a.teacher[row * a.n_top + j];
      const int token = id(j);
      if (!entry(token)) {
        t = kMasked;
        bad = bad || token != -1;
      }
      st.top = fmaxf(st.top, t);
      listed.t[j] = t;
    });
    st.top = wave_max(st.top);
    each([&](int j) { st.s += exp2_fast((listed.t[j] - st.top) * c); });
    st.s = wave_sum(st.s);
    for (int s = tid; s < a.slots; s += THREADS) {
      listed.token[s] = -1;
      listed.mass[s] = 0;
    }
    sh.first[tid] = -1;
    if ((tid & 63) == 0) sh.teacher[tid >> 6] = st;
  }
  // After a barrier: whether there is anything to learn from.
  __device__ __forceinline__ bool any() {
    all = join_all<THREADS / 64>(sh.teacher, c);
    return all.s != 0.f;
  }
  // q of an entry: NaN, all of them, where the teacher has a NaN or +inf
  __device__ __forceinline__ float q(int j) const { return exp2_fast((listed.t[j] - all.top) * c) / all.s; }
  __device__ __forceinline__ bool fine() const { return all.s < 3.0e38f; }
  // Entries into the table, their logits asked for.  An entry that stands for its token is put on the list of the thread that
  // `owner` names.  No barrier.
  template <typename F>
  __device__ __forceinline__ void insert(const T* zr, F owner) {
    z0 = zr[entry(id0) ? id0 : 0];
    each([&](int j) {
      const int token = id(j);
      int slot = -1;
      if (entry(token)) {
        if (!first(j)) listed.z[j] = Vec<T>::load1(zr + token);
        int s = (int)(((uint32_t)token * 2654435761u) >> 16) & (a.slots - 1);
        while (true) {                                 // the table has twice as many slots as there are entries
          const int held = atomicCAS(&listed.token[s], -1, token);
          if (held == -1) slot = s;
          if (held == -1 || held == token) break;
          s = (s + 1) & (a.slots - 1);
        }
        atomicAdd(&listed.mass[s], (u64)ldexp((double)(fine() ? q(j) : 0.f), kQBits));
        if (slot >= 0) listed.next[j] = atomicExch(&sh.first[owner(token)], j);
      }
      listed.slot[j] = slot;
    });
  }
  // The first entry's logit, once it is there.  No barrier.
  __device__ __forceinline__ void keep() {
    if ((int)threadIdx.x < a.n_top) listed.z[threadIdx.x] = Vec<T>::load1(&z0);
  }
  // log q - log p of every entry, weighted by q, with q = 2^((t - all.top) c) / all.s and p = 2^(z c - st.m) / st.s.  To the
  // workgroup; no barrier.  Wavefronts without entries have nothing to do with it.
  __device__ __forceinline__ void diverge(MaxSum st) {
    const int tid = threadIdx.x;
    double kl = 0.0;
    if ((tid & ~63) < a.n_top) {
      const double log_ratio = log((double)all.s) - log((double)st.s), ln2 = 0.6931471805599453 * a.exact;
      each([&](int j) {
        const float p = q(j);
        if (p <= 0.f) return;
        const double t2 = ((double)listed.t[j] - (double)all.top) * (double)c, z2 = (double)listed.z[j] * (double)c - (double)st.m;
        kl += (double)p * ((t2 - z2) * ln2 - log_ratio);
      });
      kl = wave_sum64(kl);
    }
    if ((tid & 63) == 0) sh.kl[tid >> 6] = kl;
  }
  // After a barrier.
  __device__ __forceinline__ void report() const {
    if (bad) atomicOr(a.status, AIS_STATUS_BAD_TOKEN);
    if (threadIdx.x != 0) return;
    double kl = sh.kl[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) kl += sh.kl[w];
    a.kl[row] = (float)kl;
  }
  // Element of the gradient of an entry's token, less the factor g.
  __device__ __forceinline__ float element(int j, MaxSum st) const {
    const float sum = fine() ? (float)ldexp((double)listed.mass[listed.slot[j]], -kQBits) : __builtin_nanf("");
    return exp2_fast(__builtin_fmaf(listed.z[j], c, -st.m)) / st.s - sum;
  }
  __device__ __forceinline__ float weight() const {
    return (a.weight == nullptr ? a.inv_rows : a.weight[row]) * a.inv_temperature;
  }
};

// Products with c far from zero are rounded to whole numbers or do not fit.  Where the largest logit's is, or where a thread that has
// nothing but the type's lowest value has made the sum something else than a number: the largest logit and the sum relative to it, from
// memory.  False without a finite largest one.
template <typename T, int THREADS>
__device__ __forceinline__ bool recentre(const T* zr, int vocab, float c, RowShared<THREADS>& sh, float* top, float* sum) {
  const int tid = fresh_thread();
  float m = -__builtin_inff(), s = 0.f;
#pragma unroll 1
  for (uint32_t v = tid; v < (uint32_t)vocab; v += THREADS) m = fmaxf(m, Vec<T>::load1(zr + v));
  m = wave_max(m);
  __syncthreads();
  if ((tid & 63) == 0) sh.policy[tid >> 6].m = m;
  __syncthreads();
  for (int w = 0; w < THREADS / 64; ++w) m = fmaxf(m, sh.policy[w].m);
  if (!(fabsf(m) <= 3.4028235e38f)) return false;
#pragma unroll 1
  for (uint32_t v = tid; v < (uint32_t)vocab; v += THREADS) s += exp2_fast((Vec<T>::load1(zr + v) - m) * c);
  s = wave_sum(s);
  if ((tid & 63) == 0) sh.policy[tid >> 6].s = s;
  __syncthreads();
  s = 0.f;
  for (int w = 0; w < THREADS / 64; ++w) s += sh.policy[w].s;
  *top = m;
  *sum = s;
  return true;
}
constexpr float kFar = 1e9f;           // of a product with c

// ---- rows that are read twice: any width and alignment, and the loss alone ----------------------------------------------------
constexpr int kTwiceThreads = 256;

// A thread sums up to some thousand terms of a row.  Beside a large one small ones would be lost: up to 32 are summed in pairs, pairs of
// pairs and so on, and their sums in fp64, which costs nothing beside the reading.  (In fp32 alone the divergence of rows of 260,000
// logits was 18 x 2^-24 off, root mean square, and up to 37 x 2^-24.)
struct WideSum {
  float m;
  double s;
};
template <int n>
__device__ __forceinline__ void accumulate_wide(const float* x, float scale, WideSum& st) {
  float most = x[0];
#pragma unroll
  for (int k = 1; k < n; ++k) most = fmaxf(most, x[k]);
  const float m = fmaxf(st.m, most * scale);
  float e[n];
#pragma unroll
  for (int k = 0; k < n; ++k) e[k] = exp2_fast(__builtin_fmaf(x[k], scale, -m));
#pragma unroll
  for (int d = n / 2; d > 0; d /= 2)
#pragma unroll
    for (int k = 0; k < d; ++k) e[k] += e[k + d];
  st.s = st.s * (double)exp2_fast(st.m - m) + (double)e[0];
  st.m = m;
}

template <typename T>
__global__ __launch_bounds__(kTwiceThreads) void distill_twice_kernel(const DistillArgs<T> a) {
  constexpr int N = Vec<T>::N, kAhead = 4;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ RowShared<kTwiceThreads> sh;
  const long long row = blockIdx.x;
  const int tid = threadIdx.x, vocab = a.vocab;
  const T* zr = a.logits + row * a.row_stride;
  T* dr = a.dlogits == nullptr ? nullptr : a.dlogits + row * a.dlogits_stride;
  Teacher<T, kTwiceThreads> teacher(lds, sh, a, row);
  auto nothing = [&] {                                 // nothing to learn from: no loss, no gradient
    if (tid == 0) a.kl[row] = 0.f;
    if (dr != nullptr)
      for (uint32_t v = tid; v < (uint32_t)vocab; v += kTwiceThreads) Vec<T>::store1(dr + v, 0.f);
  };
  if (a.valid != nullptr && a.valid[row] == 0) {
    nothing();
    return;
  }
  teacher.fetch();
  teacher.read();
  __syncthreads();
  if (!teacher.any()) {
    if (teacher.bad) atomicOr(a.status, AIS_STATUS_BAD_TOKEN);
    nothing();
    return;
  }
  teacher.insert(zr, [](int) { return 0; });
  // where the gradient lies has no say in the order of the sums
  const int head = (reinterpret_cast<uintptr_t>(zr) & 15) == 0 ? 0 : head_elements(zr, vocab);
  const int nvec = (vocab - head) / N, rest = vocab - nvec * N;
  const u32x4* zv = reinterpret_cast<const u32x4*>(zr + head);
  const float c = teacher.c;
  WideSum own{kNegHuge, 0.0};
  int i = tid;
  for (; i + (kAhead - 1) * kTwiceThreads < nvec; i += kAhead * kTwiceThreads) {
    u32x4 q[kAhead];
    float x[kAhead * N];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) q[u] = load_stream(zv + i + u * kTwiceThreads);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) Vec<T>::unpack(q[u], x + u * N);
    accumulate_wide<kAhead * N>(x, c, own);
  }
  for (; i < nvec; i += kTwiceThreads) {
    float x[N];
    Vec<T>::unpack(load_stream(zv + i), x);
    accumulate_wide<N>(x, c, own);
  }
  for (int r = tid; r < rest; r += kTwiceThreads) {
    const float x = Vec<T>::load1(zr + (r < head ? r : nvec * N + r));
    accumulate_wide<1>(&x, c, own);
  }
  MaxSum st = wave_merge(MaxSum{own.m, (float)own.s});
  if ((tid & 63) == 0) sh.policy[tid >> 6] = st;
  teacher.keep();
  __syncthreads();
  st = merge_all<kTwiceThreads / 64>(sh.policy);
  float origin = 0.f;                                  // that is taken from the logits
  if (!(fabsf(st.m) < kFar) || !(st.s < 3e38f)) {
    float top, sum;
    if (recentre(zr, vocab, c, sh, &top, &sum)) {
      origin = top;
      st = MaxSum{0.f, sum};
      for (int j = tid; j < a.n_top; j += kTwiceThreads) teacher.listed.z[j] -= top;
      __syncthreads();
    }
  }
  teacher.diverge(st);
  __syncthreads();
  teacher.report();
  if (dr == nullptr) return;
  const float g = teacher.weight(), g_p = g / st.s;
  const bool aligned = (reinterpret_cast<uintptr_t>(dr + head) & 15) == 0;
  for (i = tid; i < nvec; i += kTwiceThreads) {
    float x[N];
    Vec<T>::unpack(zv[i], x);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = exp2_fast(__builtin_fmaf(x[j] - origin, c, -st.m)) * g_p;
    T* d = dr + head + (long long)i * N;
    if (aligned) {
      *reinterpret_cast<u32x4*>(d) = Vec<T>::pack(x);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) Vec<T>::store1(d + j, x[j]);
    }
  }
  for (int r = tid; r < rest; r += kTwiceThreads) {
    const int v = r < head ? r : nvec * N + r;
    Vec<T>::store1(dr + v, exp2_fast(__builtin_fmaf(Vec<T>::load1(zr + v) - origin, c, -st.m)) * g_p);
  }
  // the listed tokens' elements, once every wavefront's stores have completed
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int j = tid; j < a.n_top; j += kTwiceThreads)
    if (teacher.listed.slot[j] >= 0)
      Vec<T>::store1(dr + teacher.listed.token[teacher.listed.slot[j]], g * teacher.element(j, st));
}

// ---- rows that are held ---------------------------------------------------------------------------------------------------
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef const __attribute__((address_space(1))) void* glb_ptr;

// ALIGNED: both rows are 16-byte aligned; otherwise both lie the same way relative to 128-byte lines, and the elements before the
// row's first line boundary are handled one by one together with those after the last vector.  Vector k of a lane (vector tid +
// THREADS k of the row) lies in register q[k] for k < NV and in slot k - NV of the dynamic LDS for the NL after them; up to NR more,
// of the widest rows, are read again.  (Held in registers too they made those spill.)  The row has at least KFULL THREADS vectors.
template <typename T, bool ALIGNED, int THREADS, int NV, int NL, int NR, int KFULL>
__global__ __launch_bounds__(THREADS) void distill_held_kernel(const DistillArgs<T> a) {
  constexpr int N = Vec<T>::N;
  static_assert(ALIGNED || THREADS >= 128, "a thread for every element outside the vectors");
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ RowShared<THREADS> sh;
  u32x4* slots = reinterpret_cast<u32x4*>(lds);
  const long long row = blockIdx.x;
  const int tid = threadIdx.x, vocab = a.vocab;
  const T* zr = a.logits + row * a.row_stride;
  T* dr = a.dlogits + row * a.dlogits_stride;
  const int head = ALIGNED ? 0 : head_elements(zr, vocab);
  const int nvec = (vocab - head) / N, rest = vocab - nvec * N;
  const int v_rest = ALIGNED || tid >= head ? nvec * N + tid : tid;
  const u32x4* zv = reinterpret_cast<const u32x4*>(zr + head);
  u32x4* dv = reinterpret_cast<u32x4*>(dr + head);
  Teacher<T, THREADS> teacher(lds + NL * THREADS * 16, sh, a, row);

  auto nothing = [&] {                                 // nothing to learn from: no loss, no gradient
    if (tid == 0) a.kl[row] = 0.f;
    const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int k = 0; k < NV + NL + NR; ++k)
      if (tid + k * THREADS < nvec) store_stream(dv + tid + k * THREADS, zero);
    if (tid < rest) Vec<T>::store1(dr + v_rest, 0.f);
  };
  if (a.valid != nullptr && a.valid[row] == 0) {
    nothing();
    return;
  }
  // the teacher's entries, which are waited for first, and the whole row are asked for
  teacher.fetch();
  const float g = teacher.weight();
  u32x4 q[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = tid + k * THREADS;
    if (k < KFULL) q[k] = load_stream(zv + i);
    else q[k] = i < nvec ? load_stream(zv + i) : masked_fill<T>();
    __builtin_amdgcn_sched_barrier(0);                 // in the order in which they are summed
  }
  if (NL > 0) {
    int tid0 = tid;                                    // opaque copies keep the per-vector offsets short-lived
    asm volatile("" : "+v"(tid0));
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      // lanes past the end of the row fetch its last vector, which is masked later
      const int i = min(tid0 + (NV + k) * THREADS, nvec - 1);
      __builtin_amdgcn_global_load_lds((glb_ptr)(zv + i), (lds_ptr)(slots + k * THREADS + (tid0 & ~63)), 16, 0,
                                       2 /* non-temporal */);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  const T xt_raw = zr[min(v_rest, vocab - 1)];
  teacher.read();
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");        // without a wait for the row
  if (!teacher.any()) {
    if (teacher.bad) atomicOr(a.status, AIS_STATUS_BAD_TOKEN);
    nothing();
    if (NL > 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // copies into LDS that is about to be given back
    return;
  }
  // an element belongs to the thread that holds its vector, or that has it as its one element outside them
  teacher.insert(zr, [&](int id) {
    const int at = id - head;
    if (at >= 0 && at < nvec * N) return at / N % THREADS;
    return at < 0 ? id : id - nvec * N;
  });

  const float c = teacher.c;
  MaxSum st{kNegHuge, 0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float x[N];
    Vec<T>::unpack(q[k], x);
    accumulate<N>(x, c, st);
    __builtin_amdgcn_sched_barrier(0);                 // keeps the unpacked values of one vector short-lived
  }
  if (NL > 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the copies into the slots have landed
    int tid1 = tid;
    asm volatile("" : "+v"(tid1));
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      const int i = tid1 + (NV + k) * THREADS;
      float x[N];
      Vec<T>::unpack(slots[k * THREADS + tid1], x);
      if (NV + k >= KFULL) {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = i < nvec ? x[j] : kMasked;
      }
      accumulate<N>(x, c, st);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll 1
  for (int i = tid + (NV + NL) * THREADS; NR > 0 && i < nvec; i += THREADS) {
    float x[N];
    Vec<T>::unpack(zv[i], x);
    accumulate<N>(x, c, st);
  }
  const float xt = tid < rest ? Vec<T>::load1(&xt_raw) : kMasked;
  accumulate<1>(&xt, c, st);
  st = wave_merge(st);
  if ((tid & 63) == 0) sh.policy[tid >> 6] = st;
  teacher.keep();
  __syncthreads();
  st = merge_all<THREADS / 64>(sh.policy);
  if (!(fabsf(st.m) < kFar) || !(st.s < 3e38f)) {
    float top, sum;
    if (recentre(zr, vocab, c, sh, &top, &sum)) {
      st = MaxSum{0.f, sum};
      for (int j = tid; j < a.n_top; j += THREADS) teacher.listed.z[j] -= top;
#pragma unroll 1
      for (uint32_t v = tid; v < (uint32_t)vocab; v += THREADS)
        Vec<T>::store1(dr + v, exp2_fast((Vec<T>::load1(zr + v) - top) * c) * (g / sum));
      // the listed tokens' elements after them, whoever wrote those
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      for (int j = tid; j < a.n_top; j += THREADS)
        if (teacher.listed.slot[j] >= 0)
          Vec<T>::store1(dr + teacher.listed.token[teacher.listed.slot[j]], g * teacher.element(j, st));
      teacher.diverge(st);
      __syncthreads();
      teacher.report();
      return;
    }
  }
  const float g_p = g / st.s, shift = -st.m;
  // opaque until the sum is known: neither are unpacked values kept alive nor is the unpacking below moved up
#pragma unroll
  for (int k = 0; k < NV; ++k) asm volatile("" : "+v"(q[k]) : "v"(shift));
  int tid2 = tid;                                      // opaque: the vectors' offsets are not kept from the loads on
  asm volatile("" : "+v"(tid2));
#pragma unroll
  for (int k = 0; k < NV + NL; ++k) {
    const int i = tid2 + k * THREADS;
    float x[N];
    Vec<T>::unpack(k < NV ? q[k < NV ? k : 0] : slots[(k - NV) * THREADS + tid2], x);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = exp2_fast(__builtin_fmaf(x[j], c, shift)) * g_p;
    if (k < KFULL || i < nvec) store_stream(dv + i, Vec<T>::pack(x));
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll 1
  for (int i = tid2 + (NV + NL) * THREADS; NR > 0 && i < nvec; i += THREADS) {
    float x[N];
    Vec<T>::unpack(zv[i], x);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = exp2_fast(__builtin_fmaf(x[j], c, shift)) * g_p;
    store_stream(dv + i, Vec<T>::pack(x));
  }
  if (tid < rest) Vec<T>::store1(dr + v_rest, exp2_fast(__builtin_fmaf(xt, c, shift)) * g_p);
  // the listed tokens' elements among those that this thread has written: a thread's own stores to a place keep their order
  for (int j = sh.first[tid]; j >= 0; j = teacher.listed.next[j])
    Vec<T>::store1(dr + teacher.listed.token[teacher.listed.slot[j]], g * teacher.element(j, st));
  teacher.diverge(st);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");        // without a wait for the stores
  teacher.report();
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

constexpr int kMostVectors = 20;       // of a lane, in registers alone
constexpr int kMostSlots = 13;         // ... and in LDS beside them
constexpr int kLdsSlots = 9;           // 144 KiB of the 160
constexpr int kWide = 1024;
constexpr long long kMostRows = 1LL << 21;              // of a launch

template <typename T, bool ALIGNED, int THREADS, int NV, int NL, int NR, int KFULL>
int launch_held_as(ais_ctx* ctx, const DistillArgs<T>& a, long long n_rows, size_t listed_bytes) {
  auto kernel = distill_held_kernel<T, ALIGNED, THREADS, NV, NL, NR, KFULL>;
  const size_t bytes = (size_t)NL * THREADS * 16 + listed_bytes;
  if (NL > 0) {
    static std::once_flag once[kMaxDevices];           // the attribute belongs to the function on one device
    static bool ok[kMaxDevices];
    if (!allow_dynamic_lds(ctx, reinterpret_cast<const void*>(kernel), 160 * 1024 - (int)sizeof(RowShared<THREADS>), once, ok))
      return hip_fail(ctx, hipErrorInvalidValue);
  }
  kernel<<<dim3((unsigned)n_rows), dim3(THREADS), bytes, ctx->stream>>>(a);
  return hip_fail(ctx, hipGetLastError());
}

template <typename T, bool ALIGNED>
int launch_held(ais_ctx* ctx, const DistillArgs<T>& a, long long n_rows, size_t listed_bytes) {
  const int nvec = a.vocab / Vec<T>::N, need = (nvec + kWide - 1) / kWide;
  // NV is a compile-time constant (the row lives in named registers).  Up to 8,192 vectors two rows or more share a compute unit, so
  // that one is read or written while another is summed: with 1,024 threads and with 512, us, 3,001 rows x 50,257 bf16 166 and
  // 121, 8,000 x 32,000 301 and 184, 3,000 x 64,000 184 and 142; with 256 and 512, 20,000 x 8,000 fp32 249 and 235.  PREV: the widest row of the class before; a row that
  // reaches this one has more than PREV * 1024 vectors, of which an unaligned row may have lost up to 8 to its head.
#define AIS_HELD(THREADS, PREV, NVAL, NLVAL, NRVAL) \
  return launch_held_as<T, ALIGNED, THREADS, NVAL, NLVAL, NRVAL, (ALIGNED || PREV == 0 ? PREV : PREV - 1)>(ctx, a, n_rows, listed_bytes)
  if constexpr (ALIGNED) {
    if (nvec <= 256) AIS_HELD(64, 0, 4, 0, 0);
  }
  if (nvec <= 512) AIS_HELD(128, 0, 4, 0, 0);
  if (nvec <= 1024) AIS_HELD(256, 0, 4, 0, 0);
  if (nvec <= 2048) AIS_HELD(512, 0, 4, 0, 0);
  if (nvec <= 4096) AIS_HELD(512, 0, 8, 0, 0);
  if (nvec <= 6144) AIS_HELD(512, 0, 12, 0, 0);
  if (nvec <= 7168) AIS_HELD(512, 0, 14, 0, 0);
  if (nvec <= 8192) AIS_HELD(512, 0, 16, 0, 0);
  if (need <= 12) AIS_HELD(kWide, 8, 12, 0, 0);
  if (need <= 16) AIS_HELD(kWide, 12, 16, 0, 0);
  if (need <= 18) AIS_HELD(kWide, 16, 18, 0, 0);
  if (need <= 19) AIS_HELD(kWide, 18, 19, 0, 0);
  if (need <= 20) AIS_HELD(kWide, 19, 20, 0, 0);
  if (need <= 23) AIS_HELD(kWide, 20, 18, 5, 0);
  if (need <= 27) AIS_HELD(kWide, 23, 18, kLdsSlots, 0);
  if (need <= 29) AIS_HELD(kWide, 27, 20, kLdsSlots, 0);
  if (need <= 31) AIS_HELD(kWide, 29, 21, kLdsSlots, 1);
  AIS_HELD(kWide, 31, 21, kLdsSlots, 3);
#undef AIS_HELD
}

// Whether a row can be held: its width, and both arrays lie the same way relative to 128-byte lines.
template <typename T>
bool can_be_held(const DistillArgs<T>& a, size_t listed_bytes, bool* aligned) {
  if (a.dlogits == nullptr || a.dlogits_stride != a.row_stride) return false;
  const uintptr_t z = reinterpret_cast<uintptr_t>(a.logits), d = reinterpret_cast<uintptr_t>(a.dlogits);
  *aligned = z % 16 == 0 && d % 16 == 0 && a.row_stride * (long long)sizeof(T) % 16 == 0;
  if (!*aligned && (z - d) % 128 != 0) return false;
  const int need = (a.vocab / Vec<T>::N + kWide - 1) / kWide;
  if (need <= kMostVectors) return true;
  return need <= kMostVectors + kMostSlots &&
         (size_t)kLdsSlots * kWide * 16 + listed_bytes + sizeof(RowShared<kWide>) <= 160 * 1024;
}

template <typename T>
int launch_rows(ais_ctx* ctx, const DistillArgs<T>& a, long long n_rows) {
  const size_t listed_bytes = Listed::bytes(a.n_top, a.slots);
  bool aligned = false;
  if (can_be_held(a, listed_bytes, &aligned))
    return aligned ? launch_held<T, true>(ctx, a, n_rows, listed_bytes) : launch_held<T, false>(ctx, a, n_rows, listed_bytes);
  distill_twice_kernel<T><<<dim3((unsigned)n_rows), dim3(kTwiceThreads), listed_bytes, ctx->stream>>>(a);
  return hip_fail(ctx, hipGetLastError());
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
      // no more than 2^31 threads to a launch
      for (long long r = 0; r < n_rows; r += kMostRows) {
        const DistillArgs<T> args{static_cast<const T*>(logits) + r * row_stride,
                                  row_stride,
                                  vocab,
                                  ids + r * n_top,
                                  teacher + r * n_top,
                                  n_top,
                                  slots,
                                  valid != nullptr ? valid + r : nullptr,
                                  weight != nullptr ? weight + r : nullptr,
                                  inv_rows,
                                  inv_temperature,
                                  exact_exponents(inv_temperature),
                                  kl_out + r,
                                  dlogits != nullptr ? static_cast<T*>(dlogits) + r * dlogits_stride : nullptr,
                                  dlogits_stride,
                                  ctx->status_dev};
        const int rc = launch_rows(ctx, args, n_rows - r < kMostRows ? n_rows - r : kMostRows);
        if (rc != AIS_OK) return rc;
      }
      return (int)AIS_OK;
    };
    const int rc = dtype == AIS_BF16 ? run(bf16_t{}) : run(float{});
    if (rc != AIS_OK) return rc;
  }
  distill_loss_kernel<<<dim3(1), dim3(kLossThreads), 0, ctx->stream>>>(kl_out, weight, valid, n_rows, inv_rows, loss_out);
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
