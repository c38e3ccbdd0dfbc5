// Preference loss over pairs of responses: sums of log-ratios over whole responses, a loss of each pair, a coefficient of each row.
//
//   d_i = sum over i's valid rows of logp - ref (or their mean), h = beta (d_2p - d_2p+1) - margin, loss = sum_p w_p l(h_p)
//   c_t = -d loss / d logp_t = -+ w_p l'(h_p) beta [/ |o_i|]
//
// Three launches: partial sums of tiles of rows, pairs, rows; small batches are one workgroup's, and through logits the gradient sweep's own
// (512 rows of 1,024 fp32 logits: 4.4 + 6.1 + 3.4 us with a launch for them, 4.4 + 5.8 without).  Reading 9 and writing 4 bytes a row is
// nothing beside the launches: 1.2 million rows in 4,000 responses take 6.0, 3.6 and 4.9 us, which is how long a workgroup's own chain of
// loads, scan and stores is, all of them being there at once.  All that a thread needs of its rows is therefore loaded at once, masked rows
// included, and eight rows lie in registers for the scan and the walk after it (11.2, 4.7 and 11.0 us with loads one after the other).
#include "ais_internal.h"
#include "eights.h"
#include "preference.h"

namespace ais {
namespace {

using namespace dev;

constexpr int kRowsOfThread = 8;
// A workgroup's tile of rows where there are many; where one workgroup can take them all, it does.
constexpr int kTileThreads = 256, kOneThreads = 1024;
constexpr int kTileRows = kRowsOfThread * kTileThreads, kOneRows = kRowsOfThread * kOneThreads;
constexpr int kOneResponses = 1024;

// The last response that begins at `row` or before it (cu_rows non-decreasing), by a wavefront: each step looks at 64 places.
__device__ __forceinline__ int response_at(const long long* __restrict__ cu, int n_resp, long long row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = n_resp;                        // it is one of lo .. lo + n - 1, or lo where all of them begin later
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int at = lo + lane * step;
    const bool before = lane * step < n && cu[at] <= row;
    const unsigned long long mask = __ballot(before);
    const int last = mask == 0 ? 0 : 63 - __builtin_clzll(mask);
    lo += last * step;
    n = min(step, n - last * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// What precedes a row in its response, inside the tile.
struct Run {
  double sum;
  int count, owner;      // owner: 1 + the response that began last, 0 where none has
};
__device__ __forceinline__ Run join(Run a, Run b) {
  return b.owner != 0 ? b : Run{a.sum + b.sum, a.count + b.count, a.owner};
}

struct Owner {
  float coeff;
  long long lo, hi;
};

// Eight rows of a thread: log-ratios, 0 in rows that do not count, and which of them do.
struct Rows {
  double x[kRowsOfThread];
  unsigned live;
  __device__ __forceinline__ void load(const Preference& in, long long r, int here) {
    typedef u32x2 __attribute__((aligned(1))) Bytes;
    float lp[kRowsOfThread] = {}, rf[kRowsOfThread] = {};
    live = 0;
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) x[k] = 0.0;
    if (here <= 0) return;
    // all loads at once: masked rows are loaded and dropped
    if (here == kRowsOfThread) {
      u32x2 v = {0x01010101u, 0x01010101u};
      if (in.valid != nullptr) v = *reinterpret_cast<const Bytes*>(in.valid + r);
      if (in.ref != nullptr) Eight<float>::unpack(Eight<float>::load_kept(in.ref + r), rf);
      if (in.fine != nullptr) {
#pragma unroll
        for (int k = 0; k < kRowsOfThread; ++k) x[k] = in.fine[r + k];
      } else {
        Eight<float>::unpack(Eight<float>::load_kept(in.logp + r), lp);
      }
#pragma unroll
      for (int k = 0; k < kRowsOfThread; ++k) live |= ((v[k >> 2] >> (8 * (k & 3)) & 255u) != 0 ? 1u : 0u) << k;
    } else {
#pragma unroll
      for (int k = 0; k < kRowsOfThread; ++k) {
        if (k >= here) break;
        if (in.valid == nullptr || in.valid[r + k] != 0) live |= 1u << k;
        if (in.fine != nullptr) x[k] = in.fine[r + k];
        else lp[k] = in.logp[r + k];
        if (in.ref != nullptr) rf[k] = in.ref[r + k];
      }
    }
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k)
      x[k] = live >> k & 1 ? (in.fine != nullptr ? x[k] : (double)lp[k]) - (double)rf[k] : 0.0;
  }
};

// A tile of rows from r0 on: which response each row belongs to, as marks where responses begin.
template <int THREADS>
struct Tile {
  static constexpr int kRows = kRowsOfThread * THREADS;
  alignas(16) int begins[kRows];                 // 1 + response, 0
  Run waves[THREADS / 64];

  // The marks of a thread's rows; there are none past the end.
  __device__ __forceinline__ void marks(int* o) const {
    const int4 a = reinterpret_cast<const int4*>(begins)[2 * threadIdx.x], b = reinterpret_cast<const int4*>(begins)[2 * threadIdx.x + 1];
    o[0] = a.x, o[1] = a.y, o[2] = a.z, o[3] = a.w;
    o[4] = b.x, o[5] = b.y, o[6] = b.z, o[7] = b.w;
  }

  __device__ __forceinline__ void clear() {
    reinterpret_cast<int4*>(begins)[threadIdx.x] = int4{0, 0, 0, 0};
    reinterpret_cast<int4*>(begins)[threadIdx.x + THREADS] = int4{0, 0, 0, 0};
  }
  // Response i begins in row `at` of the tile; of several that begin there all but the last are empty.
  __device__ __forceinline__ void mark(int i, long long at, int rows) {
    if (at >= 0 && at < rows) atomicMax(&begins[at], i + 1);
  }

  // Partial sums: a segmented scan over the tile's rows, eight to a thread.  `first`: the response that row 0 belongs to; leave(i,
  // sum, count) is called once for every response with a row here.
  template <typename Leave>
  __device__ __forceinline__ void sum(const Rows& mine, int first, int rows, Leave leave) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int at = kRowsOfThread * tid;
    int o[kRowsOfThread];
    marks(o);
    Run scan{0.0, 0, 0};
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) {
      if (o[k] != 0) scan = Run{0.0, 0, o[k]};
      scan.sum += mine.x[k];
      scan.count += mine.live >> k & 1;
    }
    // what lies before this thread's rows
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const Run before{__shfl_up(scan.sum, off), __shfl_up(scan.count, off), __shfl_up(scan.owner, off)};
      if (lane >= off) scan = join(before, scan);
    }
    if (lane == 63) waves[wave] = scan;
    __syncthreads();
    Run run{__shfl_up(scan.sum, 1), __shfl_up(scan.count, 1), __shfl_up(scan.owner, 1)};
    if (lane == 0) run = Run{0.0, 0, 0};
    Run ahead{0.0, 0, first + 1};
    for (int w = 0; w < wave; ++w) ahead = join(ahead, waves[w]);
    run = join(ahead, run);
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) {
      if (o[k] != 0) {
        if (at + k > 0) leave(run.owner - 1, run.sum, run.count);
        run = Run{0.0, 0, o[k]};
      }
      run.sum += mine.x[k];
      run.count += mine.live >> k & 1;
    }
    if (at < rows && at + kRowsOfThread >= rows) leave(run.owner - 1, run.sum, run.count);
  }

  // Coefficients of the rows from r0 on, whose responses have been marked; of(i): response i's coefficient and rows.
  template <typename Of>
  __device__ __forceinline__ void spread(const Preference& in, unsigned live, int first, long long r0, int rows, Of of) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int at = kRowsOfThread * tid, here = min(max(rows - at, 0), kRowsOfThread);
    int o[kRowsOfThread];
    marks(o);
    // owners grow along the tile where the offsets do: the last mark is the largest so far
    int own = 0;
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) own = max(own, o[k]);
    int scan = own;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int before = __shfl_up(scan, off);
      if (lane >= off) scan = max(scan, before);
    }
    if (lane == 63) waves[wave].owner = scan;
    __syncthreads();
    own = __shfl_up(scan, 1);
    if (lane == 0) own = 0;
    own = max(own, first + 1);
    for (int w = 0; w < wave; ++w) own = max(own, waves[w].owner);
    Owner owner = of(own - 1);
    float g[kRowsOfThread];
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) {
      if (o[k] > own) {
        own = o[k];
        owner = of(own - 1);
      }
      const long long r = r0 + at + k;
      g[k] = (live >> k & 1) != 0 && owner.lo <= r && r < owner.hi ? owner.coeff * in.scale : 0.f;
    }
    if (here == kRowsOfThread) Eight<float>::store(in.g + r0 + at, g);
    else if (here > 0) store_some(in.g + r0 + at, here, g);
  }
};

__device__ __forceinline__ unsigned live_rows(const Preference& in, long long r, int here) {
  typedef u32x2 __attribute__((aligned(1))) Bytes;
  if (here <= 0) return 0;
  if (in.valid == nullptr) return 255u;
  unsigned live = 0;
  if (here == kRowsOfThread) {
    const u32x2 v = *reinterpret_cast<const Bytes*>(in.valid + r);
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) live |= ((v[k >> 2] >> (8 * (k & 3)) & 255u) != 0 ? 1u : 0u) << k;
  } else {
    for (int k = 0; k < here; ++k) live |= (in.valid[r + k] != 0 ? 1u : 0u) << k;
  }
  return live;
}

// The sum of a workgroup's values, by its first thread, in the order of the wavefronts.
template <int THREADS>
__device__ __forceinline__ void add_up(double s, float* out) {
  __shared__ double waves[THREADS / 64];
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < THREADS / 64; ++w) s += waves[w];
  *out = (float)s;
}

__global__ __launch_bounds__(kTileThreads) void preference_sums_kernel(Preference in) {
  __shared__ Tile<kTileThreads> tile;
  __shared__ int range[2];
  const int tid = threadIdx.x, b = blockIdx.x;
  const long long r0 = (long long)b * kTileRows;
  const int rows = (int)min((long long)kTileRows, in.n_rows - r0);
  Rows mine;
  mine.load(in, r0 + kRowsOfThread * tid, min(max(rows - kRowsOfThread * tid, 0), kRowsOfThread));
  tile.clear();
  // two wavefronts look for the tile's first and last response
  if (tid < 128) {
    const int i = response_at(in.cu, in.n_resp, tid < 64 ? r0 : r0 + rows - 1);
    if ((tid & 63) == 0) range[tid >> 6] = i;
    if (tid == 0) in.firsts[b] = i;
  }
  __syncthreads();
  const int first = range[0];
  for (int i = first + 1 + tid; i <= range[1]; i += kTileThreads) tile.mark(i, in.cu[i] - r0, rows);
  __syncthreads();
  tile.sum(mine, first, rows, [&](int i, double sum, int count) {
    in.sums[(size_t)i + b] = sum;
    in.counts[(size_t)i + b] = count;
  });
}

// A thread to a pair.
__global__ __launch_bounds__(kTileThreads) void preference_pairs_kernel(Preference in) {
  const int pair = blockIdx.x * kTileThreads + threadIdx.x;
  if (2 * pair >= in.n_resp) return;
  const long long cu[3] = {in.cu[2 * pair], in.cu[2 * pair + 1], in.cu[2 * pair + 2]};
  double s[2] = {};
  int n[2] = {};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const RowRange r = rows_of(in, 2 * pair + j, cu[j], cu[j + 1]);
    if (!r.sound) atomicOr(in.status, AIS_STATUS_BAD_CU);
    if (r.hi > r.lo)
      for (unsigned b = r.lo / kTileRows; b <= (r.hi - 1) / kTileRows; ++b) {
        s[j] += in.sums[2 * pair + j + (size_t)b];
        n[j] += in.counts[2 * pair + j + (size_t)b];
      }
  }
  const PairTerm t = pair_term<true>(in, pair, s, n);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    in.reward[2 * pair + j] = t.reward[j];
    in.coeff[2 * pair + j] = t.coeff[j];
  }
  in.loss[pair] = t.loss;
}

// A workgroup to a tile; one more adds up the pairs' losses.
__global__ __launch_bounds__(kTileThreads) void preference_rows_kernel(Preference in, int tiles) {
  __shared__ Tile<kTileThreads> tile;
  const int tid = threadIdx.x, b = blockIdx.x;
  if (b == tiles) {
    double s = 0.0;
    for (int p = tid; p < in.n_resp / 2; p += kTileThreads) s += in.loss[p];
    add_up<kTileThreads>(s, in.loss_out);
    return;
  }
  const long long r0 = (long long)b * kTileRows;
  const int rows = (int)min((long long)kTileRows, in.n_rows - r0);
  const unsigned live = live_rows(in, r0 + kRowsOfThread * tid, min(max(rows - kRowsOfThread * tid, 0), kRowsOfThread));
  const int first = in.firsts[b], last = b + 1 < tiles ? in.firsts[b + 1] : in.n_resp - 1;
  tile.clear();
  __syncthreads();
  for (int i = first + 1 + tid; i <= last; i += kTileThreads) tile.mark(i, in.cu[i] - r0, rows);
  __syncthreads();
  tile.spread(in, live, first, r0, rows, [&](int i) { return Owner{in.coeff[i], in.cu[i], in.cu[i + 1]}; });
}

// All of it in one workgroup, with the responses' offsets, sums and coefficients in LDS.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void preference_one_kernel(Preference in) {
  __shared__ Tile<THREADS> tile;
  __shared__ long long cu[kOneResponses + 1];
  __shared__ double sums[kOneResponses];
  __shared__ int counts[kOneResponses];
  __shared__ float coeff[kOneResponses];
  __shared__ int first;
  const int tid = threadIdx.x, rows = (int)in.n_rows;
  Rows mine;
  mine.load(in, kRowsOfThread * tid, min(max(rows - kRowsOfThread * tid, 0), kRowsOfThread));
  for (int i = tid; i <= in.n_resp; i += THREADS) cu[i] = in.cu[i];
  tile.clear();
  if (tid == 0) first = 0;
  __syncthreads();
  for (int i = tid; i < in.n_resp; i += THREADS) {
    sums[i] = 0.0;
    counts[i] = 0;
    tile.mark(i, cu[i], rows);
    if (cu[i] <= 0) atomicMax(&first, i);
  }
  __syncthreads();
  tile.sum(mine, first, rows, [&](int i, double sum, int count) {
    sums[i] = sum;
    counts[i] = count;
  });
  __syncthreads();
  double s = 0.0;
  for (int pair = tid; pair < in.n_resp / 2; pair += THREADS) {
    const PairTerm t = pair_term<true>(in, pair, sums + 2 * pair, counts + 2 * pair);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (!rows_of(in, 2 * pair + j, cu[2 * pair + j], cu[2 * pair + j + 1]).sound) atomicOr(in.status, AIS_STATUS_BAD_CU);
      in.reward[2 * pair + j] = t.reward[j];
      coeff[2 * pair + j] = t.coeff[j];
    }
    s += t.loss;
  }
  __syncthreads();
  tile.spread(in, mine.live, first, 0, rows, [&](int i) { return Owner{coeff[i], cu[i], cu[i + 1]}; });
  add_up<THREADS>(s, in.loss_out);
}

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

PreferenceRoom preference_room(long long n_rows, int n_resp, bool through_logits) {
  const size_t places = (size_t)n_resp + (size_t)((n_rows + kTileRows - 1) / kTileRows);
  PreferenceRoom r;
  r.counts = padded(8 * places);
  r.loss = r.counts + padded(4 * places);
  r.coeff = r.loss + padded(4 * (size_t)n_resp);
  r.firsts = r.coeff + padded(4 * (size_t)n_resp);
  r.g = r.firsts + padded(4 * places);
  r.lse = r.g + padded(4 * (size_t)n_rows);
  r.fine = r.lse + padded(4 * (size_t)n_rows);
  r.total = through_logits ? r.fine + padded(8 * (size_t)n_rows) : r.g;
  return r;
}

Preference preference_batch(ais_ctx* ctx, const float* logp, const double* fine, const float* ref, const unsigned char* valid,
                            long long n_rows, const long long* cu_rows, int n_resp, const float* weight,
                            const ais_preference_params& p, const PreferenceRoom& room, float scale, float* reward, float* loss_out,
                            float* g) {
  char* ws = static_cast<char*>(ctx->ws);
  return {logp, fine, ref, valid, cu_rows, weight, n_resp, n_rows, p, scale, reinterpret_cast<double*>(ws),
          reinterpret_cast<int*>(ws + room.counts), reinterpret_cast<double*>(ws + room.loss), reinterpret_cast<float*>(ws + room.coeff),
          reinterpret_cast<int*>(ws + room.firsts), reward, loss_out, g, ctx->status_dev};
}

int launch_preference(ais_ctx* ctx, const Preference& in) {
  ScopedTimer timer(ctx, AIS_K_PREFERENCE);
  if (in.n_rows <= kOneRows && in.n_resp <= kOneResponses) {
    // 2,048 rows take 9.1 us with 1,024 threads and 6.1 with 256
    if (in.n_rows <= kTileRows) preference_one_kernel<kTileThreads><<<dim3(1), dim3(kTileThreads), 0, ctx->stream>>>(in);
    else if (in.n_rows <= 2 * kTileRows) preference_one_kernel<2 * kTileThreads><<<dim3(1), dim3(2 * kTileThreads), 0, ctx->stream>>>(in);
    else preference_one_kernel<kOneThreads><<<dim3(1), dim3(kOneThreads), 0, ctx->stream>>>(in);
    return hip_fail(ctx, hipGetLastError());
  }
  const int tiles = (int)((in.n_rows + kTileRows - 1) / kTileRows);
  if (tiles > 0) preference_sums_kernel<<<dim3((unsigned)tiles), dim3(kTileThreads), 0, ctx->stream>>>(in);
  preference_pairs_kernel<<<dim3((unsigned)((in.n_resp / 2 - 1) / kTileThreads + 1)), dim3(kTileThreads), 0, ctx->stream>>>(in);
  preference_rows_kernel<<<dim3((unsigned)tiles + 1), dim3(kTileThreads), 0, ctx->stream>>>(in, tiles);
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
