// Preference loss over pairs of responses: sums of log-ratios over whole responses, a loss of each pair, a coefficient of each row.
//
//   d_i = sum over i's valid rows of logp - ref (or their mean), h = beta (d_2p - d_2p+1) - margin, loss = sum_p w_p l(h_p)
//   c_t = -d loss / d logp_t = -+ w_p l'(h_p) beta [/ |o_i|]
//
// Three launches: partial sums of tiles of rows, pairs, rows.  Bound by launches and, over millions of rows, by reading 9 and
// writing 4 bytes a row.
#include "ais_internal.h"
#include "eights.h"

namespace ais {
namespace {

using namespace dev;

constexpr int kRowsOfThread = 8;
// A workgroup's tile of rows where there are many; where one workgroup can take them all, it does.
constexpr int kTileThreads = 256, kOneThreads = 1024;
constexpr int kTileRows = kRowsOfThread * kTileThreads, kOneRows = kRowsOfThread * kOneThreads;

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

// The batch, as the entry points take it.
struct Preference {
  const float* logp;
  const double* fine;                            // the log-probs in 64 bits, or null
  const float* ref;
  const unsigned char* valid;
  const long long* cu;
  const float* weight;
  int n_resp;
  long long n_rows;
  ais_preference_params p;
  float scale;                                   // of the rows' coefficients
  // in the workspace: partial sums and counts (response i in tile b has place i + b, which no other pair of them has), the
  // pairs' losses, the responses' coefficients
  double* sums;
  int* counts;
  double* loss;
  float* coeff;
  float *reward, *loss_out, *g;
  int* status;
};

// The tile of rows that begins at r0: which response each row belongs to, as marks where responses begin.
template <int THREADS>
struct Tile {
  static constexpr int kRows = kRowsOfThread * THREADS;
  int begins[kRows];                             // 1 + response, 0
  Run waves[THREADS / 64];
  int first;

  __device__ __forceinline__ void mark(const Preference& in, long long r0, long long r1) {
    for (int k = threadIdx.x; k < kRows; k += THREADS) begins[k] = 0;
    const int i0 = response_at(in.cu, in.n_resp, r0), i1 = response_at(in.cu, in.n_resp, r1 - 1);
    if (threadIdx.x == 0) first = i0;
    __syncthreads();
    for (int i = i0 + 1 + threadIdx.x; i <= i1; i += THREADS) {
      const long long at = in.cu[i] - r0;
      if (at >= 0 && at < r1 - r0) atomicMax(&begins[at], i + 1);      // of several that begin there all but the last are empty
    }
    __syncthreads();
  }

  // Partial sums of tile b, between r0 and r1: a segmented scan over the tile's rows, eight to a thread.
  __device__ __forceinline__ void sum(const Preference& in, int b, long long r0, long long r1) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int rows = (int)(r1 - r0);
    const int at = kRowsOfThread * tid, here = min(max(rows - at, 0), kRowsOfThread);
    double x[kRowsOfThread] = {};
    unsigned live = 0;
    if (here > 0) {
      const long long r = r0 + at;
#pragma unroll
      for (int k = 0; k < kRowsOfThread; ++k) live |= (k < here && (in.valid == nullptr || in.valid[r + k] != 0) ? 1u : 0u) << k;
#pragma unroll
      for (int k = 0; k < kRowsOfThread; ++k) {
        if ((live >> k & 1) == 0) continue;
        x[k] = in.fine != nullptr ? in.fine[r + k] : (double)in.logp[r + k];
        if (in.ref != nullptr) x[k] -= (double)in.ref[r + k];
      }
    }
    mark(in, r0, r1);
    Run mine{0.0, 0, 0};
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) {
      if (k >= here) break;
      const int o = begins[at + k];
      if (o != 0) mine = Run{0.0, 0, o};
      mine.sum += x[k];
      mine.count += live >> k & 1;
    }
    // what lies before this thread's rows
    Run scan = mine;
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
    auto leave = [&] {
      const size_t place = (size_t)(run.owner - 1) + b;
      in.sums[place] = run.sum;
      in.counts[place] = run.count;
    };
#pragma unroll
    for (int k = 0; k < kRowsOfThread; ++k) {
      if (k >= here) break;
      const int o = begins[at + k];
      if (o != 0) {
        if (at + k > 0) leave();
        run = Run{0.0, 0, o};
      }
      run.sum += x[k];
      run.count += live >> k & 1;
    }
    if (here > 0 && at + here == rows) leave();
  }

  // Coefficients of the rows between r0 and r1, whose responses have been marked.
  __device__ __forceinline__ void spread(const Preference& in, long long r0, long long r1) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int at = kRowsOfThread * tid, here = min(max((int)(r1 - r0) - at, 0), kRowsOfThread);
    // owners grow along the tile where the offsets do: the last mark is the largest so far
    int own = 0;
    for (int k = 0; k < here; ++k) own = max(own, begins[at + k]);
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
    for (int k = 0; k < here; ++k) {
      own = max(own, begins[at + k]);
      const long long r = r0 + at + k;
      const int i = own - 1;
      const bool mine = (in.valid == nullptr || in.valid[r] != 0) && in.cu[i] <= r && r < in.cu[i + 1];
      in.g[r] = mine ? in.coeff[i] * in.scale : 0.f;
    }
  }
};

// A pair's loss, rewards and coefficients from the partial sums of tiles of `tile_rows` rows.
__device__ __forceinline__ double pair_terms(const Preference& in, int pair, int tile_rows) {
  const ais_preference_params& p = in.p;
  double d[2], share[2];
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = 2 * pair + j;
    const long long from = in.cu[i], to = in.cu[i + 1];
    bad |= from < 0 || to < from || to > in.n_rows || (i == 0 && from != 0) || (i == in.n_resp - 1 && to != in.n_rows);
    const long long lo = min(max(from, 0LL), in.n_rows), hi = min(max(to, lo), in.n_rows);
    double s = 0.0;
    int n = 0;
    if (hi > lo)
      for (unsigned b = (unsigned)lo / (unsigned)tile_rows; b <= (unsigned)(hi - 1) / (unsigned)tile_rows; ++b) {
        s += in.sums[i + (size_t)b];
        n += in.counts[i + (size_t)b];
      }
    share[j] = p.mean_logp ? (n > 0 ? 1.0 / (double)n : 0.0) : 1.0;
    d[j] = s * share[j];
    in.reward[i] = (float)((double)p.beta * d[j]);
  }
  if (bad) atomicOr(in.status, AIS_STATUS_BAD_CU);
  const double beta = (double)p.beta, h = beta * (d[0] - d[1]) - (double)p.margin;
  const double w = in.weight != nullptr ? (double)in.weight[pair] : 2.0 / (double)in.n_resp;
  double l, slope;
  if (p.kind == 0) {
    const double e = exp(-fabs(h)), both = log1p(e), wrong = (double)p.label_smoothing;
    // sigmoid(-h) and sigmoid(h), neither from 1 less the other
    const double small = e / (1.0 + e), large = 1.0 / (1.0 + e);
    const double down = h >= 0.0 ? small : large, up = h >= 0.0 ? large : small;
    l = (1.0 - wrong) * (both + (h < 0.0 ? -h : 0.0)) + wrong * (both + (h > 0.0 ? h : 0.0));
    slope = wrong * up - (1.0 - wrong) * down;
    if (h != h) l = slope = h;
  } else if (p.kind == 1) {
    l = h < 1.0 ? 1.0 - h : 0.0;
    slope = h < 1.0 ? -1.0 : 0.0;
    if (h != h) l = slope = h;
  } else {
    const double q = (h - 0.5) / beta;
    l = q * q;
    slope = 2.0 * q / beta;
  }
  const double c = w * slope * beta;
  in.coeff[2 * pair] = (float)(-c * share[0]);
  in.coeff[2 * pair + 1] = (float)(c * share[1]);
  return w * l;
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
  const long long r0 = (long long)blockIdx.x * kTileRows;
  tile.sum(in, (int)blockIdx.x, r0, min(r0 + kTileRows, in.n_rows));
}

// A thread to a pair.
__global__ __launch_bounds__(kTileThreads) void preference_pairs_kernel(Preference in) {
  const int pair = blockIdx.x * kTileThreads + threadIdx.x;
  if (2 * pair < in.n_resp) in.loss[pair] = pair_terms(in, pair, kTileRows);
}

// A workgroup to a tile; one more adds up the pairs' losses.
__global__ __launch_bounds__(kTileThreads) void preference_rows_kernel(Preference in, int tiles) {
  __shared__ Tile<kTileThreads> tile;
  if ((int)blockIdx.x == tiles) {
    double s = 0.0;
    for (int p = threadIdx.x; p < in.n_resp / 2; p += kTileThreads) s += in.loss[p];
    add_up<kTileThreads>(s, in.loss_out);
    return;
  }
  const long long r0 = (long long)blockIdx.x * kTileRows, r1 = min(r0 + kTileRows, in.n_rows);
  tile.mark(in, r0, r1);
  tile.spread(in, r0, r1);
}

// All of it in one workgroup.
__global__ __launch_bounds__(kOneThreads) void preference_one_kernel(Preference in) {
  __shared__ Tile<kOneThreads> tile;
  if (in.n_rows > 0) tile.sum(in, 0, 0, in.n_rows);
  __threadfence_block();
  __syncthreads();
  double s = 0.0;
  for (int p = threadIdx.x; p < in.n_resp / 2; p += kOneThreads) s += pair_terms(in, p, kOneRows);
  __threadfence_block();
  __syncthreads();
  if (in.n_rows > 0) tile.spread(in, 0, in.n_rows);
  add_up<kOneThreads>(s, in.loss_out);
}

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

PreferenceRoom preference_room(long long n_rows, int n_resp, bool through_logits) {
  const size_t places = (size_t)n_resp + (size_t)((n_rows + kTileRows - 1) / kTileRows);
  PreferenceRoom r;
  r.counts = padded(8 * places);
  r.loss = r.counts + padded(4 * places);
  r.coeff = r.loss + padded(4 * (size_t)n_resp);
  r.g = r.coeff + padded(4 * (size_t)n_resp);
  r.lse = r.g + padded(4 * (size_t)n_rows);
  r.fine = r.lse + padded(4 * (size_t)n_rows);
  r.total = through_logits ? r.fine + padded(8 * (size_t)n_rows) : r.g;
  return r;
}

int launch_preference(ais_ctx* ctx, const float* logp, const double* fine, const float* ref, const unsigned char* valid,
                      long long n_rows, const long long* cu_rows, int n_resp, const float* weight, const ais_preference_params& p,
                      const PreferenceRoom& room, float scale, float* reward, float* loss_out, float* g) {
  ScopedTimer timer(ctx, AIS_K_PREFERENCE);
  char* ws = static_cast<char*>(ctx->ws);
  const Preference in{logp, fine, ref, valid, cu_rows, weight, n_resp, n_rows, p, scale, reinterpret_cast<double*>(ws),
                      reinterpret_cast<int*>(ws + room.counts), reinterpret_cast<double*>(ws + room.loss),
                      reinterpret_cast<float*>(ws + room.coeff), reward, loss_out, g, ctx->status_dev};
  if (n_rows <= kOneRows && n_resp <= kOneRows) {
    preference_one_kernel<<<dim3(1), dim3(kOneThreads), 0, ctx->stream>>>(in);
    return hip_fail(ctx, hipGetLastError());
  }
  const int tiles = (int)((n_rows + kTileRows - 1) / kTileRows);
  if (tiles > 0) preference_sums_kernel<<<dim3((unsigned)tiles), dim3(kTileThreads), 0, ctx->stream>>>(in);
  preference_pairs_kernel<<<dim3((unsigned)((n_resp / 2 - 1) / kTileThreads + 1)), dim3(kTileThreads), 0, ctx->stream>>>(in);
  preference_rows_kernel<<<dim3((unsigned)tiles + 1), dim3(kTileThreads), 0, ctx->stream>>>(in, tiles);
  return hip_fail(ctx, hipGetLastError());
}

}  // namespace ais
