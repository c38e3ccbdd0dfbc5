// A pair of responses in the preference loss, in fp64: shared by the kernels that write the coefficients of a batch and by the gradient
// sweep of small batches, which forms its own.
#pragma once

#include "row_coeff.h"

namespace ais {

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
  // In the workspace: partial sums and counts (response i in tile b has place i + b, which no other pair of them has), the
  // pairs' losses, the responses' coefficients
  double* sums;
  int* counts;
  double* loss;
  float* coeff;
  int* firsts;                                   // response that each tile begins in
  float *reward, *loss_out, *g;
  int* status;
};

namespace dev {

struct PairTerm {
  float reward[2], coeff[2];
  double loss;                                   // times the pair's weight
};

// From the sums of the two responses' log-ratios and their numbers of tokens.  LOSS: the loss, too.
template <bool LOSS>
__device__ __forceinline__ PairTerm pair_term(const Preference& in, int pair, const double* s, const int* n) {
  const ais_preference_params& p = in.p;
  PairTerm t;
  double d[2], share[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    share[j] = p.mean_logp ? (n[j] > 0 ? 1.0 / (double)n[j] : 0.0) : 1.0;
    d[j] = s[j] * share[j];
    t.reward[j] = (float)((double)p.beta * d[j]);
  }
  const double beta = (double)p.beta, h = beta * (d[0] - d[1]) - (double)p.margin;
  const double w = in.weight != nullptr ? (double)in.weight[pair] : 2.0 / (double)in.n_resp;
  double l = 0.0, slope;
  if (p.kind == 0) {
    const double e = exp64(-fabs(h)), wrong = (double)p.label_smoothing;
    // sigmoid(-h) and sigmoid(h), neither from 1 less the other
    const double large = 1.0 / (1.0 + e), small = e * large;
    const double down = h >= 0.0 ? small : large, up = h >= 0.0 ? large : small;
    slope = wrong * up - (1.0 - wrong) * down;
    if (LOSS) {
      const double both = log1p(e);
      l = (1.0 - wrong) * (both + (h < 0.0 ? -h : 0.0)) + wrong * (both + (h > 0.0 ? h : 0.0));
    }
  } else if (p.kind == 1) {
    l = h < 1.0 ? 1.0 - h : 0.0;
    slope = h < 1.0 ? -1.0 : 0.0;
  } else {
    const double q = (h - 0.5) / beta;
    l = q * q;
    slope = 2.0 * q / beta;
  }
  if (h != h) l = slope = h;
  const double c = w * slope * beta;
  t.coeff[0] = (float)(-c * share[0]);
  t.coeff[1] = (float)(c * share[1]);
  t.loss = w * l;
  return t;
}

// Rows of response i, whose offsets are from and to, inside the batch.
struct RowRange {
  unsigned lo, hi;
  bool sound;
};
__device__ __forceinline__ RowRange rows_of(const Preference& in, int i, long long from, long long to) {
  const bool sound = !(from < 0 || to < from || to > in.n_rows || (i == 0 && from != 0) || (i == in.n_resp - 1 && to != in.n_rows));
  const long long lo = min(max(from, 0LL), in.n_rows), hi = min(max(to, lo), in.n_rows);
  return {(unsigned)lo, (unsigned)hi, sound};
}

}  // namespace dev
}  // namespace ais
