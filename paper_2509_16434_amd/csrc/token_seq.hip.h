// Sequences packed one behind the other: sequence k holds the tokens [offsets[k], offsets[k+1]).  Offsets are held inside
// [0, tokens] before they are used, so that a wrong one cannot reach memory outside the arrays.
#pragma once
#include "common.hip.h"

__device__ __forceinline__ int64_t hold(int64_t o, int64_t tokens) { return o < 0 ? 0 : o > tokens ? tokens : o; }

// ---------------------------------------------------------------- preference loss
// Pairs (k, pairs + k) of a chosen and a rejected sequence.  S = sum over the unmasked tokens of (logp - ref) (or their mean),
// D = S_chosen - S_rejected; loss of a pair -(1 - ls) log sigmoid(bD) - ls log sigmoid(-bD), or (D - 1/(2b))^2.  D is a small
// difference of long sums: they are held in 64 bits.  A pair with no unmasked token in one of its sequences adds nothing.
struct PairArgs {
  int64_t pairs, tokens;
  const float *logp, *ref;   // ref: may be NULL
  const uint8_t* mask;       // may be NULL
  const int64_t* offsets;    // [2 * pairs + 1]
  int32_t kind, mean;
  float beta, smoothing, scale;
  float *dlogp, *margin;
  float* stats;
  struct PairRecord* record;
};
struct PairRecord { double loss, right, margin, chosen, rejected, active; };

__device__ __forceinline__ double block_sum_d(double v, double* lds) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) v += lds[w];
  __syncthreads();
  return v;
}

// loss of a pair and its derivative by D
__device__ __forceinline__ void pair_term(int kind, double beta, double ls, double D, double* loss, double* slope) {
  if (kind == 0) {
    const double x = beta * D, soft = log1p(exp(-fabs(x)));             // -log sigmoid(|x|)
    const double pos = soft + (x < 0 ? -x : 0), neg = soft + (x > 0 ? x : 0);
    *loss = (1 - ls) * pos + ls * neg;
    *slope = beta * (ls - 1 / (1 + exp(x)));
  } else {
    const double e = D - 0.5 / beta;
    *loss = e * e;
    *slope = 2 * e;
  }
}

__global__ __launch_bounds__(256) void k_pair_loss(PairArgs a) {
  __shared__ double lds[4];
  const int64_t k = blockIdx.x;
  double S[2], n[2];
  int64_t from[2], to[2];
  for (int q = 0; q < 2; ++q) {
    const int64_t s = k + q * a.pairs;
    from[q] = hold(a.offsets[s], a.tokens); to[q] = hold(a.offsets[s + 1], a.tokens);
    double v = 0, c = 0;
    for (int64_t i = from[q] + threadIdx.x; i < to[q]; i += 256)
      if (!a.mask || a.mask[i]) { v += (double)a.logp[i] - (a.ref ? (double)a.ref[i] : 0.0); c += 1; }
    S[q] = block_sum_d(v, lds); n[q] = block_sum_d(c, lds);
  }
  const bool on = n[0] > 0 && n[1] > 0;
  double loss = 0, slope = 0;
  const double f[2] = {a.mean && on ? 1 / n[0] : 1.0, a.mean && on ? 1 / n[1] : 1.0};
  S[0] *= f[0]; S[1] *= f[1];
  if (on) pair_term(a.kind, a.beta, a.smoothing, S[0] - S[1], &loss, &slope);
  slope *= a.scale;
  for (int q = 0; q < 2; ++q) {
    const float g = (float)((q ? -slope : slope) * f[q]);
    for (int64_t i = from[q] + threadIdx.x; i < to[q]; i += 256) a.dlogp[i] = on && (!a.mask || a.mask[i]) ? g : 0.f;
  }
  if (threadIdx.x == 0) {
    const double D = S[0] - S[1], b = a.beta;
    if (a.margin) a.margin[k] = on ? (float)(b * D) : 0.f;
    a.record[k] = on ? PairRecord{loss, D > 0 ? 1.0 : 0.0, b * D, b * S[0], b * S[1], 1.0} : PairRecord{0, 0, 0, 0, 0, 0};
  }
}

// the gradient of the tokens outside every sequence
__global__ __launch_bounds__(256) void k_pair_outside(PairArgs a) {
  const int64_t first = hold(a.offsets[0], a.tokens), last = hold(a.offsets[2 * a.pairs], a.tokens);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.tokens; i += (int64_t)gridDim.x * 256)
    if (i < first || i >= last) a.dlogp[i] = 0.f;
}

// stats: loss, share of pairs with D > 0, mean margin, mean chosen and rejected reward, active pairs, non-finite
__global__ __launch_bounds__(1024) void k_pair_stats(int64_t pairs, const PairRecord* rec, float scale, float* stats) {
  __shared__ double lds[16];
  double v[6] = {0, 0, 0, 0, 0, 0};
  for (int64_t i = threadIdx.x; i < pairs; i += 1024) {
    const PairRecord r = rec[i];
    v[0] += r.loss; v[1] += r.right; v[2] += r.margin; v[3] += r.chosen; v[4] += r.rejected; v[5] += r.active;
  }
  for (int k = 0; k < 6; ++k) v[k] = block_sum_d(v[k], lds);
  if (threadIdx.x) return;
  const double n = v[5] > 0 ? v[5] : 1;
  stats[0] = (float)(v[0] * scale);
  for (int k = 1; k < 5; ++k) stats[k] = (float)(v[k] / n);
  stats[5] = (float)v[5];
  stats[6] = isfinite(stats[0]) ? 0.f : 1.f;
}

// ---------------------------------------------------------------- advantages
// A_t = r_t + gamma V' - V_t + gamma lambda A', where the primes are the next unmasked token of the sequence; behind the last
// one V' is the sequence's last value (0 without one) and A' = 0.  R_t = A_t + V_t.  Masked tokens get 0.
//
// As maps of the pair (A, V) that comes from behind, a token is  A -> a A + b V + c,  V -> v or V (masked tokens: nothing
// changes), and maps of this form compose, so that a scan over maps gives every token's pair.
struct GaeArgs {
  int64_t sequences, tokens;
  const float *reward, *value, *last_value;  // last_value: may be NULL
  const uint8_t* mask;                       // may be NULL
  const int64_t* offsets;
  double gamma, lambda;
  float *adv, *ret;
};
struct GaeMap { double a, b, c, v; int set; };  // set: V -> v, else V stays
// first `behind`, then `m`
__device__ __forceinline__ GaeMap then(const GaeMap& behind, const GaeMap& m) {
  GaeMap o;
  o.a = m.a * behind.a;
  o.b = m.a * behind.b + (behind.set ? 0.0 : m.b);
  o.c = m.a * behind.c + (behind.set ? m.b * behind.v : 0.0) + m.c;
  o.set = m.set | behind.set;
  o.v = m.set ? m.v : behind.v;
  return o;
}
__device__ __forceinline__ GaeMap shfl_down_map(const GaeMap& m, int o) {
  return GaeMap{__shfl_down(m.a, o), __shfl_down(m.b, o), __shfl_down(m.c, o), __shfl_down(m.v, o), __shfl_down(m.set, o)};
}

// the tokens outside every sequence
__global__ __launch_bounds__(256) void k_gae_outside(GaeArgs a) {
  const int64_t first = a.sequences ? hold(a.offsets[0], a.tokens) : a.tokens, last = hold(a.offsets[a.sequences], a.tokens);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.tokens; i += (int64_t)gridDim.x * 256)
    if (i < first || i >= last) a.adv[i] = a.ret[i] = 0.f;
}

// one wave per sequence, 64 tokens at a time from the end
__global__ __launch_bounds__(64) void k_token_gae(GaeArgs a) {
  const int64_t s = blockIdx.x;
  const int lane = threadIdx.x;
  const int64_t from = hold(a.offsets[s], a.tokens), to = hold(a.offsets[s + 1], a.tokens);
  double A = 0, V = a.last_value ? (double)a.last_value[s] : 0.0;
  for (int64_t end = to; end > from; end -= 64) {
    const int64_t i = end - 64 + lane;
    const bool in = i >= from, on = in && (!a.mask || a.mask[i]);
    const double r = on ? (double)a.reward[i] : 0, v = on ? (double)a.value[i] : 0;
    GaeMap m = on ? GaeMap{a.gamma * a.lambda, a.gamma, r - v, v, 1} : GaeMap{1, 0, 0, 0, 0};
    for (int o = 1; o < 64; o <<= 1) {
      const GaeMap b = shfl_down_map(m, o);
      if (lane + o < 64) m = then(b, m);
    }
    const double adv = m.a * A + m.b * V + m.c;
    if (in) { a.adv[i] = on ? (float)adv : 0.f; a.ret[i] = on ? (float)(adv + v) : 0.f; }
    V = __shfl(m.set ? m.v : V, 0);
    A = __shfl(adv, 0);
  }
}
