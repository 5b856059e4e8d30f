// Rows of logits over a vocabulary: log-probability of the chosen token, entropy, the clipped policy loss with a KL term, and
// the gradients of all of them.
//
//   z = x / temperature, m = max z, s = sum exp(z - m), p = exp(z - m) / s
//   logp = z_t - m - log s,   H = log s - sum p (z - m)
//   d/dx of g logp + h H:   [ g ([j = t] - p_j) - h p_j (log p_j + H) ] / temperature
// The kernels work with d = x - max x (exact to one fp32 rounding whatever the size of x) and e = exp2(d * log2(e) / temperature).
// A row is idle when its target is outside [0, vocab) (its logits are not read then) or none of its logits is above -infinity:
// log-probability, entropy and terms of the loss 0, gradient row 0.
#pragma once
#include "elem.hip.h"

struct RowArgs {
  int64_t rows, ld, ldd;   // row strides of the logits and of their gradient
  int32_t vocab;
  const void* logits;
  const int32_t* target;
  float inv_t;
  float *logp, *entropy, *stat;                       // results per row (entropy, stat: may be NULL); stat: (max x, log s)
  // gradients
  void* dlogits;
  const float *dlogp, *dentropy;                      // backward of the log-probability
  const float *logp_old, *logp_ref, *adv, *weight;    // loss (logp_ref, weight: may be NULL)
  float clip_lo, clip_hi, kl_coef, ent_coef, scale;
  float* record;                                      // loss: LossRecord per row
};

// What a row adds to the statistics of the loss.
struct LossRecord { float pi, kl, ent, old_kl, clipped, active; };

struct RowStat { float mx, s, sd; };  // max x; sum e; sum e d

__device__ __forceinline__ float block_max(float v, float* lds) {
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v = fmaxf(v, lds[w]);
  __syncthreads();
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* lds) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v += lds[w];
  __syncthreads();
  return v;
}

#define TOKEN_LOG2E 1.44269504088896340736f
// d of a logit of -infinity is -infinity: as a factor it is held at a finite value, so that 0 * d stays 0
__device__ __forceinline__ float finite_d(float d) { return fmaxf(d, -1e30f); }

template <class T, bool ENT>
__device__ __forceinline__ RowStat row_stat(const T* x, int V, float inv_t, float* lds) {
  RowStat r;
  float mx = -INFINITY, bad = 0.f;
  for (int i = threadIdx.x; i < V; i += blockDim.x) {
    const float v = to_f(x[i]);
    mx = fmaxf(mx, v);
    bad += v != v ? 1.f : 0.f;
  }
  r.mx = block_max(mx, lds);
  if (block_sum(bad, lds) > 0.f) r.mx = NAN;   // a row of NaN and -infinity is not an idle one
  float s = 0.f, sd = 0.f;
  for (int i = threadIdx.x; i < V; i += blockDim.x) {
    const float d = to_f(x[i]) - r.mx, e = exp2f(d * (inv_t * TOKEN_LOG2E));
    s += e;
    if (ENT) sd += e * finite_d(d);
  }
  r.s = block_sum(s, lds);
  r.sd = ENT ? block_sum(sd, lds) : 0.f;
  return r;
}

template <class T, bool ENT>
__global__ __launch_bounds__(256) void k_token_logp(RowArgs a) {
  __shared__ float lds[16];
  const int64_t row = blockIdx.x;
  const int t = a.target[row];
  const T* x = (const T*)a.logits + row * a.ld;
  float logp = 0.f, ent = 0.f, st0 = 0.f, st1 = 0.f;
  if (t >= 0 && t < a.vocab) {
    const RowStat r = row_stat<T, ENT>(x, a.vocab, a.inv_t, lds);
    if (r.mx != -INFINITY) {
      const float ls = logf(r.s);
      logp = (to_f(x[t]) - r.mx) * a.inv_t - ls;
      ent = ls - r.sd / r.s * a.inv_t;
      st0 = r.mx; st1 = ls;
    } else { st0 = -INFINITY; }
  }
  if (threadIdx.x == 0) {
    a.logp[row] = logp;
    if (a.entropy) a.entropy[row] = ent;
    if (a.stat) { a.stat[2 * row] = st0; a.stat[2 * row + 1] = st1; }
  }
}

// gradient row: -e (k0 + k1 d) and, at the target, + add
template <class T, bool ENT>
__device__ __forceinline__ void row_gradient(const T* x, T* y, int V, int t, float mx, float c, float k0, float k1, float add) {
  for (int i = threadIdx.x; i < V; i += blockDim.x) {
    const float d = to_f(x[i]) - mx, e = exp2f(d * c);
    float g = -e * (ENT ? k0 + k1 * finite_d(d) : k0);
    if (i == t) g += add;
    y[i] = from_f<T>(g);
  }
}

template <class T, bool ENT>
__global__ __launch_bounds__(256) void k_token_logp_backward(RowArgs a) {
  const int64_t row = blockIdx.x;
  const int t = a.target[row];
  const T* x = (const T*)a.logits + row * a.ld;
  T* y = (T*)a.dlogits + row * a.ldd;
  const float mx = a.stat[2 * row], ls = a.stat[2 * row + 1];
  if (t < 0 || t >= a.vocab || mx == -INFINITY) {
    for (int i = threadIdx.x; i < a.vocab; i += 256) y[i] = from_f<T>(0.f);
    return;
  }
  const float g = a.dlogp[row], h = ENT ? a.dentropy[row] : 0.f, H = ENT ? a.entropy[row] : 0.f;
  const float is = expf(-ls) * a.inv_t;
  row_gradient<T, ENT>(x, y, a.vocab, t, mx, a.inv_t * TOKEN_LOG2E, (g + h * (H - ls)) * is, h * a.inv_t * is, g * a.inv_t);
}

// Terms of the loss at one token and their derivatives by logp (g) and H (h), all without weight.
struct LossTerm { float g, h; LossRecord rec; };
__device__ __forceinline__ LossTerm loss_term(const RowArgs& a, int64_t row, float logp, float ent) {
  LossTerm o;
  const float adv = a.adv[row], lr = logp - a.logp_old[row], rho = expf(lr);
  const float lo = 1.f - a.clip_lo, hi = 1.f + a.clip_hi;
  const float s1 = rho * adv, s2 = fminf(fmaxf(rho, lo), hi) * adv;
  const bool held = s1 > s2;  // ties: the unclipped branch carries the gradient; so does a NaN, which is to be seen in the loss
  o.rec.pi = held ? -s2 : -s1;
  o.g = held ? 0.f : -s1;
  o.rec.kl = 0.f;
  if (a.logp_ref) {
    const float d = a.logp_ref[row] - logp, ed = expf(d);
    o.rec.kl = ed - d - 1.f;
    o.g += a.kl_coef * (1.f - ed);
  }
  o.rec.ent = ent;
  o.h = -a.ent_coef;
  o.rec.old_kl = (rho - 1.f) - lr;
  o.rec.clipped = rho < lo || rho > hi ? 1.f : 0.f;
  o.rec.active = 1.f;
  return o;
}

template <class T, bool ENT>
__global__ __launch_bounds__(256) void k_token_loss(RowArgs a) {
  __shared__ float lds[16];
  const int64_t row = blockIdx.x;
  const int t = a.target[row];
  const T* x = (const T*)a.logits + row * a.ld;
  T* y = (T*)a.dlogits + row * a.ldd;
  RowStat r = {-INFINITY, 0.f, 0.f};
  if (t >= 0 && t < a.vocab) r = row_stat<T, ENT>(x, a.vocab, a.inv_t, lds);
  if (r.mx == -INFINITY) {
    for (int i = threadIdx.x; i < a.vocab; i += 256) y[i] = from_f<T>(0.f);
    if (threadIdx.x == 0) { a.logp[row] = 0.f; ((LossRecord*)a.record)[row] = LossRecord{0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }
    return;
  }
  const float ls = logf(r.s), logp = (to_f(x[t]) - r.mx) * a.inv_t - ls, H = ENT ? ls - r.sd / r.s * a.inv_t : 0.f;
  LossTerm o = loss_term(a, row, logp, H);
  const float w = (a.weight ? a.weight[row] : 1.f) * a.scale, g = w * o.g, h = w * o.h, is = a.inv_t / r.s;
  __syncthreads();  // x[t] is read: the gradient may lie in the memory of the logits
  row_gradient<T, ENT>(x, y, a.vocab, t, r.mx, a.inv_t * TOKEN_LOG2E, (g + h * (H - ls)) * is, h * a.inv_t * is, g * a.inv_t);
  if (threadIdx.x == 0) {
    a.logp[row] = logp;
    o.rec.pi *= w; o.rec.kl *= w; o.rec.ent *= w;
    ((LossRecord*)a.record)[row] = o.rec;
  }
}

// Statistics of the loss: the rows' records added in a fixed order, in 64 bits.
// stats: loss, pi, kl, entropy (weighted sums), mean approx_kl, clipped share, active rows, non-finite
__global__ __launch_bounds__(1024) void k_token_stats(int64_t rows, const LossRecord* rec, float kl_coef, float ent_coef, float* stats) {
  __shared__ double lds[6][16];
  double v[6] = {0, 0, 0, 0, 0, 0};
  for (int64_t i = threadIdx.x; i < rows; i += 1024) {
    const LossRecord r = rec[i];
    v[0] += r.pi; v[1] += r.kl; v[2] += r.ent; v[3] += r.old_kl; v[4] += r.clipped; v[5] += r.active;
  }
  for (int k = 0; k < 6; ++k) {
    for (int o = 32; o; o >>= 1) v[k] += __shfl_xor(v[k], o);
    if ((threadIdx.x & 63) == 0) lds[k][threadIdx.x >> 6] = v[k];
  }
  __syncthreads();
  if (threadIdx.x) return;
  for (int k = 0; k < 6; ++k) { v[k] = 0; for (int w = 0; w < 16; ++w) v[k] += lds[k][w]; }
  const double loss = v[0] + (double)kl_coef * v[1] - (double)ent_coef * v[2], n = v[5] > 0 ? v[5] : 1;
  stats[0] = (float)loss; stats[1] = (float)v[0]; stats[2] = (float)v[1]; stats[3] = (float)v[2];
  stats[4] = (float)(v[3] / n); stats[5] = (float)(v[4] / n); stats[6] = (float)v[5];
  stats[7] = isfinite((float)loss) ? 0.f : 1.f;
}
