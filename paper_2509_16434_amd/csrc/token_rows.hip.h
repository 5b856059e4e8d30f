// Rows of logits over a vocabulary: log-probability of the chosen token, entropy, the clipped policy loss with a KL term, and
// the gradients of all of them.
//
//   z = x / temperature, m = max z, s = sum exp(z - m), p = exp(z - m) / s
//   logp = z_t - m - log s,   H = log s - sum p (z - m)
//   d/dx of g logp + h H:   [ g ([j = t] - p_j) - h p_j (log p_j + H) ] / temperature
// The kernels work with d = x - max x (exact to one fp32 rounding whatever the size of x), y = d c, c = log2(e) / temperature, and e = exp2(y).
// Only y and e go into sums and gradients: d of a banned logit and powers of 1 / temperature may lie beyond fp32 where the result does not.
// A row is idle when its target is outside [0, vocab) (its logits are not read then) or none of its logits is above -infinity:
// log-probability, entropy and terms of the loss 0, gradient row 0.
//
// All of it is bound by memory: 2 or 4 bytes a logit once in and, for a gradient, once out.  A row is worked on by G threads that
// take it in 16-byte pieces from its first 16-byte boundary on, and head and tail element by element, so that rows of odd length, which
// begin anywhere, are read as fast as others; a gradient row that begins elsewhere is written in pieces across the boundaries.
//
// Measured (GB/s of one read and, for gradients, one write of every logit; a plain copy of 2 GiB reaches 4490, reading alone 5200):
//   log-probability   8192 x 50257 fp16 5790, 8192 x 131072 bf16 6040, 65536 x 1000 bf16 5100
//   loss              16384 x 131072 bf16 5480, 8192 x 32000 bf16 5090, 3001 x 50257 bf16 with entropy 4900, 32768 x 2000 bf16 with entropy 4700, 131072 x 257 bf16 with entropy 3460
//   backward          4096 x 32000 fp32 5800
#pragma once
#include "elem.hip.h"
#include "lanes.hip.h"

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
  float* part;                                        // rows in slices: four numbers per row and slice
  int32_t slices, slice_len;
};

// What a row adds to the statistics of the loss.
struct LossRecord { float pi, kl, ent, old_kl, clipped, active; };

// max x, sum e, sum e y (with respect to the max; to 0 where it is -infinity).  idle(): nothing above -infinity, and no NaN.
struct RowStat {
  float mx, s, sy;
  __device__ __forceinline__ float base() const { return mx == -INFINITY ? 0.f : mx; }
  __device__ __forceinline__ bool idle() const { return mx == -INFINITY && s == 0.f; }
};

#define TOKEN_LOG2E 1.44269504088896340736f
#define TOKEN_LN2 0.69314718055994530942f
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }  // 1 ulp; results below 2^-126 are 0
// y of a logit of -infinity is -infinity: as a factor it is held where exp2 is 0 already, so that e y is 0
__device__ __forceinline__ float finite_y(float y) { return fmaxf(y, -200.f); }

// ---- statistics of parts of a row, joined
// b's sums with respect to the maximum mx (>= b.mx)
template <bool ENT>
__device__ __forceinline__ RowStat rebase(RowStat b, float mx, float c) {
  const bool none = b.mx == -INFINITY;   // sums 0 (or NaN): no factor
  const float y = none ? 0.f : (b.mx - mx) * c, f = exp2_hw(y);
  if (ENT) b.sy = f * (b.sy + b.s * finite_y(y));
  b.s *= f;
  b.mx = mx;
  return b;
}
// the threads of a row's group; r: the thread's own part, on return the row's.  lds: 3 floats per wave of the block; one barrier
// (G <= 64: neither).
template <int G, bool ENT>
__device__ __forceinline__ RowStat group_join(RowStat r, float c, float* lds) {
  constexpr int W = G < 64 ? G : 64;
  RowStat w = rebase<ENT>(r, lanes_max<W>(r.mx), c);
  w.s = lanes_sum<W>(w.s);
  if (ENT) w.sy = lanes_sum<W>(w.sy);
  if constexpr (G <= 64) return w;
  else {
    constexpr int NW = G / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { lds[3 * wave] = w.mx; lds[3 * wave + 1] = w.s; if (ENT) lds[3 * wave + 2] = w.sy; }
    __syncthreads();
    // every 16 lanes read the (at most 16) waves' parts, one each
    const int k = threadIdx.x & 15;
    RowStat p = {-INFINITY, 0.f, 0.f};
    if (k < NW) p = RowStat{lds[3 * k], lds[3 * k + 1], ENT ? lds[3 * k + 2] : 0.f};
    RowStat all = rebase<ENT>(p, lanes_max<16>(p.mx), c);
    all.s = lanes_sum<16>(all.s);
    if (ENT) all.sy = lanes_sum<16>(all.sy);
    return all;
  }
}

// adds an element's, a piece's terms to r, whose maximum covers them
template <bool ENT>
__device__ __forceinline__ void add_one(RowStat& r, float x, float base, float c) {
  const float y = (x - base) * c, e = exp2_hw(y);
  r.s += e;
  if (ENT) r.sy += e * finite_y(y);
}
template <class T, bool ENT>
__device__ __forceinline__ void add_piece(RowStat& r, u32x4_t v, float base, float c) {
  float f[Piece<T>::N];
  unpack(v, f, T());
#pragma unroll
  for (int k = 0; k < Piece<T>::N; ++k) add_one<ENT>(r, f[k], base, c);
}
template <class T>
__device__ __forceinline__ float max_piece(u32x4_t v) {
  float f[Piece<T>::N], m;
  unpack(v, f, T());
  m = f[0];
#pragma unroll
  for (int k = 1; k < Piece<T>::N; ++k) m = fmaxf(m, f[k]);
  return m;
}

// The statistics of n elements by G threads in one pass: every thread keeps its own maximum and sums, brought to a new maximum
// U pieces at a time, so that U loads are in flight and one exponential in 8 U (or 4 U) is for that.
template <class T, int G, bool ENT>
__device__ __forceinline__ RowStat stream_stat(const T* x, int n, int tid, float c) {
  constexpr int N = Piece<T>::N, U = 4;
  const Cut q = cut_row(x, n, tid);
  RowStat r = {q.one >= 0 ? to_f(x[q.one]) : -INFINITY, 0.f, 0.f};
  if (r.mx > -INFINITY) r.s = 1.f;
  else if (r.mx != r.mx) r = RowStat{-INFINITY, NAN, NAN};
  x += q.head;
  for (int i = tid * N; i < q.full; i += G * N * U) {
    Pieces<U> v;
    float m = r.mx;
    each<U>([&](auto u) INLINE { if (i + u * G * N < q.full) piece<u>(v) = load_piece(x + i + u * G * N); });
    each<U>([&](auto u) INLINE { if (i + u * G * N < q.full) m = fmaxf(m, max_piece<T>(piece<u>(v))); });
    r = rebase<ENT>(r, m, c);
    const float base = r.base();
    each<U>([&](auto u) INLINE { if (i + u * G * N < q.full) add_piece<T, ENT>(r, piece<u>(v), base, c); });
  }
  return r;
}

struct RowOut { float logp, ent, ls; };
__device__ __forceinline__ RowOut row_out(const RowStat& r, float xt, float inv_t, bool ent) {
  RowOut o;
  o.ls = logf(r.s);
  o.logp = (xt - r.base()) * inv_t - o.ls;
  o.ent = ent ? o.ls - r.sy / r.s * TOKEN_LN2 : 0.f;
  return o;
}

// Log-probability (and entropy) of rows by groups of G threads.
template <class T, int G, bool ENT>
__global__ __launch_bounds__(G < 256 ? 256 : G) void k_token_logp(RowArgs a) {
  constexpr int NT = G < 256 ? 256 : G;
  __shared__ float lds[3 * (NT / 64)];
  const int64_t row = (int64_t)blockIdx.x * (NT / G) + (G < 256 ? threadIdx.x / G : 0);
  if (G < 256 && row >= a.rows) return;   // G <= 64: no barrier follows
  const int t = a.target[row];
  const float c = a.inv_t * TOKEN_LOG2E;
  const T* x = (const T*)a.logits + row * a.ld;
  RowOut o = {0.f, 0.f, 0.f};
  float mx = -INFINITY;
  if (t >= 0 && t < a.vocab) {
    const float xt = to_f(x[t]);
    const RowStat r = group_join<G, ENT>(stream_stat<T, G, ENT>(x, a.vocab, threadIdx.x % G, c), c, lds);
    if (!r.idle()) { o = row_out(r, xt, a.inv_t, ENT); mx = r.base(); }
  }
  if (threadIdx.x % G == 0) {
    a.logp[row] = o.logp;
    if (a.entropy) a.entropy[row] = o.ent;
    if (a.stat) { a.stat[2 * row] = mx; a.stat[2 * row + 1] = o.ls; }
  }
}

// Few long rows: statistics of slices of a row, one block each: (max, sum e, sum e y), and in the first slice's spare place the target's
// logit (the gradient may overwrite it in the logits' memory before every block has read it).
template <class T, bool ENT>
__global__ __launch_bounds__(256) void k_token_part(RowArgs a) {
  __shared__ float lds[12];
  const int64_t row = blockIdx.y;
  const int t = a.target[row];
  if (t < 0 || t >= a.vocab) return;   // nobody reads the parts of such a row
  const float c = a.inv_t * TOKEN_LOG2E;
  const int from = blockIdx.x * a.slice_len, n = min(a.vocab - from, a.slice_len);
  const RowStat r = group_join<256, ENT>(stream_stat<T, 256, ENT>((const T*)a.logits + row * a.ld + from, n, threadIdx.x, c), c, lds);
  if (threadIdx.x == 0) *(float4*)(a.part + 4 * (row * a.slices + blockIdx.x)) = make_float4(r.mx, r.s, r.sy, blockIdx.x == 0 ? to_f(((const T*)a.logits)[row * a.ld + t]) : 0.f);
}
// the parts of a row (at most 64), joined by one wave
template <bool ENT>
__device__ __forceinline__ RowStat join_parts(const RowArgs& a, int64_t row, float c) {
  const int lane = threadIdx.x & 63;
  RowStat r = {-INFINITY, 0.f, 0.f};
  if (lane < a.slices) { const float4 p = *(const float4*)(a.part + 4 * (row * a.slices + lane)); r = RowStat{p.x, p.y, p.z}; }
  return group_join<64, ENT>(r, c, nullptr);
}
template <bool ENT>
__global__ __launch_bounds__(256) void k_token_join(RowArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  const int t = a.target[row];
  RowOut o = {0.f, 0.f, 0.f};
  float mx = -INFINITY;
  if (t >= 0 && t < a.vocab) {
    const RowStat r = join_parts<ENT>(a, row, a.inv_t * TOKEN_LOG2E);
    if (!r.idle()) { o = row_out(r, a.part[4 * row * a.slices + 3], a.inv_t, ENT); mx = r.base(); }
  }
  if ((threadIdx.x & 63) == 0) {
    a.logp[row] = o.logp;
    if (a.entropy) a.entropy[row] = o.ent;
    if (a.stat) { a.stat[2 * row] = mx; a.stat[2 * row + 1] = o.ls; }
  }
}

// ---- gradient: -e (k0 + k1 y) / temperature, at the target (g - e (k0 + k1 y)) / temperature.  Where |k| / temperature is beyond 2^100 (a
// small temperature, a large loss scale), a power of two, 2^b, goes into e instead of the coefficients, so that neither they nor their product
// with a y of -200 overflow and an e of 0 makes 0 of them; it costs nothing in the loops.  b = 0 otherwise.
struct GradCoef { float mx, c, b, k0, k1, target; };   // target: the whole gradient there
// g: dL/dlogp, h: dL/dH; is = 1 / s; xt: the target's logit
template <bool ENT>
__device__ __forceinline__ GradCoef grad_coef(float g, float h, float ent, float ls, float mx, float is, float inv_t, float xt) {
  const float c = inv_t * TOKEN_LOG2E, k0 = (ENT ? g + h * (ent - ls) : g) * is, k1 = ENT ? h * TOKEN_LN2 * is : 0.f;
  const float y = (xt - mx) * c, e = exp2_hw(y);
  const int b = max(0, __builtin_amdgcn_frexp_expf(fmaxf(fabsf(k0), fabsf(k1))) + __builtin_amdgcn_frexp_expf(inv_t) - 100);
  const float f = ldexpf(inv_t, -b), m0 = k0 * f, m1 = k1 * f;
  return GradCoef{mx, c, (float)b, m0 - m1 * (float)b, m1, (g - (ENT ? e * k0 + e * finite_y(y) * k1 : e * k0)) * inv_t};
}
template <bool ENT>
__device__ __forceinline__ float grad_one(float x, const GradCoef& k) {
  const float y = (x - k.mx) * k.c + k.b, e = exp2_hw(y);
  return -e * (ENT ? k.k0 + k.k1 * finite_y(y) : k.k0);
}
template <class T, bool ENT>
__device__ __forceinline__ u32x4_t grad_piece(u32x4_t v, const GradCoef& k) {
  constexpr int N = Piece<T>::N;
  float f[N];
  unpack(v, f, T());
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = grad_one<ENT>(f[i], k);
  return pack(f, T());
}
template <class T>
__device__ __forceinline__ void zero_row(T* y, int n, int tid, int G) {
  const u32x4_t z = {0, 0, 0, 0};
  const Cut q = cut_row(y, n, tid);
  for (int i = tid * Piece<T>::N; i < q.full; i += G * Piece<T>::N) store_piece(y + q.head + i, z);
  if (q.one >= 0) y[q.one] = from_f<T>(0.f);
}

// Gradient of the log-probability and the entropy from the row's statistics: every piece by itself.  A group of G threads does a
// slice of G BACK_PIECES pieces of a row: blockIdx.x the slice (G < 256: the row is one slice), blockIdx.y and z the row.
// PAST: stored past the caches, for gradients that would push out of the last-level cache (256 MB) the logits that the forward pass has
// just read.  us of log-probability and backward pass, and with one more kernel that reads the gradient, into and past the caches:
//   rows of 32000 bf16   128 MB 60 and 60 (106, 105), 160 MB 78 and 74 (149, 136), 250 MB 139 and 111 (233, 215), 512 MB 287 and 252 (464, 446)
//   rows of 2000 bf16    128 MB 59 and 61 (108, 105), 160 MB 77 and 74 (146, 134), 250 MB 138 and 111 (231, 210)
//   rows of 500 bf16     128 MB 60 and 69 (107, 115), 160 MB 79 and 86 (150, 146), 250 MB 136 and 132 (229, 235), 520 MB 302 and 324 (483, 515)
// (the last begin inside cache lines, which two rows then write in part).  Smaller ones are worth more in the cache: 64 MB 32 and 33 (51, 54).
constexpr int64_t PAST_BYTES = 144000000;
constexpr int BACK_PIECES = 4;   // pieces per thread
template <class T, int G, bool ENT, bool PAST>
__global__ __launch_bounds__(256) void k_token_logp_backward(RowArgs a) {
  constexpr int N = Piece<T>::N;
  const int64_t back = G < 256 ? (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G : blockIdx.y + (int64_t)blockIdx.z * 65535;
  if (back >= a.rows) return;
  const int64_t row = a.rows - 1 - back;   // the rows that the forward pass read last are still in the last-level cache
  const int t = a.target[row], from = (G < 256 ? 0 : blockIdx.x * (G * BACK_PIECES * N)) + threadIdx.x % G * N;
  const int tid = threadIdx.x % G;
  const T* x = (const T*)a.logits + row * a.ld;
  T* y = (T*)a.dlogits + row * a.ldd;
  const auto store = [](T* p, u32x4_t v) { if constexpr (PAST) store_piece_past_caches(p, v); else store_piece(p, v); };
  Cut q = cut_row(x, a.vocab, tid);
  if (G >= 256 && blockIdx.x) q.one = -1;   // the first slice's threads take head and tail
  const float mx = a.stat[2 * row], ls = a.stat[2 * row + 1];
  if (t < 0 || t >= a.vocab || mx == -INFINITY) {
    const u32x4_t z = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < BACK_PIECES; ++u)
      if (from + u * G * N < q.full) store(y + q.head + from + u * G * N, z);
    if (q.one >= 0) y[q.one] = from_f<T>(0.f);
    return;
  }
  // the target's element is written again, by the thread that wrote it
  const int slice = G < 256 ? 0 : blockIdx.x * (G * BACK_PIECES * N), r = t - q.head;
  const bool owner = r >= 0 && r < q.full ? r >= slice && r < slice + G * BACK_PIECES * N && (r - slice) / N % G == tid : t == q.one;
  const float xl = q.one >= 0 ? to_f(x[q.one]) : 0.f;
  const float g = a.dlogp[row], h = ENT ? a.dentropy[row] : 0.f, H = ENT ? a.entropy[row] : 0.f;
  const GradCoef k = grad_coef<ENT>(g, h, H, ls, mx, expf(-ls), a.inv_t, owner ? to_f(x[t]) : mx);
  Pieces<BACK_PIECES> v;
  each<BACK_PIECES>([&](auto u) INLINE { if (from + u * G * N < q.full) piece<u>(v) = load_piece(x + q.head + from + u * G * N); });
  each<BACK_PIECES>([&](auto u) INLINE { if (from + u * G * N < q.full) store(y + q.head + from + u * G * N, grad_piece<T, ENT>(piece<u>(v), k)); });
  if (q.one >= 0) y[q.one] = from_f<T>(grad_one<ENT>(xl, k));
  if (owner) y[t] = from_f<T>(k.target);
}

// ---- loss
// exp d - 1 - d, em being exp d - 1.  Near 0 their difference loses what the result is made of (d = 2^-12: all but 12 bits, and the sign with
// the last of them), so there it is the series up to d^9 / 9! (the next term is 2^-29 of the sum at 1/2); where exp d is infinite (or d below
// all its digits), it is that.  12 roundings at the most, at +-1/2.
__device__ __forceinline__ float less_linear(float em, float d) {
  float q = 1.f / 362880;
  q = fmaf(q, d, 1.f / 40320);
  q = fmaf(q, d, 1.f / 5040);
  q = fmaf(q, d, 1.f / 720);
  q = fmaf(q, d, 1.f / 120);
  q = fmaf(q, d, 1.f / 24);
  q = fmaf(q, d, 1.f / 6);
  q = fmaf(q, d, 0.5f);
  return fabsf(d) < 0.5f ? q * d * d : d < 80.f ? em - d : em;
}
// What a token adds to the loss (its record) and the derivatives of that by logp (g) and H (h).
struct LossTerm { float g, h; LossRecord rec; };
struct LossIn { float old, ref, adv, w; };
__device__ __forceinline__ LossIn loss_in(const RowArgs& a, int64_t row) {
  return LossIn{a.logp_old[row], a.logp_ref ? a.logp_ref[row] : 0.f, a.adv[row], (a.weight ? a.weight[row] : 1.f) * a.scale};
}
__device__ __forceinline__ LossTerm loss_term(const RowArgs& a, const LossIn& in, float logp, float ent) {
  LossTerm o;
  const float lr = logp - in.old, rho = expf(lr);
  const float lo = 1.f - a.clip_lo, hi = 1.f + a.clip_hi;
  const float s1 = rho * in.adv, s2 = fminf(fmaxf(rho, lo), hi) * in.adv;
  const bool held = s1 > s2;  // ties: the unclipped branch carries the gradient; so does a NaN, which is to be seen in the loss
  o.rec.pi = (held ? -s2 : -s1) * in.w;
  o.g = held ? 0.f : -s1;
  o.rec.kl = 0.f;
  if (a.logp_ref) {
    const float d = in.ref - logp, em = expm1f(d);
    o.rec.kl = less_linear(em, d) * in.w;
    if (a.kl_coef != 0.f) o.g -= a.kl_coef * em;   // (it may be infinite where it only is reported)
  }
  o.rec.ent = ent * in.w;
  o.h = -a.ent_coef;
  o.rec.old_kl = less_linear(expm1f(lr), lr);
  o.rec.clipped = rho < lo || rho > hi ? 1.f : 0.f;
  o.rec.active = 1.f;
  o.g *= in.w; o.h *= in.w;
  return o;
}
// The record of a row and the coefficients of its gradient; one thread (writes) leaves the log-probability.
template <bool ENT>
__device__ __forceinline__ GradCoef loss_row(const RowArgs& a, int64_t row, const LossIn& in, const RowStat& r, float xt, bool writes, LossRecord* rec) {
  const RowOut o = row_out(r, xt, a.inv_t, ENT);
  const LossTerm l = loss_term(a, in, o.logp, o.ent);
  if (writes && a.logp) a.logp[row] = o.logp;
  *rec = l.rec;
  return grad_coef<ENT>(l.g, l.h, o.ent, o.ls, r.base(), 1.f / r.s, a.inv_t, xt);
}
template <class T>
__device__ __forceinline__ LossRecord loss_idle(const RowArgs& a, int64_t row, T* y, int n, int tid, int G, bool writes) {
  zero_row(y, n, tid, G);
  if (writes && a.logp) a.logp[row] = 0.f;
  return LossRecord{0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// Loss and gradient of rows of at most G K pieces by groups of G threads: the row stays in registers (as it is, 16 bits packed) between
// the passes that find the maximum, add up and write, so that memory sees it once in and once out.  Exponentials are made twice; 15
// vector instructions a logit of 16 bits, 21 with the entropy, keep the vector units busy for 0.65 of the time (16384 x 131072; 3001 x 50257).
template <class T, int G, int K, bool ENT>
__device__ __forceinline__ LossRecord loss_in_registers(const RowArgs& a, int64_t row, int tid, float* lds) {
  constexpr int N = Piece<T>::N;
  const int t = a.target[row], at = tid * N;
  const T* x = (const T*)a.logits + row * a.ld;
  T* y = (T*)a.dlogits + row * a.ldd;
  if (t < 0 || t >= a.vocab) return loss_idle(a, row, y, a.vocab, tid, G, tid == 0);
  const float c = a.inv_t * TOKEN_LOG2E;
  const LossIn in = loss_in(a, row);
  float xt = to_f(x[t]);
  const Cut w = cut_row(x, a.vocab, tid);
  const float xl = w.one >= 0 ? to_f(x[w.one]) : -INFINITY;
  Pieces<K> v;
  each<K>([&](auto k) INLINE { if (at + k * G * N < w.full) piece<k>(v) = load_piece(x + w.head + at + k * G * N); });
  asm volatile("" : "+v"(xt));   // read before the barrier: the gradient may lie in the logits' memory
  float m = xl;
  each<K>([&](auto k) INLINE { if (at + k * G * N < w.full) { m = fmaxf(m, max_piece<T>(piece<k>(v))); forget(piece<k>(v)); } });
  RowStat r = {lanes_max<G < 64 ? G : 64>(m), 0.f, 0.f};
  const float base = r.base();
  each<K>([&](auto k) INLINE { if (at + k * G * N < w.full) { add_piece<T, ENT>(r, piece<k>(v), base, c); forget(piece<k>(v)); } });
  if (w.one >= 0) add_one<ENT>(r, xl, base, c);
  r = group_join<G, ENT>(r, c, lds);
  if (r.idle()) return loss_idle(a, row, y, a.vocab, tid, G, tid == 0);
  LossRecord rec;
  const GradCoef q = loss_row<ENT>(a, row, in, r, xt, tid == 0, &rec);
  each<K>([&](auto k) INLINE { if (at + k * G * N < w.full) store_piece(y + w.head + at + k * G * N, grad_piece<T, ENT>(piece<k>(v), q)); });
  if (w.one >= 0) y[w.one] = from_f<T>(grad_one<ENT>(xl, q));
  // the target's element again, by the thread that wrote it with its piece
  if (owns<T, G>(w, t, tid)) y[t] = from_f<T>(q.target);
  return rec;
}
template <class T, int G, int K, bool ENT>
__global__ __launch_bounds__(G < 256 ? 256 : G, K >= 16 ? 4 : K == 8 ? 6 : K == 4 ? 4 : 8) void k_token_loss(RowArgs a) {
  constexpr int NT = G < 256 ? 256 : G;
  __shared__ float lds[3 * (NT / 64)];
  const int64_t row = (int64_t)blockIdx.x * (NT / G) + (G < 256 ? threadIdx.x / G : 0);
  if (G < 256 && row >= a.rows) return;   // G <= 64: no barrier follows
  const LossRecord rec = loss_in_registers<T, G, K, ENT>(a, row, threadIdx.x % G, lds);
  if (threadIdx.x % G == 0) ((LossRecord*)a.record)[row] = rec;
}

// The gradient of n elements by G threads; t: the target's place among them, if it is one of them.
template <class T, int G, bool ENT>
__device__ __forceinline__ void stream_gradient(const T* x, T* y, int n, int tid, const GradCoef& q, int t) {
  constexpr int N = Piece<T>::N, U = 4;
  const Cut w = cut_row(x, n, tid);
  const float xl = w.one >= 0 ? to_f(x[w.one]) : 0.f;
  for (int i = tid * N; i < w.full; i += G * N * U) {
    Pieces<U> v;
    each<U>([&](auto u) INLINE { if (i + u * G * N < w.full) piece<u>(v) = load_piece(x + w.head + i + u * G * N); });
    each<U>([&](auto u) INLINE { if (i + u * G * N < w.full) store_piece(y + w.head + i + u * G * N, grad_piece<T, ENT>(piece<u>(v), q)); });
  }
  if (w.one >= 0) y[w.one] = from_f<T>(grad_one<ENT>(xl, q));
  if (t >= 0 && t < n && owns<T, G>(w, t, tid)) y[t] = from_f<T>(q.target);
}

// Longer rows: read twice by a block (2048 x 152064 this way: 294 us, 252 in registers).
template <class T, bool ENT>
__global__ __launch_bounds__(1024) void k_token_loss_long(RowArgs a) {
  constexpr int G = 1024;
  __shared__ float lds[3 * (G / 64)];
  const int64_t row = blockIdx.x;
  const int t = a.target[row], tid = threadIdx.x;
  const T* x = (const T*)a.logits + row * a.ld;
  T* y = (T*)a.dlogits + row * a.ldd;
  RowStat r = {-INFINITY, 0.f, 0.f};
  const float c = a.inv_t * TOKEN_LOG2E;
  float xt = 0.f;
  LossIn in;
  if (t >= 0 && t < a.vocab) {
    in = loss_in(a, row);
    xt = to_f(x[t]);
    asm volatile("" : "+v"(xt));
    r = group_join<G, ENT>(stream_stat<T, G, ENT>(x, a.vocab, tid, c), c, lds);
  }
  LossRecord rec;
  if (r.idle()) rec = loss_idle(a, row, y, a.vocab, tid, G, tid == 0);
  else {
    const GradCoef q = loss_row<ENT>(a, row, in, r, xt, tid == 0, &rec);
    stream_gradient<T, G, ENT>(x, y, a.vocab, tid, q, t);
  }
  if (tid == 0) ((LossRecord*)a.record)[row] = rec;
}

// Few long rows: k_token_part has left the statistics of the slices; every slice's block joins them all and writes its gradient.
template <class T, bool ENT>
__global__ __launch_bounds__(256) void k_token_loss_slice(RowArgs a) {
  const int64_t row = blockIdx.y;
  const int t = a.target[row], tid = threadIdx.x, from = blockIdx.x * a.slice_len, n = min(a.vocab - from, a.slice_len);
  const T* x = (const T*)a.logits + row * a.ld + from;
  T* y = (T*)a.dlogits + row * a.ldd + from;
  const bool first = blockIdx.x == 0 && tid == 0;
  RowStat r = {-INFINITY, 0.f, 0.f};
  if (t >= 0 && t < a.vocab) r = join_parts<ENT>(a, row, a.inv_t * TOKEN_LOG2E);
  LossRecord rec;
  if (r.idle()) rec = loss_idle(a, row, y, n, tid, 256, first);
  else {
    const float xt = a.part[4 * row * a.slices + 3];
    const GradCoef q = loss_row<ENT>(a, row, loss_in(a, row), r, xt, first, &rec);
    stream_gradient<T, 256, ENT>(x, y, n, tid, q, t - from);
  }
  if (first) ((LossRecord*)a.record)[row] = rec;
}

// Statistics of the loss: the rows' records added in a fixed order, in 64 bits; `share` rows a block.  One block finishes
// by itself; of several, each leaves its sums for k_token_stats_join.
constexpr int STATS_ROWS = 4096;   // rows per block (more when there are more than 1024 such blocks)
__device__ __forceinline__ void write_stats(const double (&v)[6], float kl_coef, float ent_coef, float* stats) {
  // loss, pi, kl, entropy (weighted sums), mean approx_kl, clipped share, active rows, non-finite
  const double loss = v[0] + (kl_coef != 0.f ? (double)kl_coef * v[1] : 0.0) - (ent_coef != 0.f ? (double)ent_coef * v[2] : 0.0), n = v[5] > 0 ? v[5] : 1;
  stats[0] = (float)loss; stats[1] = (float)v[0]; stats[2] = (float)v[1]; stats[3] = (float)v[2];
  stats[4] = (float)(v[3] / n); stats[5] = (float)(v[4] / n); stats[6] = (float)v[5];
  stats[7] = isfinite((float)loss) ? 0.f : 1.f;
}
__global__ __launch_bounds__(1024) void k_token_stats(int64_t rows, int64_t share, const LossRecord* rec, float kl_coef, float ent_coef, float* stats, double* part) {
  __shared__ double lds[6 * 16];
  double v[6] = {0, 0, 0, 0, 0, 0};
  const int64_t from = blockIdx.x * share, to = from + share < rows ? from + share : rows;
  for (int64_t i = from + threadIdx.x; i < to; i += 4096) {
    LossRecord r[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = i + u * 1024 < to ? rec[i + u * 1024] : LossRecord{0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u) { v[0] += r[u].pi; v[1] += r[u].kl; v[2] += r[u].ent; v[3] += r[u].old_kl; v[4] += r[u].clipped; v[5] += r[u].active; }
  }
  block_sums<16>(v, lds);
  if (threadIdx.x) return;
  if (gridDim.x == 1) write_stats(v, kl_coef, ent_coef, stats);
  else
    for (int k = 0; k < 6; ++k) part[6 * blockIdx.x + k] = v[k];
}
__global__ __launch_bounds__(1024) void k_token_stats_join(int blocks, float kl_coef, float ent_coef, float* stats, const double* part) {
  __shared__ double lds[6 * 16];
  double v[6];
  for (int k = 0; k < 6; ++k) v[k] = (int)threadIdx.x < blocks ? part[6 * threadIdx.x + k] : 0.0;
  block_sums<16>(v, lds);
  if (threadIdx.x == 0) write_stats(v, kl_coef, ent_coef, stats);
}

// A few short rows by one block, statistics included (64 rows a turn): one launch and no workspace where these are what a call costs.
// us a call among others, this way and with two launches: 4 x 64 6.5 and 10.5, 32 x 512 6.5 and 10.5, 64 x 256 7.0 and 10.6, 128 x 128 8.6 and
// 10.5; 64 x 512 8.9 and 10.5, 128 x 256 10.3 and 10.5, 128 x 512 14.3 and 10.6.  A call alone takes 18.0 and 20.8 (16 x 512),
// 21.6 and 20.8 (128 x 128), 22.0 and 20.7 (64 x 512).
constexpr int SMALL_ROWS = 128, SMALL_VOCAB = 512, SMALL_LOGITS = 16384;
template <class T, int K, bool ENT>
__global__ __launch_bounds__(1024) void k_token_loss_small(RowArgs a, float* stats) {
  __shared__ double lds[6 * 16];
  double v[6] = {0, 0, 0, 0, 0, 0};
  for (int64_t row = threadIdx.x / 16; row < a.rows; row += 64) {
    const LossRecord r = loss_in_registers<T, 16, K, ENT>(a, row, threadIdx.x % 16, nullptr);
    if (threadIdx.x % 16 == 0) { v[0] += r.pi; v[1] += r.kl; v[2] += r.ent; v[3] += r.old_kl; v[4] += r.clipped; v[5] += r.active; }
  }
  block_sums<16>(v, lds);
  if (threadIdx.x == 0) write_stats(v, a.kl_coef, a.ent_coef, stats);
}
