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
  struct PairRecord* record;
};
struct PairRecord { double loss, right, margin, chosen, rejected, active; };

// v: the same in every lane of a wave
__device__ __forceinline__ double block_sum_waves(double v, double* lds) {
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) v += lds[w];
  __syncthreads();
  return v;
}
__device__ __forceinline__ double block_sum_d(double v, double* lds) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return block_sum_waves(v, lds);
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

// What a launch of the two kernels below knows of the grid: a sequence is worked on by `slices` groups of G threads, four tokens a
// thread at a time; a group per wave (G = 64) for short sequences, per block (G = 256) for long ones.
struct PairGrid {
  int32_t slices;
  double2* part;       // [2 * pairs][slices]: sum of an unmasked sequence's terms, and how many
};
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint8_t u8x4_any_t __attribute__((ext_vector_type(4), aligned(1)));
// mask of the tokens i .. i + 3 (1: counts), those from `to` on 0
__device__ __forceinline__ void mask4(const uint8_t* mask, int64_t i, int64_t to, bool (&on)[4]) {
  if (!mask) {
#pragma unroll
    for (int k = 0; k < 4; ++k) on[k] = i + k < to;
  } else if (i + 4 <= to) {
    const u8x4_any_t m = *reinterpret_cast<const u8x4_any_t*>(mask + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) on[k] = m[k] != 0;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) on[k] = i + k < to && mask[i + k] != 0;
  }
}
__device__ __forceinline__ void load4(const float* p, int64_t i, int64_t to, float (&f)[4]) {
  if (i + 4 <= to) {
    const f32x4_any_t v = *reinterpret_cast<const f32x4_any_t*>(p + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = v[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = i + k < to ? p[i + k] : 0.f;
  }
}
__device__ __forceinline__ void store4(float* p, int64_t i, int64_t to, const float (&f)[4]) {
  if (i + 4 <= to) *reinterpret_cast<f32x4_any_t*>(p + i) = f32x4_any_t{f[0], f[1], f[2], f[3]};
  else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < to) p[i + k] = f[k];
  }
}

template <int G>
__global__ __launch_bounds__(256) void k_pair_sums(PairArgs a, PairGrid g) {
  __shared__ double lds[4];
  const int64_t item = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;   // a sequence's slice
  if (G == 64 && item >= 2 * a.pairs * g.slices) return;
  const int64_t s = item / g.slices;
  const int slice = (int)(item - s * g.slices);
  const int64_t from = hold(a.offsets[s], a.tokens), to = hold(a.offsets[s + 1], a.tokens);
  double v = 0;
  int c = 0;
  for (int64_t i = from + ((int64_t)slice * G + threadIdx.x % G) * 4; i < to; i += (int64_t)g.slices * G * 4) {
    float x[4], r[4] = {0.f, 0.f, 0.f, 0.f};
    bool on[4];
    load4(a.logp, i, to, x);
    if (a.ref) load4(a.ref, i, to, r);
    mask4(a.mask, i, to, on);
#pragma unroll
    for (int k = 0; k < 4; ++k) { v += on[k] ? (double)x[k] - (double)r[k] : 0.0; c += on[k]; }
  }
  double n = c;
  for (int o = 32; o; o >>= 1) { v += __shfl_xor(v, o); n += __shfl_xor(n, o); }
  if (G > 64) {
    v = block_sum_waves(v, lds);
    n = block_sum_waves(n, lds);
  }
  if (threadIdx.x % G == 0) g.part[item] = make_double2(v, n);
}

// S and number of unmasked tokens of a sequence, by every lane of a wave
__device__ __forceinline__ double2 pair_sum(const PairGrid& g, int64_t s) {
  double v = 0, n = 0;
  for (int k = threadIdx.x & 63; k < g.slices; k += 64) { const double2 p = g.part[s * g.slices + k]; v += p.x; n += p.y; }
  for (int o = 32; o; o >>= 1) { v += __shfl_xor(v, o); n += __shfl_xor(n, o); }
  return make_double2(v, n);
}

// Gradient (and record) of the pairs.
template <int G>
__global__ __launch_bounds__(256) void k_pair_loss(PairArgs a, PairGrid g) {
  const int64_t first = hold(a.offsets[0], a.tokens), last = hold(a.offsets[2 * a.pairs], a.tokens);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < first + (a.tokens - last); i += (int64_t)gridDim.x * 256)
    a.dlogp[i < first ? i : last + (i - first)] = 0.f;   // tokens of no sequence
  const int64_t item = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
  if (item >= 2 * a.pairs * g.slices) return;
  const int64_t s = item / g.slices;
  const int slice = (int)(item - s * g.slices);
  const int64_t k = s < a.pairs ? s : s - a.pairs;
  const double2 won = pair_sum(g, k), lost = pair_sum(g, k + a.pairs);
  const bool on = won.y > 0 && lost.y > 0;
  const double f[2] = {a.mean && on ? 1 / won.y : 1.0, a.mean && on ? 1 / lost.y : 1.0};
  const double S[2] = {won.x * f[0], lost.x * f[1]}, D = S[0] - S[1];
  double loss = 0, slope = 0;
  if (on) pair_term(a.kind, a.beta, a.smoothing, D, &loss, &slope);
  slope *= a.scale;
  const float grad = on ? (float)(s < a.pairs ? slope * f[0] : -slope * f[1]) : 0.f;
  const int64_t from = hold(a.offsets[s], a.tokens), to = hold(a.offsets[s + 1], a.tokens);
  for (int64_t i = from + ((int64_t)slice * G + threadIdx.x % G) * 4; i < to; i += (int64_t)g.slices * G * 4) {
    bool m[4];
    float d[4];
    mask4(a.mask, i, to, m);
#pragma unroll
    for (int q = 0; q < 4; ++q) d[q] = m[q] ? grad : 0.f;
    store4(a.dlogp, i, to, d);
  }
  if (s < a.pairs && slice == 0 && threadIdx.x % G == 0) {
    const double b = a.beta;
    if (a.margin) a.margin[k] = on ? (float)(b * D) : 0.f;
    a.record[k] = on ? PairRecord{loss, D > 0 ? 1.0 : 0.0, b * D, b * S[0], b * S[1], 1.0} : PairRecord{0, 0, 0, 0, 0, 0};
  }
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
// changes; the last token of a sequence first replaces the pair by (0, last value)), and maps of this form compose.  The tokens
// are cut into tiles without regard to the sequences, so that the work is even whatever their lengths: k_gae_part composes the
// maps of a tile, k_gae_tiles the tiles' maps from the end, k_token_gae applies what comes in to a tile's tokens.  With few tiles
// the last one looks at the maps behind it by itself, and one tile needs nothing else.  A sum over a long sequence (gamma lambda
// = 1) is held in 64 bits; 16 bytes a token move, so that the arithmetic does not show.
constexpr int GAE_PER = 8, GAE_TILE = 256 * GAE_PER;   // tokens per thread and per tile
constexpr int GAE_DIRECT = 512;                        // at most so many tiles are looked at directly
struct GaeMap { double a, b, c, v; int32_t flags, pad; };     // flags: 1 = V -> v (else V stays), 2 = nothing from behind matters
struct GaeArgs {
  int64_t sequences, tokens;
  const float *reward, *value, *last_value;  // last_value: may be NULL
  const uint8_t* mask;                       // may be NULL
  const int64_t* offsets;
  double gamma, lambda;
  float *adv, *ret;
  int64_t tiles;
  GaeMap* map;                               // [tiles]
  double2* in;                               // [tiles] the pair (A, V) that enters a tile; NULL: direct
};
__device__ __forceinline__ GaeMap gae_nothing() { return GaeMap{1, 0, 0, 0, 0, 0}; }
// first `behind`, then `m`
__device__ __forceinline__ GaeMap then(const GaeMap& behind, const GaeMap& m) {
  if (m.flags & 2) return m;
  GaeMap o;
  const bool set = behind.flags & 1;
  o.a = m.a * behind.a;
  o.b = m.a * behind.b + (set ? 0.0 : m.b);
  o.c = m.a * behind.c + (set ? m.b * behind.v : 0.0) + m.c;
  o.v = m.flags & 1 ? m.v : behind.v;
  o.flags = m.flags | behind.flags;
  o.pad = 0;
  return o;
}
__device__ __forceinline__ GaeMap shfl_down_map(const GaeMap& m, int o) {
  return GaeMap{__shfl_down(m.a, o), __shfl_down(m.b, o), __shfl_down(m.c, o), __shfl_down(m.v, o), __shfl_down(m.flags, o), 0};
}
// lane l: the maps of the lanes 63 .. l, composed
__device__ __forceinline__ GaeMap wave_suffix(GaeMap m) {
  const int lane = threadIdx.x & 63;
  for (int o = 1; o < 64; o <<= 1) {
    const GaeMap b = shfl_down_map(m, o);
    if (lane + o < 64) m = then(b, m);
  }
  return m;
}
// The maps of all threads behind this one in the block, composed; *whole: those of the block.
template <int NW>
__device__ __forceinline__ GaeMap block_behind(const GaeMap& mine, GaeMap* lds, GaeMap* whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const GaeMap suf = wave_suffix(mine);
  if (lane == 0) lds[wave] = suf;
  __syncthreads();
  GaeMap behind = gae_nothing(), all = gae_nothing();
  for (int w = NW - 1; w >= 0; --w) {
    if (w == wave) behind = all;
    all = then(all, lds[w]);
  }
  if (whole) *whole = all;
  const GaeMap next = shfl_down_map(suf, 1);
  return lane < 63 ? then(behind, next) : behind;
}

// The first k of [0, n) with offsets[k] > at (n: none), by the lanes of a wave together: 64 places are looked at per step.
__device__ __forceinline__ int64_t first_above(const int64_t* offsets, int64_t n, int64_t tokens, int64_t at) {
  int64_t lo = 0, hi = n;   // the answer lies in [lo, hi]
  while (lo < hi) {
    const int64_t step = (hi - lo + 63) / 64, k = lo + (threadIdx.x & 63) * step;
    const uint64_t above = __ballot(k >= hi || hold(offsets[k], tokens) > at);
    const int f = above ? __ffsll((unsigned long long)above) - 1 : 64;   // the first lane whose place is above
    const int64_t nhi = lo + f * step < hi ? lo + f * step : hi;
    lo = f ? lo + (f - 1) * step + 1 : lo;
    hi = nhi;
  }
  return lo;
}

// A tile's tokens in registers: eight in a row per thread.
struct GaeTile {
  float r[GAE_PER], v[GAE_PER];
  uint32_t on, in;          // bit k: the token counts; it lies in a sequence
  int32_t end[GAE_PER];     // 1 + its sequence, if it is that one's last token; else 0
};
__device__ __forceinline__ void gae_load(const GaeArgs& a, int64_t tile, int32_t* ends, GaeTile& t) {
  const int64_t start = tile * GAE_TILE, stop = start + GAE_TILE < a.tokens ? start + GAE_TILE : a.tokens;
  const int64_t i = start + threadIdx.x * GAE_PER;
  t.on = t.in = 0;
#pragma unroll
  for (int h = 0; h < GAE_PER; h += 4) {
    bool on[4];
    float r[4], v[4];
    mask4(a.mask, i + h, stop, on);
    load4(a.reward, i + h, stop, r);
    load4(a.value, i + h, stop, v);
#pragma unroll
    for (int k = 0; k < 4; ++k) { t.r[h + k] = r[k]; t.v[h + k] = v[k]; t.on |= (uint32_t)on[k] << (h + k); }
  }
  for (int k = threadIdx.x; k < GAE_TILE; k += 256) ends[k] = 0;
  __syncthreads();
  const int64_t first = a.sequences ? hold(a.offsets[0], a.tokens) : a.tokens, last = hold(a.offsets[a.sequences], a.tokens);
  for (int64_t j = first_above(a.offsets, a.sequences + 1, a.tokens, start) + threadIdx.x; j <= a.sequences; j += 256) {
    const int64_t o = hold(a.offsets[j], a.tokens);
    if (o > start + GAE_TILE) break;
    if (j > 0 && o > start && o > hold(a.offsets[j - 1], a.tokens)) ends[o - 1 - start] = (int32_t)j;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < GAE_PER; ++k) {
    t.end[k] = ends[threadIdx.x * GAE_PER + k];
    t.in |= (uint32_t)(i + k >= first && i + k < last) << k;
  }
  t.on &= t.in;
}
__device__ __forceinline__ double gae_last(const GaeArgs& a, int32_t end) { return a.last_value ? (double)a.last_value[end - 1] : 0.0; }
// the map of a thread's tokens
__device__ __forceinline__ GaeMap gae_map(const GaeArgs& a, const GaeTile& t) {
  GaeMap m = gae_nothing();
  const double gl = a.gamma * a.lambda;
#pragma unroll
  for (int k = GAE_PER - 1; k >= 0; --k) {
    if (t.end[k]) m = GaeMap{0, 0, 0, gae_last(a, t.end[k]), 3, 0};
    if (t.on >> k & 1) {
      const bool set = m.flags & 1;
      const double v = t.v[k];
      m.c = gl * m.c + (set ? a.gamma * m.v : 0.0) + ((double)t.r[k] - v);
      m.b = gl * m.b + (set ? 0.0 : a.gamma);
      m.a *= gl;
      m.v = v;
      m.flags |= 1;
    }
  }
  return m;
}
__device__ __forceinline__ double2 gae_apply(const GaeMap& m, double2 in) {
  if (m.flags & 2) return make_double2(m.c, m.v);
  return make_double2(m.a * in.x + m.b * in.y + m.c, m.flags & 1 ? m.v : in.y);
}

__global__ __launch_bounds__(256) void k_gae_part(GaeArgs a) {
  __shared__ int32_t ends[GAE_TILE];
  __shared__ GaeMap lds[4];
  GaeTile t;
  gae_load(a, blockIdx.x, ends, t);
  GaeMap whole;
  block_behind<4>(gae_map(a, t), lds, &whole);
  if (threadIdx.x == 0) a.map[blockIdx.x] = whole;
}

__global__ __launch_bounds__(1024) void k_gae_tiles(GaeArgs a) {
  __shared__ GaeMap lds[16];
  double2 carry = make_double2(0, 0);
  for (int64_t from = (a.tiles - 1) / 1024 * 1024; from >= 0; from -= 1024) {
    const int64_t k = from + threadIdx.x;
    GaeMap whole;
    const GaeMap behind = block_behind<16>(k < a.tiles ? a.map[k] : gae_nothing(), lds, &whole);
    if (k < a.tiles) a.in[k] = gae_apply(behind, carry);
    carry = gae_apply(whole, carry);
    __syncthreads();   // lds is written again
  }
}

__global__ __launch_bounds__(256) void k_token_gae(GaeArgs a) {
  __shared__ int32_t ends[GAE_TILE];
  __shared__ GaeMap lds[4];
  const int64_t tile = blockIdx.x;
  double2 in = make_double2(0, 0);
  if (a.in) in = a.in[tile];
  else {
    GaeMap m = gae_nothing();
    for (int64_t k = tile + 1; k < a.tiles && !(m.flags & 2); k += 64) {
      const int64_t j = k + (threadIdx.x & 63);
      const GaeMap far = wave_suffix(j < a.tiles ? a.map[j] : gae_nothing());
      m = then(GaeMap{__shfl(far.a, 0), __shfl(far.b, 0), __shfl(far.c, 0), __shfl(far.v, 0), __shfl(far.flags, 0), 0}, m);
    }
    in = gae_apply(m, in);
  }
  GaeTile t;
  gae_load(a, tile, ends, t);
  in = gae_apply(block_behind<4>(gae_map(a, t), lds, nullptr), in);
  double A = in.x, V = in.y;
  const double gl = a.gamma * a.lambda;
  float adv[GAE_PER], ret[GAE_PER];
#pragma unroll
  for (int k = GAE_PER - 1; k >= 0; --k) {
    if (t.end[k]) { A = 0; V = gae_last(a, t.end[k]); }
    const bool on = t.on >> k & 1;
    const double v = t.v[k];
    if (on) { A = gl * A + a.gamma * V + ((double)t.r[k] - v); V = v; }
    adv[k] = on ? (float)A : 0.f;
    ret[k] = on ? (float)(A + v) : 0.f;
  }
  const int64_t i = tile * GAE_TILE + threadIdx.x * GAE_PER;
#pragma unroll
  for (int h = 0; h < GAE_PER; h += 4) {
    const float x[4] = {adv[h], adv[h + 1], adv[h + 2], adv[h + 3]}, y[4] = {ret[h], ret[h + 1], ret[h + 2], ret[h + 3]};
    store4(a.adv, i + h, a.tokens, x);
    store4(a.ret, i + h, a.tokens, y);
  }
}
