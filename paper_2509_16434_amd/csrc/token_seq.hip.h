// Sequences packed one behind the other: sequence k holds the tokens [offsets[k], offsets[k+1]).  Offsets are held inside
// [0, tokens] before they are used, so that a wrong one cannot reach memory outside the arrays.
#pragma once
#include "lanes.hip.h"

__device__ __forceinline__ int64_t hold(int64_t o, int64_t tokens) { return o < 0 ? 0 : o > tokens ? tokens : o; }

// ---------------------------------------------------------------- preference loss
// Pairs (k, pairs + k) of a chosen and a rejected sequence.  S = sum over the unmasked tokens of (logp - ref) (or their mean),
// D = S_chosen - S_rejected; loss of a pair -(1 - ls) log sigmoid(bD) - ls log sigmoid(-bD), or (D - 1/(2b))^2.  D is a small
// difference of long sums: they are held in 64 bits.  A pair with no unmasked token in one of its sequences adds nothing.
// 13 bytes a token move; what a call costs is its two launches and the latency of the longest sequence's chain of loads
// (2 M tokens in 512 sequences of uneven length: 7.6 us for the sums, 8.5 for the gradient; 4 and 2 at the rate of a copy).
struct PairArgs {
  int64_t pairs, tokens;
  const float *logp, *ref;   // ref: may be NULL
  const uint8_t* mask;       // may be NULL
  const int64_t* offsets;    // [2 * pairs + 1]
  int32_t kind, mean;
  float beta, smoothing, scale;
  float *dlogp, *margin;
  struct PairRecord* record; // [pairs]; NULL: k_pair_loss finishes the statistics by itself
  float* stats;
};
struct PairRecord { double loss, right, margin, chosen, rejected, active; };

// loss of a pair, and its derivative by D
__device__ __forceinline__ double pair_value(int kind, double beta, double ls, double D) {
  if (kind != 0) { const double e = D - 0.5 / beta; return e * e; }
  const double x = beta * D, soft = log1p(exp(-fabs(x)));             // -log sigmoid(|x|)
  // a term whose weight is 0 may be infinite (D is where a token's log-probability is)
  return (ls < 1 ? (1 - ls) * (soft + (x < 0 ? -x : 0)) : 0) + (ls > 0 ? ls * (soft + (x > 0 ? x : 0)) : 0);
}
__device__ __forceinline__ double pair_slope(int kind, double beta, double ls, double D) {
  return kind != 0 ? 2 * (D - 0.5 / beta) : beta * (ls - 1 / (1 + exp(beta * D)));
}

// What a launch of the two kernels below knows of the grid: a sequence is worked on by `slices` groups of G threads, four tokens a
// thread at a time; blocks of G = 256, and G = 16 or 64 threads where there are many short sequences (200000 of 10 tokens: 156 us by
// waves, 48 by 16 threads; one that is long among them takes a thread's chain of loads of its length / 4 G).
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
  __shared__ double lds[8];
  const int64_t item = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;   // a sequence's slice
  if (G < 256 && item >= 2 * a.pairs * g.slices) return;
  const int64_t s = g.slices == 1 ? item : item / g.slices;
  const int slice = (int)(item - s * g.slices);
  const int64_t from = hold(a.offsets[s], a.tokens), to = hold(a.offsets[s + 1], a.tokens);
  double v = 0;
  int c = 0;
  // groups of four tokens between boundaries of four, so that all but the arrays' last one are read whole
  const int64_t step = (int64_t)g.slices * G * 4;
  for (int64_t i = (from & ~(int64_t)3) + ((int64_t)slice * G + threadIdx.x % G) * 4; i < to; i += step) {
    float x[4], r[4] = {0.f, 0.f, 0.f, 0.f};
    bool on[4];
    load4(a.logp, i, a.tokens, x);
    if (a.ref) load4(a.ref, i, a.tokens, r);
    mask4(a.mask, i, a.tokens, on);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool count = on[k] && i + k >= from && i + k < to;
      v += count ? (double)x[k] - (double)r[k] : 0.0;
      c += count;
    }
  }
  double sums[2] = {v, (double)c};
  if constexpr (G < 64) { sums[0] = lanes_sum<G>(sums[0]); sums[1] = lanes_sum<G>(sums[1]); }
  else block_sums<G / 64>(sums, lds);
  if (threadIdx.x % G == 0) g.part[item] = make_double2(sums[0], sums[1]);
}

// S and number of unmasked tokens of a sequence, by every lane of a wave
__device__ __forceinline__ double2 pair_sum(const PairGrid& g, int64_t s) {
  if (g.slices == 1) return g.part[s];
  double v = 0, n = 0;
  for (int k = threadIdx.x & 63; k < g.slices; k += 64) { const double2 p = g.part[s * g.slices + k]; v += p.x; n += p.y; }
  return make_double2(lanes_sum<64>(v), lanes_sum<64>(n));
}

__device__ __forceinline__ PairRecord pair_record(const PairArgs& a, const double (&S)[2], bool on) {
  const double b = a.beta, D = S[0] - S[1];
  if (!on) return PairRecord{0, 0, 0, 0, 0, 0};
  return PairRecord{pair_value(a.kind, b, a.smoothing, D), D > 0 ? 1.0 : 0.0, b * D, b * S[0], b * S[1], 1.0};
}
// stats: loss, share of pairs with D > 0, mean margin, mean chosen and rejected reward, active pairs, non-finite
__device__ __forceinline__ void write_pair_stats(const double (&v)[6], float scale, float* stats) {
  const double n = v[5] > 0 ? v[5] : 1;
  stats[0] = (float)(v[0] * scale);
  for (int k = 1; k < 5; ++k) stats[k] = (float)(v[k] / n);
  stats[5] = (float)v[5];
  stats[6] = isfinite(stats[0]) ? 0.f : 1.f;
}
// The statistics (and margins) of at most PAIRS_INLINE pairs by one block: L lanes per sequence add up its slices' sums, then a thread
// does a pair.  Saves a launch where launches are what a call costs.
constexpr int PAIRS_INLINE = 256;
__device__ __forceinline__ void pair_stats_block(const PairArgs& a, const PairGrid& g) {
  __shared__ double2 sum[2 * PAIRS_INLINE];
  __shared__ double lds[6 * 4];
  const int n = 2 * (int)a.pairs;
  int L = 64;
  while (L > 1 && L * n > 256) L >>= 1;
  for (int s0 = 0; s0 < n; s0 += 256 / L) {
    const int s = s0 + (int)threadIdx.x / L;
    double v = 0, c = 0;
    if (s < n)
      for (int k = threadIdx.x & (L - 1); k < g.slices; k += L) { const double2 p = g.part[(int64_t)s * g.slices + k]; v += p.x; c += p.y; }
    for (int o = L >> 1; o; o >>= 1) { v += __shfl_xor(v, o); c += __shfl_xor(c, o); }
    if (s < n && (threadIdx.x & (L - 1)) == 0) sum[s] = make_double2(v, c);
  }
  __syncthreads();
  PairRecord r = {0, 0, 0, 0, 0, 0};
  if ((int)threadIdx.x < a.pairs) {
    const double2 won = sum[threadIdx.x], lost = sum[threadIdx.x + a.pairs];
    const bool on = won.y > 0 && lost.y > 0;
    const double S[2] = {a.mean && on ? won.x / won.y : won.x, a.mean && on ? lost.x / lost.y : lost.x};
    r = pair_record(a, S, on);
    if (a.margin) a.margin[threadIdx.x] = (float)r.margin;
  }
  double v[6] = {r.loss, r.right, r.margin, r.chosen, r.rejected, r.active};
  block_sums<4>(v, lds);
  if (threadIdx.x == 0) write_pair_stats(v, a.scale, a.stats);
}

// Gradient and records of the pairs; without room for records, one more block does the statistics.
template <int G>
__global__ __launch_bounds__(256) void k_pair_loss(PairArgs a, PairGrid g) {
  const int64_t blocks = gridDim.x - (a.record ? 0 : 1);
  if (blockIdx.x == blocks) { pair_stats_block(a, g); return; }
  const int64_t first = hold(a.offsets[0], a.tokens), last = hold(a.offsets[2 * a.pairs], a.tokens);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < first + (a.tokens - last); i += blocks * 256)
    a.dlogp[i < first ? i : last + (i - first)] = 0.f;   // tokens of no sequence
  const int64_t item = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
  if (item >= 2 * a.pairs * g.slices) return;
  const int64_t s = g.slices == 1 ? item : item / g.slices;
  const int slice = (int)(item - s * g.slices);
  const int64_t k = s < a.pairs ? s : s - a.pairs;
  const double2 won = pair_sum(g, k), lost = pair_sum(g, k + a.pairs);
  const bool on = won.y > 0 && lost.y > 0;
  const double f[2] = {a.mean && on ? 1 / won.y : 1.0, a.mean && on ? 1 / lost.y : 1.0};
  const double S[2] = {won.x * f[0], lost.x * f[1]}, D = S[0] - S[1];
  const double slope = pair_slope(a.kind, a.beta, a.smoothing, D) * a.scale;
  const float grad = on ? (float)(s < a.pairs ? slope * f[0] : -slope * f[1]) : 0.f;
  const int64_t from = hold(a.offsets[s], a.tokens), to = hold(a.offsets[s + 1], a.tokens);
  const int64_t step = (int64_t)g.slices * G * 4;
  for (int64_t i = (from & ~(int64_t)3) + ((int64_t)slice * G + threadIdx.x % G) * 4; i < to; i += step) {
    bool m[4];
    float d[4];
    mask4(a.mask, i, a.tokens, m);
#pragma unroll
    for (int q = 0; q < 4; ++q) d[q] = m[q] ? grad : 0.f;
    if (i >= from && i + 4 <= to) store4(a.dlogp, i, to, d);
    else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (i + q >= from && i + q < to) a.dlogp[i + q] = d[q];
    }
  }
  if (a.record && s < a.pairs && slice == 0 && threadIdx.x % G == 0) {
    const PairRecord r = pair_record(a, S, on);
    if (a.margin) a.margin[k] = (float)r.margin;
    a.record[k] = r;
  }
}

// More pairs: their records, `share` of them per block; several blocks leave their sums for k_pair_stats_join.
__global__ __launch_bounds__(1024) void k_pair_stats(int64_t pairs, int64_t share, const PairRecord* rec, float scale, float* stats, double* part) {
  __shared__ double lds[6 * 16];
  double v[6] = {0, 0, 0, 0, 0, 0};
  const int64_t from = blockIdx.x * share, to = from + share < pairs ? from + share : pairs;
  for (int64_t i = from + threadIdx.x; i < to; i += 1024) {
    const PairRecord r = rec[i];
    v[0] += r.loss; v[1] += r.right; v[2] += r.margin; v[3] += r.chosen; v[4] += r.rejected; v[5] += r.active;
  }
  block_sums<16>(v, lds);
  if (threadIdx.x) return;
  if (gridDim.x == 1) write_pair_stats(v, scale, stats);
  else
    for (int k = 0; k < 6; ++k) part[6 * blockIdx.x + k] = v[k];
}
__global__ __launch_bounds__(1024) void k_pair_stats_join(int blocks, float scale, float* stats, const double* part) {
  __shared__ double lds[6 * 16];
  double v[6];
  for (int k = 0; k < 6; ++k) v[k] = (int)threadIdx.x < blocks ? part[6 * threadIdx.x + k] : 0.0;
  block_sums<16>(v, lds);
  if (threadIdx.x == 0) write_pair_stats(v, scale, stats);
}

// ---------------------------------------------------------------- advantages
// A_t = r_t + gamma V' - V_t + gamma lambda A', where the primes are the next unmasked token of the sequence; behind the last
// one V' is the sequence's last value (0 without one) and A' = 0.  R_t = A_t + V_t.  Masked tokens get 0.
//
// The tokens are cut into tiles without regard to the sequences, so that the work is even whatever their lengths.  A thread has
// eight tokens in a row.  The V' of a thread's last token is the value in front of the nearest thread behind it that has an unmasked
// token or the end of a sequence (a ballot finds it).  Then the tokens are maps A -> a A + c (masked ones: 1 and 0; the last token of a
// sequence first replaces what comes in by 0), maps of this form compose, and a scan from the end gives every thread what comes in.
// Of a tile as a whole, what comes from behind also enters through V': its map is A -> a A + b V + c, V -> v (or V).  k_gae_part
// makes the tiles' maps, k_gae_tiles scans them, k_token_gae does the tokens; with few tiles the last one scans the maps behind its
// own by itself, and one tile needs nothing else.  A sum over a long sequence (gamma lambda = 1) is held in 64 bits.
//
// Bound: 16 to 17 bytes a token, the inputs twice (from the last-level cache the second time) where there is more than one tile:
// 3 M tokens 9.8 + 14.6 us, 11 at the rate of a copy; 200000 tokens 5.2 + 6.4 us, which is latency.
constexpr int GAE_PER = 8, GAE_TILE = 256 * GAE_PER;   // tokens per thread and per tile
// At most so many tiles (8.4 M tokens) are scanned directly.  What that costs goes by how far the ends of sequences lie apart, which the host does
// not know: us a call directly and with k_gae_tiles, one sequence: 3 M tokens 26 and 32, 6 M 57 and 54, 8.3 M 85 and 68, 16 M 222 and 120,
// 33 M 774 and 253; 24 sequences: 3 M 23 and 32, 8.3 M 50 and 68, 16 M 84 and 120, 33 M 198 and 253.
constexpr int GAE_DIRECT = 4096;
struct GaeMap { double a, b, c; float v; int32_t set, stop, offset; };   // set: V -> v, else V stays; stop: nothing from behind
                                                                       // matters; offset: first_above at the tile's start
struct GaeArgs {
  int64_t sequences, tokens;
  const float *reward, *value, *last_value;  // last_value: may be NULL
  const uint8_t* mask;                       // may be NULL
  const int64_t* offsets;
  double gamma, lambda;
  float *adv, *ret;
  int64_t tiles;
  GaeMap* map;                               // [tiles]
  double2* in;                               // [tiles] the pair (A, V) that enters a tile (V a number of 32 bits); NULL: direct
};
// A -> a A + c; with a = 0 nothing of A matters, not even NaN: another sequence's is not to be seen
struct Affine { double a, c; };
__device__ __forceinline__ double apply(const Affine& m, double A) { return m.a == 0 ? m.c : m.a * A + m.c; }
__device__ __forceinline__ Affine then(const Affine& behind, const Affine& m) { return Affine{m.a * behind.a, apply(m, behind.c)}; }
template <int N> __device__ __forceinline__ double row_down(double old, double v) {   // of lane + N of the same 16, else `old`
  const int lo = __builtin_amdgcn_update_dpp(__double2loint(old), __double2loint(v), DPP_ROW_SHL(N), 0xf, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(__double2hiint(old), __double2hiint(v), DPP_ROW_SHL(N), 0xf, 0xf, false);
  return __hiloint2double(hi, lo);
}
template <int N> __device__ __forceinline__ Affine suffix_step(const Affine& m) {
  return then(Affine{row_down<N>(1.0, m.a), row_down<N>(0.0, m.c)}, m);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
// What the threads behind this one (in a block of NW waves) do to A; *whole: what the block does.  One barrier.
template <int NW>
__device__ __forceinline__ Affine block_behind(const Affine& mine, Affine* lds, Affine* whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Affine m = mine;                          // on the way: the lanes of the same 16 from this one on
  m = suffix_step<1>(m); m = suffix_step<2>(m); m = suffix_step<4>(m); m = suffix_step<8>(m);
  const Affine r3 = {lane_value(m.a, 48), lane_value(m.c, 48)};
  const Affine r2 = then(r3, Affine{lane_value(m.a, 32), lane_value(m.c, 32)});
  const Affine r1 = then(r2, Affine{lane_value(m.a, 16), lane_value(m.c, 16)});
  const Affine one = {1.0, 0.0};
  const Affine far = lane >= 48 ? one : lane >= 32 ? r3 : lane >= 16 ? r2 : r1;
  m = then(far, m);                         // the lanes of the wave from this one on
  if (lane == 0) lds[wave] = m;
  __syncthreads();
  Affine behind = one, all = one;
#pragma unroll 4
  for (int w = NW - 1; w >= 0; --w) {
    if (w == wave) behind = all;
    all = then(all, lds[w]);
  }
  if (whole) *whole = all;
  const Affine next = {__shfl_down(m.a, 1), __shfl_down(m.c, 1)};
  return lane < 63 ? then(behind, next) : behind;
}
// The value that enters a thread from behind: that in front of the nearest thread behind it which has one (set), or `in`.  *front, *any:
// what leaves the block, and whether it is the block's own.  One barrier.
template <int NW>
__device__ __forceinline__ float block_value(bool set, float v, float in, float* lds_v, int* lds_set, float* front, bool* any) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t who = __ballot(set);
  if (set && lane == __ffsll((unsigned long long)who) - 1) lds_v[wave] = v;
  if (lane == 0) lds_set[wave] = who != 0;
  __syncthreads();
  const uint64_t above = lane == 63 ? 0 : who >> (lane + 1);
  const float near = __shfl(v, above ? lane + __ffsll((unsigned long long)above) : 0);
  float x = in, out = in;
  bool found = false;
#pragma unroll 4
  for (int w = NW - 1; w >= 0; --w) {
    if (w == wave) x = out;
    if (lds_set[w]) { out = lds_v[w]; found = true; }
  }
  if (front) { *front = out; *any = found; }
  return above ? near : x;
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
  float last[GAE_PER];      // the last value of the sequence that ends with the token
  uint32_t on, end;         // bit k: the token counts; it is a sequence's last one
};
// What ends in a tile: a bit per token, and the last values where one is set.
struct GaeEnds { uint32_t bits[GAE_TILE / 32]; float last[GAE_TILE]; };
// offset: first_above at the tile's start, or -1: it is looked for, and returned.  Two barriers.
__device__ __forceinline__ int64_t gae_load(const GaeArgs& a, int64_t tile, int64_t offset, GaeEnds& ends, GaeTile& t) {
  const int64_t start = tile * GAE_TILE, i = start + threadIdx.x * GAE_PER;
  t.on = 0;
  if (start + GAE_TILE <= a.tokens) {   // all but the last tile
#pragma unroll
    for (int h = 0; h < GAE_PER; h += 4) {
      const f32x4_any_t r = *reinterpret_cast<const f32x4_any_t*>(a.reward + i + h), v = *reinterpret_cast<const f32x4_any_t*>(a.value + i + h);
#pragma unroll
      for (int k = 0; k < 4; ++k) { t.r[h + k] = r[k]; t.v[h + k] = v[k]; }
    }
    if (a.mask) {
      const u8x4_any_t m0 = *reinterpret_cast<const u8x4_any_t*>(a.mask + i), m1 = *reinterpret_cast<const u8x4_any_t*>(a.mask + i + 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) t.on |= (uint32_t)(m0[k] != 0) << k | (uint32_t)(m1[k] != 0) << (k + 4);
    } else t.on = 0xff;
  } else {
#pragma unroll
    for (int k = 0; k < GAE_PER; ++k) {
      const int64_t j = i + k < a.tokens ? i + k : a.tokens - 1;   // no branch around a load: they are all in flight together
      t.r[k] = a.reward[j];
      t.v[k] = a.value[j];
      t.on |= (uint32_t)((!a.mask || a.mask[j] != 0) && i + k < a.tokens) << k;
    }
  }
  if (threadIdx.x < GAE_TILE / 32) ends.bits[threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = a.sequences ? hold(a.offsets[0], a.tokens) : a.tokens, last = hold(a.offsets[a.sequences], a.tokens);
  if (offset < 0) offset = first_above(a.offsets, a.sequences + 1, a.tokens, start);
  for (int64_t j = offset + threadIdx.x; j <= a.sequences; j += 256) {
    const int64_t o = hold(a.offsets[j], a.tokens), before = j > 0 ? hold(a.offsets[j - 1], a.tokens) : o;
    if (o > start + GAE_TILE) break;
    if (o > start && o > before) {   // the sequence j - 1 is not empty: its last token is o - 1
      const int at = (int)(o - 1 - start);
      ends.last[at] = a.last_value ? a.last_value[j - 1] : 0.f;
      atomicOr(&ends.bits[at >> 5], 1u << (at & 31));
    }
  }
  __syncthreads();
  t.end = ends.bits[threadIdx.x >> 2] >> (threadIdx.x & 3) * 8 & 0xff;
#pragma unroll
  for (int k = 0; k < GAE_PER; ++k) t.last[k] = ends.last[threadIdx.x * GAE_PER + k];   // used where the bit is set
  const int64_t lo = first - i, hi = last - i;   // this thread's tokens that lie in a sequence
  const int l = lo < 0 ? 0 : lo > 8 ? 8 : (int)lo, h = hi < 0 ? 0 : hi > 8 ? 8 : (int)hi;
  t.on &= ((1u << h) - 1) & ~((1u << l) - 1);
  return offset;
}
// whether a thread's tokens hide what comes from behind, and the value in front of them then
__device__ __forceinline__ bool gae_front(const GaeTile& t, float* v) {
  float f = 0.f;
#pragma unroll
  for (int k = GAE_PER - 1; k >= 0; --k) f = t.on >> k & 1 ? t.v[k] : t.end >> k & 1 ? t.last[k] : f;
  *v = f;
  return (t.on | t.end) != 0;
}
// what a thread's tokens do to A, V being the value that enters them; delta: r + gamma V' - V of every token
__device__ __forceinline__ Affine gae_map(const GaeArgs& a, const GaeTile& t, float V, double (&delta)[GAE_PER]) {
  const double gl = a.gamma * a.lambda;
  double c = 0;
#pragma unroll
  for (int k = GAE_PER - 1; k >= 0; --k) {
    const bool on = t.on >> k & 1, end = t.end >> k & 1;
    if (end) { c = 0; V = t.last[k]; }
    delta[k] = a.gamma * V + ((double)t.r[k] - (double)t.v[k]);
    if (on) { c = gl * c + delta[k]; V = t.v[k]; }
  }
  // gamma lambda once for every unmasked token
  const int n = __popc(t.on);
  const double g2 = gl * gl, g4 = g2 * g2;
  double m = n & 1 ? gl : 1.0;
  if (n & 2) m *= g2;
  if (n & 4) m *= g4;
  if (n & 8) m = g4 * g4;
  return Affine{t.end ? 0.0 : m, c};
}

__global__ __launch_bounds__(256) void k_gae_part(GaeArgs a) {
  __shared__ GaeEnds ends;
  __shared__ Affine lds[4];
  __shared__ float lds_v[4];
  __shared__ int lds_set[4];
  __shared__ int counts[4], ends_in[4];
  GaeTile t;
  const int64_t offset = gae_load(a, blockIdx.x, -1, ends, t);   // with barriers
  float v, front;
  bool any;
  const bool set = gae_front(t, &v);
  // the tile's unmasked tokens and whether a sequence ends in it, by the waves' ballots (an atomic addition in LDS by every thread costs 4 us
  // of 13 here)
  int on = 0;
#pragma unroll
  for (int k = 0; k < GAE_PER; ++k) on += __popcll(__ballot(t.on >> k & 1));
  const bool ends_here = __ballot(t.end != 0) != 0;
  if ((threadIdx.x & 63) == 0) { counts[threadIdx.x >> 6] = on; ends_in[threadIdx.x >> 6] = ends_here; }
  const float V = block_value<4>(set, v, 0.f, lds_v, lds_set, &front, &any);
  Affine whole;
  double delta[GAE_PER];
  block_behind<4>(gae_map(a, t, V, delta), lds, &whole);
  if (threadIdx.x == 0) {
    // without the end of a sequence in the tile, V comes into the last of its n unmasked tokens, and n - 1 more times gamma lambda
    const double gl = a.gamma * a.lambda;
    const int count = counts[0] + counts[1] + counts[2] + counts[3], stops = ends_in[0] | ends_in[1] | ends_in[2] | ends_in[3];
    const double b = stops || count == 0 ? 0.0 : count == 1 ? a.gamma : gl > 0 ? whole.a / gl * a.gamma : 0.0;
    a.map[blockIdx.x] = GaeMap{stops ? 0.0 : whole.a, b, whole.c, front, any, stops, (int32_t)offset};
  }
}

// The pair that leaves a run of tiles at its front, by a block of NW waves, one tile's map a thread (the farthest in the last thread), `far`
// being the pair that enters the last of them.  The pair that enters this thread's tile goes to *mine.
template <int NW>
__device__ __forceinline__ double2 gae_tiles(const GaeMap& m, double2 far, double2* mine, Affine* lds, float* lds_v, int* lds_set) {
  float front;
  bool any;
  const float V = block_value<NW>(m.set, m.v, (float)far.y, lds_v, lds_set, &front, &any);
  Affine whole;
  const Affine behind = block_behind<NW>(Affine{m.a, m.b == 0 ? m.c : m.c + m.b * V}, lds, &whole);
  if (mine) *mine = make_double2(apply(behind, far.x), V);
  return make_double2(apply(whole, far.x), front);
}
__device__ __forceinline__ GaeMap gae_nothing() { return GaeMap{1, 0, 0, 0, 0, 0, 0}; }

__global__ __launch_bounds__(1024) void k_gae_tiles(GaeArgs a) {
  __shared__ Affine lds[16];
  __shared__ float lds_v[16];
  __shared__ int lds_set[16];
  double2 far = make_double2(0, 0);
  for (int64_t from = (a.tiles - 1) / 1024 * 1024; from >= 0; from -= 1024) {
    const int64_t k = from + threadIdx.x;
    double2 mine;
    far = gae_tiles<16>(k < a.tiles ? a.map[k] : gae_nothing(), far, &mine, lds, lds_v, lds_set);
    if (k < a.tiles) a.in[k] = mine;
    __syncthreads();   // the LDS is written again
  }
}

__global__ __launch_bounds__(256) void k_token_gae(GaeArgs a) {
  __shared__ GaeEnds ends;
  __shared__ Affine lds[2][4];
  __shared__ float lds_v[2][4];
  __shared__ int lds_set[2][4];
  const int64_t tile = blockIdx.x;
  double2 in = make_double2(0, 0);
  if (a.in) in = a.in[tile];
  else if (tile + 1 < a.tiles) {
    // 256 maps at a time: first up to those among which nothing from behind matters any more (mostly the first ones), then back
    int64_t k = tile + 1 + threadIdx.x;
    GaeMap m = k < a.tiles ? a.map[k] : gae_nothing();
    while (k - threadIdx.x + 256 < a.tiles && !__syncthreads_or(m.stop)) {
      k += 256;
      m = k < a.tiles ? a.map[k] : gae_nothing();
    }
    for (;;) {
      in = gae_tiles<4>(m, in, nullptr, lds[1], lds_v[1], lds_set[1]);
      if (k <= tile + 256) break;
      k -= 256;
      m = a.map[k];
      __syncthreads();   // the LDS is written again
    }
  }
  GaeTile t;
  gae_load(a, tile, a.tiles > 1 ? a.map[tile].offset : -1, ends, t);
  float v;
  const bool set = gae_front(t, &v);
  const float V = block_value<4>(set, v, (float)in.y, lds_v[0], lds_set[0], nullptr, nullptr);
  double delta[GAE_PER];
  double A = apply(block_behind<4>(gae_map(a, t, V, delta), lds[0], nullptr), in.x);
  const double gl = a.gamma * a.lambda;
  float adv[GAE_PER], ret[GAE_PER];
#pragma unroll
  for (int k = GAE_PER - 1; k >= 0; --k) {
    const bool on = t.on >> k & 1, end = t.end >> k & 1;
    if (end) A = 0;
    if (on) A = gl * A + delta[k];
    adv[k] = on ? (float)A : 0.f;
    ret[k] = on ? (float)(A + (double)t.v[k]) : 0.f;
  }
  const int64_t i = tile * GAE_TILE + threadIdx.x * GAE_PER;
  if (tile * GAE_TILE + GAE_TILE <= a.tokens) {
#pragma unroll
    for (int h = 0; h < GAE_PER; h += 4) {
      *reinterpret_cast<f32x4_any_t*>(a.adv + i + h) = f32x4_any_t{adv[h], adv[h + 1], adv[h + 2], adv[h + 3]};
      *reinterpret_cast<f32x4_any_t*>(a.ret + i + h) = f32x4_any_t{ret[h], ret[h + 1], ret[h + 2], ret[h + 3]};
    }
  } else {
#pragma unroll
    for (int k = 0; k < GAE_PER; ++k)
      if (i + k < a.tokens) { a.adv[i + k] = adv[k]; a.ret[i + k] = ret[k]; }
  }
}
