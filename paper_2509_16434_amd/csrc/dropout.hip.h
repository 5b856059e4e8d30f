// Dropout whose mask is never stored: a function of (seed, layer, row id, column).
//
// Row id r has the SplitMix64 stream of (seed, layer, r) that the minibatch permutations are made of (perm_stream); its
// output number c / 4 holds four 16-bit fields, and column c is kept when field c % 4 is at least q = round(65536 p).
// So y = keep ? x * 65536 / (65536 - q) : 0, plus the residual, in fp32, rounded once to the tensors' type.  The backward
// pass is the same call on the gradient.
//
// Bound by memory: an output serves four columns (fp32) or two outputs eight (16 bits), 13 vector instructions a column (16 with the
// residual) where the time of its bytes holds 22 (38); the hash of (seed, layer) is made on the host, that of the row id once per thread.
// Pieces are cut from the row's start, where the generator's outputs begin: rows of odd length cross the boundaries of cache lines and run at
// 0.94 of the rate (134 MB each way in the last-level cache: 16384 x 4096 bf16 7030 GB/s, 16388 x 4095 6600).
#pragma once
#include "elem.hip.h"
#include "splitmix.hip.h"

struct DropoutArgs {
  int64_t rows, cols, ldx, ldr, ldy;
  const void *x, *residual;  // residual: may be NULL
  void* y;
  const int64_t* ids;        // NULL: a row's id is its number
  uint64_t prefix;           // hash of (seed, layer)
  uint32_t border;           // q
  float scale;
};

// A group of G threads does a slice of G DROP_PIECES pieces of a row: blockIdx.x the slice (G < 256: the row is one slice),
// blockIdx.y and z the row.
constexpr int DROP_PIECES = 4;
template <class T, int G, bool RES>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  constexpr int N = Piece<T>::N;
  const int64_t row = G < 256 ? (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G : blockIdx.y + (int64_t)blockIdx.z * 65535;
  if (row >= a.rows) return;
  const int n = (int)a.cols, from = (G < 256 ? 0 : blockIdx.x * (G * DROP_PIECES * N)) + threadIdx.x % G * N;
  const T *x = (const T*)a.x + row * a.ldx, *r = RES ? (const T*)a.residual + row * a.ldr : nullptr;
  T* y = (T*)a.y + row * a.ldy;
  const int full = n & ~(N - 1), tid = threadIdx.x % G;   // the last n % N columns are taken one by one
  const uint64_t G64 = 0x9E3779B97F4A7C15ULL;
  u32x4_t v[DROP_PIECES], w[DROP_PIECES];
#pragma unroll
  for (int u = 0; u < DROP_PIECES; ++u)
    if (from + u * G * N < full) {
      v[u] = load_piece(x + from + u * G * N);
      if (RES) w[u] = load_piece(r + from + u * G * N);
    }
  const uint64_t state = sm64_mix(a.prefix ^ ((a.ids ? (uint64_t)a.ids[row] : (uint64_t)row) + G64));
#pragma unroll
  for (int u = 0; u < DROP_PIECES; ++u) {
    const int at = from + u * G * N;
    if (at >= full) break;
    float f[N], g[N];
    unpack(v[u], f, T());
    if (RES) unpack(w[u], g, T());
#pragma unroll
    for (int h = 0; h < N; h += 4) {
      const uint64_t z = sm64_mix(state + (uint64_t)(at / 4 + h / 4 + 1) * G64);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t half = (uint32_t)(z >> (k & 2 ? 32 : 0)), field = k & 1 ? half >> 16 : half & 0xffffu;
        const float kept = field >= a.border ? f[h + k] * a.scale : 0.f;
        f[h + k] = RES ? kept + g[h + k] : kept;
      }
    }
    store_piece(y + at, pack(f, T()));
  }
  if ((G < 256 || blockIdx.x == 0) && tid < n - full) {
    const int c = full + tid;
    const uint64_t z = sm64_mix(state + (uint64_t)(c / 4 + 1) * G64);
    const float kept = ((uint32_t)(z >> (c % 4 * 16)) & 0xffffu) >= a.border ? to_f(x[c]) * a.scale : 0.f;
    y[c] = from_f<T>(RES ? kept + to_f(r[c]) : kept);
  }
}
