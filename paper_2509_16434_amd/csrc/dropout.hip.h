// Dropout whose mask is never stored: a function of (seed, layer, row id, column).
//
// Row id r has the SplitMix64 stream of (seed, layer, r) that the minibatch permutations are made of (perm_stream); its
// output number c / 4 holds four 16-bit fields, and column c is kept when field c % 4 is at least q = round(65536 p).
// So y = keep ? x * 65536 / (65536 - q) : 0, plus the residual, in fp32, rounded once to the tensors' type.  The backward
// pass is the same call on the gradient.
#pragma once
#include "elem.hip.h"
#include "splitmix.hip.h"

struct DropoutArgs {
  int64_t rows, cols, ldx, ldr, ldy;
  const void *x, *residual;  // residual: may be NULL
  void* y;
  const int64_t* ids;        // NULL: a row's id is its number
  uint64_t seed, layer;
  uint32_t border;           // q
  float scale;
};

template <class T>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const int64_t groups = (a.cols + 3) / 4, n = a.rows * groups;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / groups, g = i - row * groups;
    const uint64_t state = perm_stream(a.seed, a.layer, a.ids ? (uint64_t)a.ids[row] : (uint64_t)row);
    const uint64_t z = sm64_mix(state + (uint64_t)(g + 1) * 0x9E3779B97F4A7C15ULL);
    for (int k = 0; k < 4; ++k) {
      const int64_t c = 4 * g + k;
      if (c >= a.cols) break;
      const bool keep = ((uint32_t)(z >> (16 * k)) & 0xffffu) >= a.border;
      float y = keep ? to_f(((const T*)a.x)[row * a.ldx + c]) * a.scale : 0.f;
      if (a.residual) y += to_f(((const T*)a.residual)[row * a.ldr + c]);
      ((T*)a.y)[row * a.ldy + c] = from_f<T>(y);
    }
  }
}
