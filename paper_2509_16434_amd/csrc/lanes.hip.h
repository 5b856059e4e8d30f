// Sums and maxima over the lanes of a wave without LDS: permutations of the operand inside 16 lanes, then swaps of 16 and of 32 lanes.
// Every lane of a group of W lanes (16 or 64) gets the result; the order of the additions is fixed.
#pragma once
#include "common.hip.h"

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ double dpp(double v) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, true);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, true);
  return __hiloint2double(hi, lo);
}
#define DPP_XOR1 0xB1         // quad_perm [1,0,3,2]
#define DPP_XOR2 0x4E         // quad_perm [2,3,0,1]
#define DPP_HALF_MIRROR 0x141
#define DPP_MIRROR 0x140
#define DPP_ROW_SHL(n) (0x100 + (n))   // lane i takes lane i + n of its 16

// v of this lane's and of the other half of 32 lanes (16 and 16), and of 64 lanes (32 and 32): *a and *b, the same in both halves
__device__ __forceinline__ void halves32(float v, float* a, float* b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  *a = __uint_as_float(r[0]); *b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void halves64(float v, float* a, float* b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  *a = __uint_as_float(r[0]); *b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void halves32(double v, double* a, double* b) {
  const auto l = __builtin_amdgcn_permlane16_swap((uint32_t)__double2loint(v), (uint32_t)__double2loint(v), false, false);
  const auto h = __builtin_amdgcn_permlane16_swap((uint32_t)__double2hiint(v), (uint32_t)__double2hiint(v), false, false);
  *a = __hiloint2double((int)h[0], (int)l[0]); *b = __hiloint2double((int)h[1], (int)l[1]);
}
__device__ __forceinline__ void halves64(double v, double* a, double* b) {
  const auto l = __builtin_amdgcn_permlane32_swap((uint32_t)__double2loint(v), (uint32_t)__double2loint(v), false, false);
  const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)__double2hiint(v), (uint32_t)__double2hiint(v), false, false);
  *a = __hiloint2double((int)h[0], (int)l[0]); *b = __hiloint2double((int)h[1], (int)l[1]);
}
template <int W, class F> __device__ __forceinline__ F lanes_sum(F v) {
  v += dpp<DPP_XOR1>(v); v += dpp<DPP_XOR2>(v); v += dpp<DPP_HALF_MIRROR>(v); v += dpp<DPP_MIRROR>(v);
  if (W == 64) {
    F a, b;
    halves32(v, &a, &b); v = a + b;
    halves64(v, &a, &b); v = a + b;
  }
  return v;
}
template <int W> __device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, dpp<DPP_XOR1>(v)); v = fmaxf(v, dpp<DPP_XOR2>(v));
  v = fmaxf(v, dpp<DPP_HALF_MIRROR>(v)); v = fmaxf(v, dpp<DPP_MIRROR>(v));
  if (W == 64) {
    float a, b;
    halves32(v, &a, &b); v = fmaxf(a, b);
    halves64(v, &a, &b); v = fmaxf(a, b);
  }
  return v;
}
// N sums over a block of NW waves at once; lds: N NW values; one barrier.  Every thread gets them.
template <int NW, int N> __device__ __forceinline__ void block_sums(double (&v)[N], double* lds) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = lanes_sum<64>(v[k]);
  if (NW == 1) return;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) lds[k * NW + (threadIdx.x >> 6)] = v[k];
  }
  __syncthreads();
  const int w = threadIdx.x & 15;   // every 16 lanes read the (at most 16) waves' sums, one each
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = lanes_sum<16>(w < NW ? lds[k * NW + w] : 0.0);
}
