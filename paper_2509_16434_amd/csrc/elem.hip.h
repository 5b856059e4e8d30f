// Element types of the operators that take fp32, bf16 or fp16 arrays, to and from fp32, and the 16-byte pieces that they are
// read and written in.
#pragma once
#include "common.hip.h"

typedef _Float16 f16_t;

template <class T> __device__ __forceinline__ float to_f(T x) { return (float)x; }
template <> __device__ __forceinline__ float to_f<bf16_t>(bf16_t x) { return bf2f(x); }
template <class T> __device__ __forceinline__ T from_f(float x) { return (T)x; }
template <> __device__ __forceinline__ bf16_t from_f<bf16_t>(float x) { return f2bf(x); }

// ---- 16 bytes of a row
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_any_t __attribute__((aligned(2)));
// From here on the compiler knows nothing of a piece's value, so that it unpacks it again in the next pass over the row instead of
// keeping all of it in 32 bits (which needs two to four times the registers).
__device__ __forceinline__ void forget(u32x4_t& v) { asm volatile("" : "+v"(v)); }
template <class T> struct Piece { static constexpr int N = 16 / sizeof(T); };
template <class T> __device__ __forceinline__ u32x4_t load_piece(const T* p) { return *reinterpret_cast<const u32x4_any_t*>(p); }
template <class T> __device__ __forceinline__ void store_piece(T* p, u32x4_t v) { *reinterpret_cast<u32x4_any_t*>(p) = v; }
__device__ __forceinline__ void unpack(u32x4_t v, float (&f)[4], float) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
}
__device__ __forceinline__ void unpack(u32x4_t v, float (&f)[8], bf16_t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
}
__device__ __forceinline__ void unpack(u32x4_t v, float (&f)[8], f16_t) {
  typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = v[i];  // a copy: the cast of a vector's element itself takes element 0
    const h2_t h = __builtin_bit_cast(h2_t, w);
    f[2 * i] = (float)h[0]; f[2 * i + 1] = (float)h[1];
  }
}
__device__ __forceinline__ u32x4_t pack(const float (&f)[4], float) {
  u32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
  return v;
}
__device__ __forceinline__ u32x4_t pack(const float (&f)[8], bf16_t) {
  u32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2bf(f[2 * i], f[2 * i + 1]);
  return v;
}
__device__ __forceinline__ u32x4_t pack(const float (&f)[8], f16_t) {
  typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
  u32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) { const h2_t h = {(_Float16)f[2 * i], (_Float16)f[2 * i + 1]}; v[i] = __builtin_bit_cast(uint32_t, h); }
  return v;
}
// two lowest-valued logits, for the places behind the end of a row
__device__ __forceinline__ uint32_t no_logits(float) { return 0xff800000u; }
__device__ __forceinline__ uint32_t no_logits(bf16_t) { return 0xff80ff80u; }
__device__ __forceinline__ uint32_t no_logits(f16_t) { return 0xfc00fc00u; }
// elements i .. i + N - 1 of a row (or part) of n elements; those behind its end are -infinity
template <class T>
__device__ __forceinline__ u32x4_t load_row(const T* x, int i, int n) {
  constexpr int N = Piece<T>::N;
  const uint32_t none = no_logits(T());
  u32x4_t v = {none, none, none, none};
  if (i + N <= n) v = load_piece(x + i);
  else if (i < n) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (i + k < n) {
        if constexpr (sizeof(T) == 4) v[k] = __float_as_uint(x[i + k]);
        else { const T one = x[i + k]; const uint32_t h = __builtin_bit_cast(uint16_t, one); v[k >> 1] = k & 1 ? (v[k >> 1] & 0xffffu) | (h << 16) : (v[k >> 1] & 0xffff0000u) | h; }
      }
    }
  }
  return v;
}
template <class T>
__device__ __forceinline__ void store_row(T* y, int i, int n, u32x4_t v) {
  constexpr int N = Piece<T>::N;
  if (i + N <= n) store_piece(y + i, v);
  else if (i < n) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (i + k < n) {
        if constexpr (sizeof(T) == 4) y[i + k] = __uint_as_float(v[k]);
        else { const uint16_t h = (uint16_t)(v[k >> 1] >> (k & 1 ? 16 : 0)); y[i + k] = __builtin_bit_cast(T, h); }
      }
    }
  }
}
