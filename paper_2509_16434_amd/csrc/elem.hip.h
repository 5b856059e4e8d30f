// Element types of the operators that take fp32, bf16 or fp16 arrays, to and from fp32, and the 16-byte pieces that they are
// read and written in.
#pragma once
#include <utility>

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
// K pieces in registers, each a variable of its own, and f(0), ..., f(K - 1) with the number as a constant to go over them.  (An array of 4
// or 8 pieces is taken for one vector of 16 or 32 registers in a row, which every condition on the way copies as a whole: 304 registers,
// or thousands of spills.)
#define INLINE __attribute__((always_inline))
template <int K> struct Pieces : Pieces<K - 1> { u32x4_t v; };
template <> struct Pieces<0> {};
template <int k, int K> __device__ __forceinline__ u32x4_t& piece(Pieces<K>& p) { return static_cast<Pieces<k + 1>&>(p).v; }
template <class F, int... k> __device__ __forceinline__ void each_of(std::integer_sequence<int, k...>, F f) { (f(std::integral_constant<int, k>()), ...); }
template <int K, class F> __device__ __forceinline__ void each(F f) { each_of(std::make_integer_sequence<int, K>(), f); }
template <class T> struct Piece { static constexpr int N = 16 / sizeof(T); };
template <class T> __device__ __forceinline__ u32x4_t load_piece(const T* p) { return *reinterpret_cast<const u32x4_any_t*>(p); }
template <class T> __device__ __forceinline__ void store_piece(T* p, u32x4_t v) { *reinterpret_cast<u32x4_any_t*>(p) = v; }
template <class T> __device__ __forceinline__ void store_piece_past_caches(T* p, u32x4_t v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any_t*>(p)); }
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
// A row of n elements at x, as a group of threads takes it: `head` elements up to the first 16-byte boundary, `full` elements in
// whole pieces from there, and a tail.  Head and tail (fewer than N elements each) are taken one by one, by the threads 0 .. and
// 8 .. : `one` is this thread's place among them, or -1.  Pieces across the boundaries of cache lines cost a sixth of the rate.
struct Cut { int head, full, one; };
template <class T> __device__ __forceinline__ Cut cut_row(const T* x, int n, int tid) {
  constexpr int N = Piece<T>::N;
  Cut c;
  c.head = min(n, (int)((0u - (uint32_t)((uintptr_t)x / sizeof(T))) & (N - 1)));
  c.full = (n - c.head) & ~(N - 1);
  const int tail = n - c.head - c.full;
  c.one = tid < c.head ? tid : tid >= 8 && tid - 8 < tail ? c.head + c.full + tid - 8 : -1;
  return c;
}
// whether a group's thread tid writes element t of the row (G threads, its pieces G apart)
template <class T, int G> __device__ __forceinline__ bool owns(const Cut& c, int t, int tid) {
  const int r = t - c.head;
  return r >= 0 && r < c.full ? r / Piece<T>::N % G == tid : t == c.one;
}
