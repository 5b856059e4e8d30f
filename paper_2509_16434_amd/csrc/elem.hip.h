// Element types of the operators that take fp32, bf16 or fp16 arrays, to and from fp32.
#pragma once
#include "common.hip.h"

typedef _Float16 f16_t;

template <class T> __device__ __forceinline__ float to_f(T x) { return (float)x; }
template <> __device__ __forceinline__ float to_f<bf16_t>(bf16_t x) { return bf2f(x); }
template <class T> __device__ __forceinline__ T from_f(float x) { return (T)x; }
template <> __device__ __forceinline__ bf16_t from_f<bf16_t>(float x) { return f2bf(x); }
