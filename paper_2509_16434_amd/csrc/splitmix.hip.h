// The counter-based generator of the library: SplitMix64 streams whose state is a hash chain of three numbers
// ((seed, update, epoch) for a minibatch permutation, (seed, layer, row id) for a dropout mask).
#pragma once
#include "common.hip.h"

__host__ __device__ __forceinline__ uint64_t sm64_mix(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
  return z ^ (z >> 31);
}
__host__ __device__ __forceinline__ uint64_t perm_stream(uint64_t seed, uint64_t update, uint64_t epoch) {
  const uint64_t G = 0x9E3779B97F4A7C15ULL;
  uint64_t s = sm64_mix(seed + G);
  s = sm64_mix(s ^ (update + G));
  s = sm64_mix(s ^ (epoch + G));
  return s;
}
__device__ __forceinline__ uint64_t perm_key(uint64_t stream, uint64_t i) {
  return sm64_mix(stream + (i + 1) * 0x9E3779B97F4A7C15ULL);
}
