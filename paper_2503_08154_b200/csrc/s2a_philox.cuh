// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): 128 bits for a
// counter of two 64-bit words under a 64-bit key, whose ten round keys are computed once.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace s2a {

struct PhiloxKey {
  uint32_t k0[10], k1[10];
  __device__ __forceinline__ explicit PhiloxKey(uint64_t seed) {
    uint32_t a = (uint32_t)seed, b = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      k0[i] = a;
      k1[i] = b;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
  }
};

__device__ __forceinline__ void philox_round(uint32_t& c0, uint32_t& c1, uint32_t& c2, uint32_t& c3, uint32_t k0, uint32_t k1) {
  const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
  c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
  c1 = (uint32_t)p1;
  c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
  c3 = (uint32_t)p0;
}

__device__ __forceinline__ uint4 philox(const PhiloxKey& key, uint64_t block, uint64_t count) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)count, c3 = (uint32_t)(count >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) philox_round(c0, c1, c2, c3, key.k0[i], key.k1[i]);
  return make_uint4(c0, c1, c2, c3);
}

}  // namespace s2a
