// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011): a block of four random words as a function of a
// 128-bit counter and a 64-bit key.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hydra {

__device__ __forceinline__ uint4 philox4x32(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// Dropout's random numbers: sixteen bits an element, eight elements a block.
// `seed` is the key, `offset` the counter's upper half, `group` (the element's flat
// index / 8) its lower half; element 8 group + j has half j % 2 (0: the
// lower) of word j / 2.
__device__ __forceinline__ uint4 dropout_words(uint64_t seed, uint64_t offset, uint64_t group) {
  return philox4x32(make_uint4((uint32_t)group, (uint32_t)(group >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)),
                    (uint32_t)seed, (uint32_t)(seed >> 32));
}
__device__ __forceinline__ bool dropout_keeps(const uint4& w, int j, uint32_t drop) {
  const uint32_t word = j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w;
  return (j & 1 ? word >> 16 : word & 0xFFFFu) >= drop;
}

}  // namespace hydra
