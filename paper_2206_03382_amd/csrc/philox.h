// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011), key = seed[0], counter = (number of the group of eight elements, seed[1]).  16 of the 128 bits for an element: a group is one
// 16-byte piece of bf16, and ten rounds of four 32-bit products serve eight elements, which HBM takes longer for than the rounds do (32 bits for an element would not be).
// Kept apart from the kernels so that a test can compile it for the host.
#pragma once
#include "ffn_rules.h"

namespace moe {

struct Philox {
  uint32_t k0 = 0, k1 = 0, o0 = 0, o1 = 0;
  Philox() = default;                                               // where nothing is dropped: there need be no seed
  MOE_HOST_DEVICE explicit Philox(const uint64_t* seed) : k0((uint32_t)seed[0]), k1((uint32_t)(seed[0] >> 32)), o0((uint32_t)seed[1]), o1((uint32_t)(seed[1] >> 32)) {}
  // the 16-bit numbers of group g, the lower one of a word first
  MOE_HOST_DEVICE inline __attribute__((always_inline)) void bits(uint64_t g, uint32_t (&w)[4]) const {
    uint32_t c0 = (uint32_t)g, c1 = (uint32_t)(g >> 32), c2 = o0, c3 = o1, a = k0, b = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
      c0 = (uint32_t)(p1 >> 32) ^ c1 ^ a;
      c1 = (uint32_t)p1;
      c2 = (uint32_t)(p0 >> 32) ^ c3 ^ b;
      c3 = (uint32_t)p0;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
    w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
  }
};

}  // namespace moe
