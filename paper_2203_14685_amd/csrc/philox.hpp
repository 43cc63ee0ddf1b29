// Dropout's random words: Philox4x32-10, the counter-based generator of Salmon, Moraes, Dror
// and Shaw, "Parallel random numbers: as easy as 1, 2, 3" (SC 2011), written from its formulas.
//
// Block b of 8 elements takes one call, 16 bits per element: a word of 32 per element would
// take twice the multiplications, which run at a quarter of the rate of additions (20 of them per
// call: 480 cycles of a SIMD per 512 elements, 2.6e12 elements/s on the chip, where memory
// brings 0.9e12 bf16 elements/s with a residual).
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace hetumoe {

__device__ __forceinline__ uint64_t drop_call(const DropArgs& m) { return m.step ? m.call + *m.step : m.call; }

// The four words of block `block`: element 8 block + j has half j % 2 of word j / 2.  UNROLL 1
// keeps large epilogues small.
template <int UNROLL = 10>
__device__ __forceinline__ u32x4 philox(const DropArgs& m, uint64_t call, uint64_t block) {
  uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32);
  uint32_t c2 = static_cast<uint32_t>(call), c3 = static_cast<uint32_t>(call >> 32);
  uint32_t k0 = m.k0, k1 = m.k1;
#pragma unroll UNROLL
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c0, p1 = static_cast<uint64_t>(0xCD9E8D57u) * c2;
    c0 = static_cast<uint32_t>(p1 >> 32) ^ c1 ^ k0;
    c2 = static_cast<uint32_t>(p0 >> 32) ^ c3 ^ k1;
    c1 = static_cast<uint32_t>(p1);
    c3 = static_cast<uint32_t>(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

__device__ __forceinline__ bool drop_keeps(const DropArgs& m, const u32x4& words, int j) {
  return ((words[j / 2] >> (16 * (j % 2))) & 0xffffu) >= m.t;
}

// v kept and scaled, or 0 whatever v holds.
__device__ __forceinline__ float dropped(const DropArgs& m, const u32x4& words, int j, float v) {
  return drop_keeps(m, words, j) ? v * m.scale : 0.f;
}

}  // namespace hetumoe
