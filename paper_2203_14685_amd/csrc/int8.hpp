// Quantization to 8-bit integers: q = the integer next to 127 x / a, a = max |x| of a row or a
// column, scale = a / 127.
#pragma once

#include "common.hpp"

namespace hetumoe {

// |x| as an integer that orders like it, infinities and then NaNs above all.
__device__ __forceinline__ int abs_bits(float x) { return static_cast<int>(__float_as_uint(x) & 0x7fffffffu); }

struct Quantizer {
  float most, inverse, up;  // a and x are multiplied by `up` first: 127 / a stays finite
  float scale;

  __device__ __forceinline__ explicit Quantizer(int bits) {
    const float a = __uint_as_float(static_cast<uint32_t>(bits));
    const bool finite = bits < 0x7f800000;
    scale = finite ? a / 127.f : __uint_as_float(0x7fc00000u);
    up = a < 0x1p-100f ? 0x1p100f : 1.f;
    most = a * up;
    inverse = finite && bits > 0 ? 127.f / most : 0.f;
  }
  // The product rounds twice, so near a border (half of the largest value lies on one, whatever
  // the row) the exact distance decides: 127 x and q a have 31 bits, 64 hold their difference.
  __device__ __forceinline__ int operator()(float x) const {
    if (inverse == 0.f) return 0;
    const float xs = x * up, v = xs * inverse;
    float q = rintf(v);
    if (fabsf(v - q) > 0.499f) {
      const double e = 127.0 * static_cast<double>(xs) - static_cast<double>(q) * static_cast<double>(most);
      const double over = 2.0 * fabs(e) - static_cast<double>(most);
      if (over > 0.0 || (over == 0.0 && (static_cast<int>(q) & 1))) q += e > 0.0 ? 1.f : -1.f;
    }
    return static_cast<int>(q);
  }
  __device__ __forceinline__ uint32_t four(const float* f) const {
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) r |= (static_cast<uint32_t>((*this)(f[j])) & 0xffu) << (8 * j);
    return r;
  }
};

}  // namespace hetumoe
