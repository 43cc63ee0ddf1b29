// Quantization to 8-bit integers: q = the integer next to 127 x / a, a = max |x| of a row or a
// column, scale = a / 127.
#pragma once

#include "common.hpp"

namespace hetumoe {

// |x| as an integer that orders like it, infinities and then NaNs above all.
__device__ __forceinline__ int abs_bits(float x) { return static_cast<int>(__float_as_uint(x) & 0x7fffffffu); }

// Running maximum of |x| over 16-byte pieces: of bf16 two 16-bit halves at once.
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
template <class T>
struct MostOf;
template <>
struct MostOf<float> {
  int most = 0;
  __device__ __forceinline__ void take(const u32x4& v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) most = max(most, static_cast<int>(v[j] & 0x7fffffffu));
  }
  __device__ __forceinline__ int bits() const { return most; }
};
template <>
struct MostOf<bf16_t> {
  u16x2_t most = {0, 0};
  __device__ __forceinline__ void take(const u32x4& v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, v[j] & 0x7fff7fffu));
  }
  __device__ __forceinline__ int bits() const { return static_cast<int>(most[0] > most[1] ? most[0] : most[1]) << 16; }
};

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

  // The same for a bf16 x, without the test.  With x = m 2^-j and a of 8 bits, 127 x / a that is not on a
  // border is off it by 1 / (2 a 2^j) at least, 2^-17 of itself; v is off by 2^-23 of itself.  So v rounded
  // to 19 bits lies on the border exactly where the quotient does.  1.5 2^23 added leaves the
  // integer next to it, ties to even, in the lowest byte.
  __device__ __forceinline__ uint32_t byte_of_bf16(float x) const {
    const uint32_t v = (__float_as_uint(x * up * inverse) + 16u) & ~31u;
    return __float_as_uint(__uint_as_float(v) + 12582912.f);
  }
  // Four elements as integers.
  __device__ __forceinline__ uint32_t four(const float* f, bf16_t) const {
    const uint32_t lo = __builtin_amdgcn_perm(byte_of_bf16(f[1]), byte_of_bf16(f[0]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(byte_of_bf16(f[3]), byte_of_bf16(f[2]), 0x04000c0cu);
    return lo | hi;
  }
  __device__ __forceinline__ uint32_t four(const float* f, float) const {
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) r |= (static_cast<uint32_t>((*this)(f[j])) & 0xffu) << (8 * j);
    return r;
  }
};

// A piece of 16 elements: 16 bytes of integers.
template <class T>
__device__ __forceinline__ u32x4 quantize_piece(const Quantizer& quant, const u32x4 (&v)[16 / Chunk<T>::kElems]) {
  constexpr int PE = Chunk<T>::kElems;
  float f[16];
#pragma unroll
  for (int q = 0; q < 16 / PE; ++q) Chunk<T>::unpack(v[q], f + q * PE);
  const u32x4 q = {quant.four(f, T()), quant.four(f + 4, T()), quant.four(f + 8, T()), quant.four(f + 12, T())};
  return quant.inverse != 0.f ? q : u32x4{0, 0, 0, 0};  // rows of zeros, and those that are not finite
}

}  // namespace hetumoe
