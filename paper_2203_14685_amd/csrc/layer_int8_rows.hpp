// The 8-bit layer for few tokens: how much of its rows a block quantizes itself.  Host arithmetic and
// the kernel's alike, without a device header.
#pragma once

namespace hetumoe {

constexpr int kInt8Waves = 4;                  // of a block
constexpr int kInt8Step = 256;                 // K of one stage: bytes of a row that are read together
// Rows that a block quantizes itself: up to 4 at a time of at most 8192 elements, the bytes of its range of K
// in LDS beside the rings of two blocks.
constexpr int kInt8HeldRows = 4, kInt8HeldK = 8192, kInt8HeldBytes = 12 * 1024;

// Steps of each wave, with K split over z blocks of kInt8Waves.
constexpr int layer_int8_steps(int K, int z) {
  return ((K + kInt8Step - 1) / kInt8Step + z * kInt8Waves - 1) / (z * kInt8Waves);
}

// Bytes of a row that a block holds in LDS.
constexpr int layer_int8_row_bytes(int K, int z) { return kInt8Waves * layer_int8_steps(K, z) * kInt8Step; }

// Rows of that many bytes that a block takes at a time.  The room alone decides: how many choices name the
// block's expert is known on the device only, and with a caller's ids a token may name one several times.
constexpr int layer_int8_held_rows(int bytes) {
  int rows = kInt8HeldRows;
  while (rows > 0 && rows * bytes > kInt8HeldBytes) --rows;
  return rows;
}

// Whether the blocks of the strips quantize their rows themselves (layer_int8.hip says why).
constexpr bool layer_int8_held(int S, int k, bool by_choice, int K, int z) {
  return (S <= kInt8HeldRows || by_choice) && S * k <= 64 && K <= kInt8HeldK &&
         layer_int8_held_rows(layer_int8_row_bytes(K, z)) >= (S < kInt8HeldRows ? S : kInt8HeldRows);
}

}  // namespace hetumoe
