// The 8-bit codes on the device: a block of 32 channels shares a power of two, e is the exponent of its
// largest magnitude, and q stands for q 2^(e-6).  Scaling by powers of two is exact in f32, so the codes do
// not depend on the arithmetic that made them, and |q| <= 127 has 7 bits: the restored value is exact in
// bf16 and f32.
#pragma once

#include "train.hpp"

namespace ginex {

constexpr int LEAST_EXPONENT = -120;      // q 2^(e-6) is a normal number of bf16 and f32
constexpr uint32_t NO_NUMBER = 255;       // the scale byte of a block with an infinity or a NaN

// The scale byte of a block from the largest of its magnitudes' bit patterns (NaNs are the largest).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  const uint32_t exponent = top >> 23;
  if (exponent == 255) return NO_NUMBER;
  constexpr uint32_t least = LEAST_EXPONENT + 127;
  return exponent > least ? exponent : least;
}

// What a block's values are multiplied with to become codes, 2^(6-e); 0 for a block without numbers.
__device__ __forceinline__ float to_codes(uint32_t scale) {
  return scale == NO_NUMBER ? 0.f : __uint_as_float((260 - scale) << 23);
}

// What a code stands for, 2^(e-6).
__device__ __forceinline__ float code_step(uint32_t scale) {
  return scale == NO_NUMBER ? __uint_as_float(0x7FC00000) : ldexpf(1.f, (int)scale - 133);
}

}  // namespace ginex
