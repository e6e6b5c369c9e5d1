// Rows and weights as operands of the matrix instructions, 128 bytes of a row at a time.
#pragma once

#include "layers.hpp"

namespace ginex {

// Rows are taken in units of 128 bytes, of which a lane has 32.  16-bit numbers are two operands of the matrix instructions as they
// are.  f32 is a sum of three bf16, each the rounded rest of those before it: x = h + m + l with |m| <= 2^-8 |x| and
// |l| <= 2^-17 |x| (h leaves at most 2^-8 of x's power of two, and m has the 8 upper bits of that),
// exactly as long as l is not below 2^-133, the least bf16.  Of the nine products the six largest count; the others are
// 2 * 2^-8 * 2^-17 + 2^-34 of the whole at most, no more than a rounding of it to f32, and the smallest are added first.  Six bf16
// instructions take 96 cycles where the f32 ones take 256 (820 000 x 256 -> 256: 700 us instead of 954).  What is no number, or none
// in bf16, leaves a sum that is none, and such a sum is computed again with the f32 instructions.
template <typename T>
struct Operand {
  static constexpr int PARTS = 2;
  typedef T Kind;
};
template <>
struct Operand<float> {
  static constexpr int PARTS = 3;
  typedef bf16 Kind;
};

// A lane's 32 bytes, as operands.
template <typename T>
__device__ __forceinline__ void parts_of(const ChunkWords<T> (&from)[2], ChunkWords<T> (&to)[2]) {
  to[0] = from[0];
  to[1] = from[1];
}
__device__ __forceinline__ void parts_of(const ChunkWords<float> (&from)[2], ChunkWords<bf16> (&to)[3]) {
  typedef float pair __attribute__((ext_vector_type(2)));
  typedef bf16 half_pair __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    pair v = {from[i / 2].wide[i % 2 * 2], from[i / 2].wide[i % 2 * 2 + 1]};
#pragma unroll
    for (int z = 0; z < 3; ++z) {
      const uint32_t two = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half_pair));
      to[z].words[i] = two;
      v[0] -= __uint_as_float(two << 16);
      v[1] -= __uint_as_float(two & 0xFFFF0000u);
    }
  }
}

// The products of a unit of weights with one of each of MT x 16 rows.
template <typename T, int MT>
__device__ __forceinline__ void products_of(const ChunkWords<T> (&w)[2], const ChunkWords<T> (&x)[MT][2], float4v* sum, int apart) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int m = 0; m < MT; ++m) sum[m * apart] = product(w[k], x[m][k], sum[m * apart]);
}
template <typename T, int MT>
__device__ __forceinline__ void products_of(const ChunkWords<T> (&w)[3], const ChunkWords<T> (&x)[MT][3], float4v* sum, int apart) {
  // (the smallest first)
  constexpr int of_w[6] = {2, 1, 0, 1, 0, 0}, of_x[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
  for (int k = 0; k < 6; ++k)
#pragma unroll
    for (int m = 0; m < MT; ++m) sum[m * apart] = product(w[of_w[k]], x[m][of_x[k]], sum[m * apart]);
}

// Whether one of a wave's sums is no number.
template <int K>
__device__ __forceinline__ bool any_none(const float4v* sum) {
  bool fine = true;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) fine = fine && __builtin_isfinite(sum[k][j]);
  return __ballot(!fine) != 0;
}

// What sums computed again replace: those that are no numbers, so that no row's result hangs on the others of its tile.
__device__ __forceinline__ float4v with_again(float4v sum, float4v again) {
#pragma unroll
  for (int j = 0; j < 4; ++j) sum[j] = __builtin_isfinite(sum[j]) ? sum[j] : again[j];
  return sum;
}

// `start` and the products of this lane's row (of 16) with its column of weights (of 16), by the f32 instructions and from memory.
__device__ __forceinline__ float4v sums_again(const float* row, bool there, const float* column, int64_t stride, int32_t width,
                                              float4v start) {
  for (int32_t k = 0; k < width; k += 4) {
    const int32_t at = k + lane_id() / 16;
    const bool in = at < width;
    start = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? column[(in ? at : 0) * stride] : 0.f, in && there ? row[at] : 0.f, start, 0, 0, 0);
  }
  return start;
}

}  // namespace ginex
