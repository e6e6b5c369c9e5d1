// What happens to the sums of a linear layer, 16 neighbouring columns of a row at a time: activation, residual, codes, rounding.
#pragma once

#include "activations.hpp"
#include "codes.hpp"
#include "layers.hpp"

namespace ginex {

// 16 neighbouring columns of a row as they are in memory; what is behind the row is 0.
template <typename T>
struct Columns {
  static constexpr int N = Chunk<T>::N, CHUNKS = LANE_COLUMNS / N;
  ChunkWords<T> chunk[CHUNKS];
  template <bool WIDE = false>
  __device__ __forceinline__ void load(const T* row, int32_t c, Width width) {
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) chunk[k] = load_words<WIDE>(row, c + k * N, width);
  }
  // In two halves: the loads, of a row that has a chunk at least, ...
  __device__ __forceinline__ void read(const T* row, int32_t c, Width width) {
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      const int32_t at = c + k * N;
      chunk[k].wide = *reinterpret_cast<const typename Chunk<T>::At*>(row + (at < width.width - N ? at : width.width - N));
    }
  }
  // ... and what becomes of them.
  __device__ __forceinline__ void place(int32_t c, Width width) {
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) chunk[k] = placed<T>(chunk[k], c + k * N, width);
  }
  __device__ __forceinline__ float of(int i) const { return (float)chunk[i / N].wide[i % N]; }
};

template <int ACT, typename T>
__device__ __forceinline__ void activate_columns(float (&v)[LANE_COLUMNS]) {
#pragma unroll
  for (int i = 0; i < LANE_COLUMNS; ++i) v[i] = activated<ACT, sizeof(T) == 4>(v[i]);
}

// Codes of 16 columns from c on; the block's other half is 16 lanes away.
template <typename T>
__device__ __forceinline__ void keep_columns(const Epilogue& e, int64_t r, bool mine, int32_t c, Width width,
                                             const float (&v)[LANE_COLUMNS]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < LANE_COLUMNS; ++i) {
    const uint32_t magnitude = c + i < width.width ? __float_as_uint(v[i]) & 0x7FFFFFFFu : 0;
    top = top > magnitude ? top : magnitude;
  }
  const uint32_t other = (uint32_t)__shfl_xor((int)top, 16, WAVE);
  const uint32_t scale = scale_byte(top > other ? top : other);
  const float by = to_codes(scale);
  constexpr float whole = 12582912.f;       // 1.5 2^23: v by + whole is rounded to a whole number, halves to even
  words2 word[2];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[i] = __builtin_amdgcn_fmed3f(fmaf(v[4 * k + i], by, whole), whole - 127.f, whole + 127.f);
      q[i] = c + 4 * k + i < width.width ? q[i] : whole;
    }
    word[k / 2][k % 2] = scale == NO_NUMBER ? 0 : low_bytes(q[0], q[1], q[2], q[3]);
  }
  if (!mine || c >= e.blocks * GINEX_CODE_BLOCK) return;
  words2* const at = reinterpret_cast<words2*>(e.codes + r * ((int64_t)e.blocks * GINEX_CODE_BLOCK) + c);
  at[0] = word[0];
  at[1] = word[1];
  if (c % GINEX_CODE_BLOCK == 0) e.scales[r * e.blocks + c / GINEX_CODE_BLOCK] = (uint8_t)scale;
}

// whole (the same for all lanes): the row has all 16.
template <typename T>
__device__ __forceinline__ void store_columns(const Epilogue& e, int64_t r, int32_t c, bool whole, Width width,
                                              const float (&v)[LANE_COLUMNS]) {
  constexpr int N = Chunk<T>::N;
  T* const to = static_cast<T*>(e.y) + r * e.y_stride;
#pragma unroll
  for (int k = 0; k < LANE_COLUMNS / N; ++k) {
    ChunkWords<T> u;
#pragma unroll
    for (int i = 0; i < N; ++i) u.wide[i] = (T)v[k * N + i];
    if (whole) *reinterpret_cast<typename Chunk<T>::At*>(to + c + k * N) = u.wide;
    else if (c + k * N < width.width) store_words<true>(to, c + k * N, width, u);
  }
}

// The same without a branch where the row's chunks are whole, for rows that are `mine`.
template <typename T>
__device__ __forceinline__ void store_columns_masked(const Epilogue& e, int64_t r, bool mine, int32_t c, Width width,
                                                     const float (&v)[LANE_COLUMNS]) {
  constexpr int N = Chunk<T>::N;
  T* const to = static_cast<T*>(e.y) + r * e.y_stride + c;
  ChunkWords<T> u[LANE_COLUMNS / N];
#pragma unroll
  for (int k = 0; k < LANE_COLUMNS / N; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) u[k].wide[i] = (T)v[k * N + i];
#pragma unroll
  for (int k = 0; k < LANE_COLUMNS / N; ++k)
    if (mine && c + (k + 1) * N <= width.width) *reinterpret_cast<typename Chunk<T>::At*>(to + k * N) = u[k].wide;
  if (width.missing == 0) return;
#pragma unroll
  for (int k = 0; k < LANE_COLUMNS / N; ++k)
    if (mine && c + k * N < width.width && c + (k + 1) * N > width.width) store_words<true>(to - c, c + k * N, width, u[k]);
}

// Sums and bias of 16 columns of row r: their codes, and what y gets but for the residual, in `v`.  All lanes call it; the row
// is there if it is `mine`.
template <typename T>
__device__ __forceinline__ void finish_values(const Epilogue& e, int64_t r, bool mine, int32_t c, Width width,
                                              float (&v)[LANE_COLUMNS]) {
  if (e.codes) keep_columns<T>(e, r, mine, c, width, v);
  switch (e.activation) {           // (the same for all lanes)
    case GINEX_ACT_RELU: activate_columns<GINEX_ACT_RELU, T>(v); break;
    case GINEX_ACT_SILU: activate_columns<GINEX_ACT_SILU, T>(v); break;
    case GINEX_ACT_GELU: activate_columns<GINEX_ACT_GELU, T>(v); break;
  }
}
template <typename T>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t r, int32_t c, bool whole, Width width, float (&v)[LANE_COLUMNS],
                                       const Columns<T>& residual) {
  finish_values<T>(e, r, true, c, width, v);
  if (e.residual) {
#pragma unroll
    for (int i = 0; i < LANE_COLUMNS; ++i) v[i] += residual.of(i);
  }
  store_columns<T>(e, r, c, whole, width, v);
}

// A slot without a row.
template <typename T>
__device__ __forceinline__ void clear_columns(const Epilogue& e, int64_t r, int32_t c, Width width) {
  const float zero[LANE_COLUMNS] = {};
  if (e.codes) keep_columns<T>(e, r, true, c, width, zero);
  store_columns<T>(e, r, c, false, width, zero);
}

// The bias of 16 columns.
template <typename T>
__device__ __forceinline__ void load_bias(const Epilogue& e, int32_t expert, int32_t c, Width width, float (&v)[LANE_COLUMNS]) {
  Columns<T> b;
  if (e.bias) b.load(static_cast<const T*>(e.bias) + (int64_t)expert * width.width, c, width);
#pragma unroll
  for (int i = 0; i < LANE_COLUMNS; ++i) v[i] = e.bias ? b.of(i) : 0.f;
}

}  // namespace ginex
