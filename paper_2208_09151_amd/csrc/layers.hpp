// Shared by the layers: descriptors of weights, products of chunks of 16 bytes on the matrix cores, tiles of slots that no
// two experts share.
#pragma once

#include "ginex_layers.h"
#include "train.hpp"

namespace ginex {

typedef float float4v __attribute__((ext_vector_type(4)));

// 16 x 16 sums of products over 4 chunks of each of 16 rows of either operand: lane l brings chunk l / 16 of row l % 16 and
// gets rows 4 (l / 16) .. + 3 of `a` with row l % 16 of `b`.  Products of 16-bit numbers are exact, sums are f32.
__device__ __forceinline__ float4v product(const ChunkWords<bf16>& a, const ChunkWords<bf16>& b, float4v sum) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.wide, b.wide, sum, 0, 0, 0);
}
__device__ __forceinline__ float4v product(const ChunkWords<f16>& a, const ChunkWords<f16>& b, float4v sum) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.wide, b.wide, sum, 0, 0, 0);
}
__device__ __forceinline__ float4v product(const ChunkWords<float>& a, const ChunkWords<float>& b, float4v sum) {
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(a.wide[i], b.wide[i], sum, 0, 0, 0);
  return sum;
}
template <typename T>
struct WeightsOf {
  const T* data;
  int64_t stride, expert_stride;
  __device__ __forceinline__ const T* of(int32_t expert) const { return data + expert * expert_stride; }
};

constexpr int LANE_COLUMNS = 16;        // neighbouring columns of one row that a lane ends up with
constexpr int WAVE_COLUMNS = 64;

// A chunk of weights' columns at any place of a row of `columns`: 4 of them (8 bytes of 16 bits, 16 of f32).
template <typename T>
struct Four {
  typedef T Wide __attribute__((ext_vector_type(4)));
  typedef Wide At __attribute__((aligned(sizeof(T))));
};

// Four neighbouring columns of a row of weights, from column n on; what is behind the last one is 0.  The last ones are read so
// that they end with the row, and moved.
template <typename T>
__device__ __forceinline__ typename Four<T>::Wide four_read(const T* row, int32_t n, int32_t columns) {
  return *reinterpret_cast<const typename Four<T>::At*>(row + (n + 4 > columns ? columns - 4 : n));
}
template <typename T>
__device__ __forceinline__ typename Four<T>::Wide four_placed(typename Four<T>::Wide v, int32_t n, int32_t columns) {
  const int32_t over = n + 4 - columns;
  if (over > 0) {
#pragma unroll
    for (int l = 0; l < 4; ++l) {
      T to = (T)0.f;
#pragma unroll
      for (int m = l + 1; m < 4; ++m) to = m == l + over ? v[m] : to;
      v[l] = to;
    }
  }
  return v;
}
template <bool WIDE = false, typename T>
__device__ __forceinline__ typename Four<T>::Wide four_of(const T* row, int32_t n, int32_t columns) {
  if (!WIDE && columns < 4) {
    typename Four<T>::Wide v;
#pragma unroll
    for (int l = 0; l < 4; ++l) v[l] = n + l < columns ? row[n + l] : (T)0.f;
    return v;
  }
  return four_placed<T>(four_read(row, n, columns), n, columns);
}

// What happens to the sums of a linear layer.
struct Epilogue {
  const void* bias;
  const void* residual;
  int64_t residual_stride;
  void* y;
  int64_t y_stride;
  int8_t* codes;
  uint8_t* scales;
  int32_t blocks;       // of 32 codes in a row
  int32_t activation;
};

// A linear layer of few rows, 16 of them and 64 columns to a workgroup.
int64_t few_groups(const ginex_weights_t* weights, const ginex_routing_t* route, int64_t slots);
int32_t linear_few(const ginex_rows_t* x, const ginex_weights_t* weights, const ginex_routing_t* route, bool by_slot,
                   int64_t slots, const Epilogue& epilogue, hipStream_t st);

// A linear layer of many rows whose weights find room in LDS; false: not for these sizes.
bool resident_fits(const ginex_weights_t* weights, int64_t slots);
int32_t linear_resident(const ginex_rows_t* x, const ginex_weights_t* weights, const ginex_routing_t* route, bool by_slot,
                        int64_t slots, const Epilogue& epilogue, hipStream_t st);

// The rows that a tile has: `first` .. `end` - 1, at most as many as a tile takes are its own.  expert == experts: the rows that no
// expert has.
struct TileRows {
  int32_t expert;
  int64_t first, end;
};

// Tile `t` of the tiles of `height` slots that the experts' slots are cut into, one expert after the other, and behind them
// the slots without an expert.  All lanes of a wave call it and get the same; false: there is no such tile.
__device__ __forceinline__ bool find_tile(const int64_t* __restrict__ offsets, int32_t experts, int64_t slots, uint32_t t,
                                          int32_t height, TileRows& tile) {
  uint32_t before = 0;
  for (int32_t e0 = 0; e0 <= experts; e0 += WAVE) {
    const int32_t e = e0 + lane_id();
    int64_t begin = 0, end = 0;
    if (e < experts) {
      begin = offsets[e];
      end = offsets[e + 1];
      bound_slots(slots, begin, end);
    } else if (e == experts) {
      begin = inside(offsets[experts], slots);
      end = slots;
    }
    const uint32_t tiles = (uint32_t)(end - begin + height - 1) / (uint32_t)height;
    const uint32_t upto = before + wave_inclusive_scan(tiles);
    const uint64_t has = __ballot(upto > t);
    if (has) {
      const int lane = __ffsll((unsigned long long)has) - 1;
      const uint32_t k = t - (of_lane(upto, lane) - of_lane(tiles, lane));
      tile.expert = e0 + lane;
      tile.first = (int64_t)of_lane((uint64_t)begin, lane) + (int64_t)k * height;
      tile.end = (int64_t)of_lane((uint64_t)end, lane);
      return tile.first < tile.end;       // (offsets that do not ascend may have more tiles than 32 bits count)
    }
    before = of_lane(upto, WAVE - 1);
  }
  return false;
}

// How many tiles there are.
__device__ __forceinline__ uint32_t count_tiles(const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                                int32_t height) {
  uint32_t tiles = 0;
  for (int32_t e = lane_id(); e <= experts; e += WAVE) {
    int64_t begin = inside(offsets[e], slots), end = slots;
    if (e < experts) {
      begin = offsets[e];
      end = offsets[e + 1];
      bound_slots(slots, begin, end);
    }
    tiles += (uint32_t)(end - begin + height - 1) / (uint32_t)height;
  }
  return wave_reduce_sum(tiles);
}

// As many tiles as find_tile can find: every group of slots has one that is not full.
inline int64_t most_tiles(int64_t slots, int32_t experts, int32_t height) {
  const int64_t groups = (int64_t)experts + 1;
  return slots / height + (groups < slots ? groups : slots);
}

inline int32_t check_weights(const ginex_weights_t* w) {
  if (!w) return fail(GINEX_ERR_ARG, "weights: null descriptor");
  if (w->type != GINEX_F32 && w->type != GINEX_BF16 && w->type != GINEX_F16)
    return fail(GINEX_ERR_ARG, "weights: unknown type %d", w->type);
  if (w->experts < 1 || w->experts > GINEX_MAX_EXPERTS)
    return fail(GINEX_ERR_ARG, "weights: experts=%d (1..%d)", w->experts, GINEX_MAX_EXPERTS);
  if (w->turned != 0 && w->turned != 1) return fail(GINEX_ERR_ARG, "weights: turned=%d", w->turned);
  if (w->width < 1 || w->width > GINEX_MAX_WIDTH || w->out < 1 || w->out > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "weights: width %lld or out %lld (1..%d)", (long long)w->width, (long long)w->out, GINEX_MAX_WIDTH);
  const int64_t dense = w->turned ? w->width : w->out;
  if ((w->stride != 0 && w->stride < dense) || w->stride >= ((int64_t)1 << 31))
    return fail(GINEX_ERR_ARG, "weights: stride %lld below %lld, or too large", (long long)w->stride, (long long)dense);
  if (w->expert_stride < 0 || w->expert_stride > ((int64_t)1 << 42))
    return fail(GINEX_ERR_ARG, "weights: expert_stride=%lld", (long long)w->expert_stride);
  if (!w->data) return fail(GINEX_ERR_ARG, "weights: null data");
  if (reinterpret_cast<uintptr_t>(w->data) % element_bytes(w->type))
    return fail(GINEX_ERR_ARG, "weights: not aligned to their elements");
  return GINEX_OK;
}

inline int32_t check_vector(const char* what, const void* v, int32_t type) {
  if (reinterpret_cast<uintptr_t>(v) % element_bytes(type)) return fail(GINEX_ERR_ARG, "%s: not aligned to its elements", what);
  return GINEX_OK;
}

template <typename T>
inline WeightsOf<T> weights_of(const ginex_weights_t* w) {
  return {static_cast<const T*>(w->data), w->stride, w->expert_stride};
}

}  // namespace ginex
