// Sums of parts that workgroups left in the workspace, added up in their order: columns of f32.
#pragma once

#include "layers.hpp"

namespace ginex {

constexpr int JOIN_COLUMNS = 32, JOIN_SLICES = 32;

// out[group][c] = the sum of parts[p][c] over the parts p of the group; columns from `split` on go to `more`.  Groups are
// experts with a part for every tile of `height` slots (offsets not NULL), or one with all `parts`.  32 threads a column
// take every 32nd part each, and are added up in their order.
static __global__ __launch_bounds__(JOIN_COLUMNS* JOIN_SLICES) void k_join(const float* __restrict__ part,
                                                                           const int64_t* __restrict__ offsets,
                                                                           int32_t experts, int64_t slots, int32_t height,
                                                                           int64_t parts, int32_t columns, int32_t split,
                                                                           float* __restrict__ out,
                                                                           float* __restrict__ more) {
  __shared__ float sums[JOIN_SLICES][JOIN_COLUMNS + 1];
  const int32_t column = threadIdx.x % JOIN_COLUMNS, slice = threadIdx.x / JOIN_COLUMNS;
  const int32_t c = blockIdx.x * JOIN_COLUMNS + column, group = blockIdx.y;
  int64_t first = 0, end = parts;
  if (offsets) {
    uint32_t before = 0;
    for (int32_t e0 = 0; e0 <= group; e0 += WAVE) {
      const int32_t e = e0 + lane_id();
      uint32_t tiles = 0;
      if (e <= group) {
        int64_t begin = offsets[e], until = offsets[e + 1];
        bound_slots(slots, begin, until);
        tiles = (uint32_t)(until - begin + height - 1) / (uint32_t)height;
      }
      const uint32_t upto = wave_inclusive_scan(tiles);
      if (group < e0 + WAVE) {
        first = before + of_lane(upto, group - e0) - of_lane(tiles, group - e0);
        end = before + of_lane(upto, group - e0);
      }
      before += of_lane(upto, WAVE - 1);
    }
    end = end < parts ? end : parts;        // (offsets that do not ascend name more tiles than there are)
  }
  float sum = 0.f;
  if (c < columns) {
    constexpr int U = 8;
    int64_t p = first + slice;
    for (; p + (U - 1) * JOIN_SLICES < end; p += U * JOIN_SLICES) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = part[(p + u * JOIN_SLICES) * columns + c];
#pragma unroll
      for (int u = 0; u < U; ++u) sum += v[u];
    }
    for (; p < end; p += JOIN_SLICES) sum += part[p * columns + c];
  }
  sums[slice][column] = sum;
  __syncthreads();
  if (slice > 0 || c >= columns) return;
#pragma unroll
  for (int s = 1; s < JOIN_SLICES; ++s) sum += sums[s][column];
  if (c < split) out[(int64_t)group * split + c] = sum;
  else more[(int64_t)group * (columns - split) + c - split] = sum;
}

inline hipError_t join_async(const float* part, const int64_t* offsets, int32_t experts, int64_t slots, int32_t height,
                             int64_t parts, int32_t columns, int32_t split, float* out, float* more, hipStream_t st) {
  hipLaunchKernelGGL(k_join, dim3((unsigned)ceil_div(columns, JOIN_COLUMNS), (unsigned)experts),
                     dim3(JOIN_COLUMNS * JOIN_SLICES), 0, st, part, offsets, experts, slots, height, parts, columns, split, out,
                     more);
  return hipGetLastError();
}

}  // namespace ginex
