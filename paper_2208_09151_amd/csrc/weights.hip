// Weight gradients of one linear layer per expert, from rows kept in 8 bits:
//
//   dw[e][c][d] = sum over the slots s of expert e of  x(source[s], c) * dy(s, d)
//
// A product of two matrices whose long axis, the slots, is cut into pieces of equal length within the
// experts, so that few experts or uneven ones still fill the GPU.  An expert of one piece is written where
// it belongs; the pieces of a longer one go to the workspace and are added up in their order by a second
// launch, so that equal inputs give equal bits.
#include "codes.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;
constexpr int TILE = 64;          // channels and outputs of a workgroup
constexpr int DEPTH = 16;         // slots in LDS at a time

// The pieces of all experts: ceil(slots of the expert / length) each, numbered in order.
struct Piece {
  int32_t expert;      // -1: no such piece
  int64_t begin, end;  // its slots
  int32_t part;        // its place in the workspace; -1: the expert's only piece
};

struct Shares {
  int64_t length;      // slots of a piece
  int64_t pieces;      // at most, of all experts
  int64_t parts;       // at most, of experts with more than one
};

// An expert's slots; a routing that was not made by ginex_route cannot name slots that are not there.
__device__ __forceinline__ void slots_of(const int64_t* __restrict__ offsets, int32_t e, int64_t slots, int64_t& begin,
                                         int64_t& end) {
  begin = offsets ? offsets[e] : 0;
  end = offsets ? offsets[e + 1] : slots;
  begin = begin < 0 ? 0 : (begin < slots ? begin : slots);
  end = end < begin ? begin : (end < slots ? end : slots);
}

__device__ __forceinline__ Piece find_piece(const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                            int64_t length, int64_t wanted, int64_t most_parts, Piece* found,
                                            uint32_t* smem) {
  if (threadIdx.x == 0) *found = {-1, 0, 0, -1};
  __syncthreads();
  uint32_t pieces_before = 0, parts_before = 0;
  for (int32_t e0 = 0; e0 < experts; e0 += THREADS) {
    const int32_t e = e0 + (int32_t)threadIdx.x;
    int64_t begin = 0, end = 0;
    if (e < experts) slots_of(offsets, e, slots, begin, end);
    const uint32_t pieces = (uint32_t)((end - begin + length - 1) / length);
    const uint32_t parts = pieces > 1 ? pieces : 0;
    uint32_t all_pieces, all_parts;
    const uint32_t piece = pieces_before + block_exclusive_scan<uint32_t, THREADS>(pieces, smem, all_pieces);
    const uint32_t part = parts_before + block_exclusive_scan<uint32_t, THREADS>(parts, smem, all_parts);
    // (parts beyond the workspace: offsets that do not ascend, which ginex_route does not make)
    if (wanted >= piece && wanted < piece + pieces && (parts == 0 || part + (wanted - piece) < most_parts)) {
      const int64_t at = begin + (wanted - piece) * length;
      *found = {e, at, at + length < end ? at + length : end, parts ? (int32_t)(part + (wanted - piece)) : -1};
    }
    pieces_before += all_pieces;
    parts_before += all_parts;
  }
  __syncthreads();
  return *found;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void k_weights(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                     int64_t rows, int32_t blocks, const int32_t* __restrict__ source,
                                                     const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                                     int64_t length, int64_t most_parts, RowsOf<const T> dy, int32_t width,
                                                     int32_t out_width, float* __restrict__ dw, float* __restrict__ partial) {
  __shared__ uint32_t smem[THREADS / WAVE + 1];
  __shared__ Piece found;
  __shared__ float xs[DEPTH][TILE], ys[DEPTH][TILE];
  const Piece piece = find_piece(offsets, experts, slots, length, blockIdx.z, most_parts, &found, smem);
  if (piece.expert < 0) return;
  const int32_t c0 = blockIdx.x * TILE, d0 = blockIdx.y * TILE;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float sum[4][4] = {};
  for (int64_t s0 = piece.begin; s0 < piece.end; s0 += DEPTH) {
    __syncthreads();
    for (int i = threadIdx.x; i < DEPTH * TILE; i += THREADS) {
      const int k = i / TILE, col = i % TILE;
      const int64_t s = s0 + k;
      float x = 0.f, y = 0.f;
      if (s < piece.end) {
        const int64_t r = source ? source[s] : s;
        const int32_t c = c0 + col, d = d0 + col;
        if (r >= 0 && r < rows && c < width)
          x = (float)codes[r * blocks * GINEX_CODE_BLOCK + c] * code_step(scales[r * blocks + c / GINEX_CODE_BLOCK]);
        if (r >= 0 && r < rows && d < out_width) y = (float)*dy.at(s, d);
      }
      xs[k][col] = x;
      ys[k][col] = y;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < DEPTH; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][j] = fmaf(xs[k][ty * 4 + i], ys[k][tx * 4 + j], sum[i][j]);
  }
  const int64_t size = (int64_t)width * out_width;
  float* const to = piece.part < 0 ? dw + piece.expert * size : partial + piece.part * size;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int32_t c = c0 + ty * 4 + i, d = d0 + tx * 4 + j;
      if (c < width && d < out_width) to[(int64_t)c * out_width + d] = sum[i][j];
    }
}

// Experts of several pieces: added up in order.  Experts without slots: cleared.
__global__ __launch_bounds__(THREADS) void k_weights_join(const int64_t* __restrict__ offsets, int32_t experts,
                                                          int64_t slots, int64_t length, int64_t most_parts, int64_t size,
                                                          const float* __restrict__ partial, float* __restrict__ dw) {
  __shared__ uint32_t smem[THREADS / WAVE + 1];
  const int32_t mine = blockIdx.y;
  uint32_t before = 0;
  for (int32_t e0 = 0; e0 < mine; e0 += THREADS) {
    const int32_t e = e0 + (int32_t)threadIdx.x;
    int64_t begin = 0, end = 0;
    if (e < mine) slots_of(offsets, e, slots, begin, end);
    const uint32_t pieces = (uint32_t)((end - begin + length - 1) / length);
    uint32_t total;
    block_exclusive_scan<uint32_t, THREADS>(pieces > 1 ? pieces : 0, smem, total);
    before += total;
  }
  int64_t begin, end;
  slots_of(offsets, mine, slots, begin, end);
  const int64_t pieces = (end - begin + length - 1) / length;
  if (pieces == 1) return;
  for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < size; i += (int64_t)gridDim.x * THREADS) {
    float sum = 0.f;
    for (int64_t p = 0; p < pieces && before + p < most_parts; ++p) sum += partial[(before + p) * size + i];
    dw[mine * size + i] = sum;
  }
}

Shares shares_of(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  const int64_t tiles = ceil_div(width, TILE) * ceil_div(out_width, TILE);
  int64_t cuts = ceil_div(1024, tiles);
  const int64_t most = ceil_div(slots, 512);
  cuts = cuts < most ? cuts : most;
  cuts = cuts < 1 ? 1 : cuts;
  Shares s;
  s.length = ceil_div(ceil_div(slots, cuts), DEPTH) * DEPTH;
  if (s.length < DEPTH) s.length = DEPTH;
  // sum over the experts of ceil(n / length), for those of more than one piece: fewer than cuts of them
  s.pieces = cuts + experts;
  s.parts = cuts + (experts < cuts ? experts : cuts);
  return s;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

static int32_t check_sizes(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  if (slots < 0 || slots >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "slots=%lld", (long long)slots);
  if (experts < 1 || experts > GINEX_MAX_EXPERTS) return fail(GINEX_ERR_ARG, "experts=%d (1..%d)", experts, GINEX_MAX_EXPERTS);
  if (width < 1 || width > GINEX_MAX_WIDTH || out_width < 1 || out_width > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "%lld x %lld weights (1..%d each)", (long long)width, (long long)out_width, GINEX_MAX_WIDTH);
  return GINEX_OK;
}

extern "C" size_t ginex_weight_gradient_workspace_bytes(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  if (check_sizes(slots, experts, width, out_width) != GINEX_OK) return 0;
  Arena a(nullptr);
  a.take<float>(shares_of(slots, experts, width, out_width).parts * width * out_width);
  a.take<char>(256);
  return a.used;
}

extern "C" int32_t ginex_weight_gradient(const ginex_codes_t* kept, const ginex_routing_t* route, const ginex_rows_t* dy,
                                         float* dw, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_codes(kept)) return rc;
  if (route)
    if (int32_t rc = check_routing(route)) return rc;
  if (int32_t rc = check_rows("dy", dy, false)) return rc;
  if (route && route->rows != kept->rows)
    return fail(GINEX_ERR_ARG, "the routing has %lld rows, the codes %lld", (long long)route->rows, (long long)kept->rows);
  const int64_t slots = route ? route->rows * route->top : kept->rows;
  const int32_t experts = route ? route->experts : 1;
  if (dy->rows != slots) return fail(GINEX_ERR_ARG, "dy has %lld rows for %lld slots", (long long)dy->rows, (long long)slots);
  if (!dw || reinterpret_cast<uintptr_t>(dw) % 4) return fail(GINEX_ERR_ARG, "dw: null or misaligned");
  const size_t need = ginex_weight_gradient_workspace_bytes(slots, experts, kept->width, dy->width);
  if (need == 0) return GINEX_ERR_ARG;
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256)
    return fail(GINEX_ERR_ARG, "weight gradient: null or misaligned workspace (256 bytes)");
  if (ws_bytes < need) return fail(GINEX_ERR_WORKSPACE, "weight gradient: workspace %zu bytes, need %zu", ws_bytes, need);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const Shares share = shares_of(slots, experts, kept->width, dy->width);
  const int32_t* const source = route ? route->source : nullptr;
  const int64_t* const offsets = route ? route->offsets : nullptr;
  float* const partial = static_cast<float*>(ws);
  const int64_t size = kept->width * dy->width;
  return with_type(dy->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const dim3 grid((unsigned)ceil_div(kept->width, TILE), (unsigned)ceil_div(dy->width, TILE), (unsigned)share.pieces);
    hipLaunchKernelGGL(k_weights<T>, grid, dim3(THREADS), 0, st, kept->codes, kept->scales, kept->rows,
                       (int32_t)code_blocks(kept->width), source, offsets, experts, slots, share.length,
                       share.parts, RowsOf<const T>{static_cast<const T*>(dy->data), dy->stride}, (int32_t)kept->width,
                       (int32_t)dy->width, dw, partial);
    GINEX_LAUNCH_CHECK();
    const int64_t blocks = ceil_div(size, THREADS);
    hipLaunchKernelGGL(k_weights_join, dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)experts), dim3(THREADS), 0,
                       st, offsets, experts, slots, share.length, share.parts, size, partial, dw);
    GINEX_LAUNCH_CHECK();
    return GINEX_OK;
  });
}
