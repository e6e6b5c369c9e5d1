// Gradients of biases: dbias[e] = sum over the slots s of expert e of dy[s], bound by HBM (152 000 x 256 bf16 12.4 us, 6.3 TB/s,
// and 4.1 for the parts of 8 experts).
//
// The slots are cut into tiles of equal height that no two experts share.  A workgroup adds up the columns of a tile, a lane
// a chunk of 16 bytes of every so many rows, and leaves a part; a second launch adds the parts up in their order.
#include "joins.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;

// Chunks of a workgroup beside each other, rows of a tile: by the sizes alone.
struct Cut {
  int32_t shift, height;
  int64_t tiles, columns;       // of tiles
};
Cut cut_of(int64_t slots, int32_t experts, int64_t width, int chunk) {
  Cut c;
  const int64_t cpr = ceil_div(width, chunk);
  c.shift = 0;
  while (c.shift < 6 && 1 << c.shift < cpr) ++c.shift;
  c.columns = ceil_div(cpr, 1 << c.shift);
  c.height = 64;
  while (c.height < 1 << 30 && slots / c.height * c.columns > 2048) c.height *= 2;
  c.tiles = most_tiles(slots, experts, c.height);
  return c;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void k_bias(RowsOf<const T> dy, const int64_t* __restrict__ offsets, int32_t experts,
                                                  int64_t slots, Width width, int32_t shift, int32_t height,
                                                  float* __restrict__ part) {
  constexpr int N = Chunk<T>::N, U = 4;
  __shared__ float sums[THREADS][N + 1];
  TileRows tile = {0, (int64_t)blockIdx.x * height, slots};
  if (offsets) {
    if (!find_tile(offsets, experts, slots, blockIdx.x, height, tile) || tile.expert == experts) return;
  }
  if (tile.end > tile.first + height) tile.end = tile.first + height;
  const int32_t beside = 1 << shift, rows = THREADS >> shift;
  const int32_t c = ((int32_t)blockIdx.y * beside + (threadIdx.x & (beside - 1))) * N;
  float sum[N] = {};
  // U rows in flight; one behind the end is read as the last and not counted
  for (int64_t r = tile.first + (threadIdx.x >> shift); r < tile.end; r += U * rows) {
    float v[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = r + u * rows;
      load_chunk(dy.at(at < tile.end ? at : tile.end - 1), c, width, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += r + u * rows < tile.end ? v[u][i] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) sums[threadIdx.x][i] = sum[i];
  __syncthreads();
  // a thread a column of the workgroup's, in the order of its rows
  for (int32_t k = threadIdx.x; k < beside * N; k += THREADS) {
    const int32_t column = (int32_t)blockIdx.y * beside * N + k;
    if (column >= width.width) break;
    float total = 0.f;
    for (int32_t s = 0; s < rows; ++s) total += sums[s * beside + k / N][k % N];
    part[(int64_t)blockIdx.x * width.width + column] = total;
  }
}

int32_t check_sizes(int64_t slots, int32_t experts, int64_t width) {
  if (slots < 0 || slots >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "slots=%lld", (long long)slots);
  if (experts < 1 || experts > GINEX_MAX_EXPERTS) return fail(GINEX_ERR_ARG, "experts=%d (1..%d)", experts, GINEX_MAX_EXPERTS);
  if (width < 1 || width > GINEX_MAX_WIDTH) return fail(GINEX_ERR_ARG, "width=%lld (1..%d)", (long long)width, GINEX_MAX_WIDTH);
  return GINEX_OK;
}

// (of 16-bit rows, which have the fewer columns of tiles and so the more tiles)
size_t space_of(int64_t slots, int32_t experts, int64_t width) {
  int64_t tiles = 0;
  for (int chunk = 4; chunk <= 8; chunk += 4) {
    const Cut c = cut_of(slots, experts, width, chunk);
    tiles = c.tiles > tiles ? c.tiles : tiles;
  }
  return (size_t)tiles * (size_t)width * sizeof(float) + 256;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

extern "C" size_t ginex_bias_gradient_workspace_bytes(int64_t slots, int32_t experts, int64_t width) {
  if (check_sizes(slots, experts, width)) return 0;
  return space_of(slots, experts, width);
}

extern "C" int32_t ginex_bias_gradient(const ginex_rows_t* dy, const ginex_routing_t* route, float* dbias, void* ws,
                                       size_t ws_bytes, void* stream) {
  if (int32_t rc = check_rows("dy", dy, false)) return rc;
  int32_t experts = 1;
  if (route) {
    if (int32_t rc = check_routing(route)) return rc;
    if (dy->rows != route->rows * route->top)
      return fail(GINEX_ERR_ARG, "dy has %lld rows, the routing %lld slots", (long long)dy->rows, (long long)(route->rows * route->top));
    experts = route->experts;
  }
  if (!dbias || reinterpret_cast<uintptr_t>(dbias) % 4) return fail(GINEX_ERR_ARG, "dbias: null or misaligned");
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(GINEX_ERR_ARG, "workspace: null or misaligned");
  const size_t need = space_of(dy->rows, experts, dy->width);
  if (ws_bytes < need) return fail(GINEX_ERR_WORKSPACE, "workspace: need %zu bytes, got %zu", need, ws_bytes);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  float* const part = static_cast<float*>(ws);
  const int64_t* const offsets = route ? route->offsets : nullptr;
  const Cut cut = cut_of(dy->rows, experts, dy->width, 16 / element_bytes(dy->type));
  if (dy->rows > 0) {
    const int32_t rc = with_type(dy->type, [&](auto t) -> int32_t {
      using T = decltype(t);
      hipLaunchKernelGGL(k_bias<T>, dim3((unsigned)cut.tiles, (unsigned)cut.columns), dim3(THREADS), 0, st, read_rows<T>(dy),
                         offsets, experts, dy->rows, Width::of<T>(dy->width), cut.shift, cut.height, part);
      GINEX_LAUNCH_CHECK();
      return GINEX_OK;
    });
    if (rc) return rc;
  }
  // (of a single sum's tiles one may have no rows: its part is zeros, and is not read)
  const int64_t parts = route ? cut.tiles : ceil_div(dy->rows, cut.height);
  GINEX_HIP(join_async(part, offsets, experts, dy->rows, cut.height, parts, (int32_t)dy->width, (int32_t)dy->width, dbias,
                       nullptr, st));
  return GINEX_OK;
}
