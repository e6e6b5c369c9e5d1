// Linear layers with their epilogue, one for all rows or one per expert:
//
//   y[s] = f(x[source(s)] W_e + bias_e) + residual[s]
//
// A workgroup has a tile of rows and 64 columns a wave.  It goes through the width 128 bytes of a row at a time: rows and
// weights come from HBM into registers while the matrix cores work on the step before, and go to LDS with the width as the
// dense direction (weights that have it as the other one are turned over on the way, in registers).  The columns are the
// matrix instruction's first operand and are dealt to its rows so that a lane ends up with 16 neighbouring columns of one
// row: bias, activation, residual, codes and rounding are done in registers and stored in whole chunks.
#include "epilogue.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;
constexpr int CHUNKS = 8;         // of a row in LDS: 128 bytes
// Where chunk c of row r of a tile is in LDS.  Lanes that read or write together (8 at a time) differ in the lowest three bits
// of the row; of the weights' rows in bits 0, 1 and 4 (read), or 2, 3 and 4 (written turned over).
__device__ __forceinline__ int row_chunk(int r, int c) { return r * CHUNKS + (c ^ (r & 7)); }
__device__ __forceinline__ int column_chunk(int n, int c) {
  return n * CHUNKS + (c ^ (((n ^ n >> 2) & 3) | (n >> 4 & 1) << 2));
}

// WM x WN waves of 16 MT rows and 64 columns.  TURNED: the weights have the width as their dense direction.
template <typename T, int MT, int WM, int WN, bool TURNED>
__global__ __launch_bounds__(THREADS, 2) void k_linear(RowsOf<const T> x, int64_t rows, WeightsOf<T> weights,
                                                       const int32_t* __restrict__ source,
                                                       const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                                       int32_t width, Width out, uint32_t first_tile, uint32_t tiles,
                                                       Divisor tiles_n, Epilogue epilogue) {
  constexpr int N = Chunk<T>::N, NT = 4, BM = 16 * MT * WM, BN = WAVE_COLUMNS * WN, DEPTH = CHUNKS * N;
  constexpr int AN = BM * CHUNKS / THREADS;                       // chunks of rows a thread fetches
  constexpr int BN_CHUNKS = BN * CHUNKS / THREADS;                // and of weights, turned
  constexpr int ALL_BLOCKS = CHUNKS * BN / 4;                     // or blocks of N x 4 of them
  constexpr int BLOCKS = (ALL_BLOCKS + THREADS - 1) / THREADS;
  static_assert(WM * WN * WAVE == THREADS && AN >= 1 && (ALL_BLOCKS % THREADS == 0 || ALL_BLOCKS < THREADS), "chunks of a thread");
  __shared__ words4 lds[(BM + BN) * CHUNKS];
  words4* const lds_a = lds;
  words4* const lds_b = lds + BM * CHUNKS;

  // Workgroups go to the 8 dies in turn: the tiles of the same rows follow each other on one die, whose cache has the rows.
  const uint32_t turn = blockIdx.x / 8, m_of = tiles_n.of(turn);
  const uint32_t tile_m = m_of * 8 + blockIdx.x % 8, tile_n = turn - m_of * tiles_n.d;
  if (tile_m >= tiles) return;
  const int32_t n0 = (int32_t)tile_n * BN;
  TileRows tile = {0, (int64_t)(first_tile + tile_m) * BM, slots};
  if (offsets) {
    if (!find_tile(offsets, experts, slots, first_tile + tile_m, BM, tile)) return;
  }
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int wm = wave % WM, wn = wave / WM, group = lane / 16;
  const int32_t c0 = n0 + wn * WAVE_COLUMNS + group * LANE_COLUMNS;
  if (tile.expert == experts) {                 // slots without an expert
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int64_t r = tile.first + (wm * MT + m) * 16 + lane % 16;
      if (r < tile.end) clear_columns<T>(epilogue, r, c0, out);
    }
    return;
  }
  const T* const w = weights.of(tile.expert);

  // What a thread fetches: chunk t % 8 of rows t / 8, t / 8 + 32, ..  A row behind the end repeats the last one: its sums
  // are not written.
  const T* a_row[AN];
  bool a_there[AN];
#pragma unroll
  for (int i = 0; i < AN; ++i) {
    int64_t r = tile.first + threadIdx.x / CHUNKS + i * (THREADS / CHUNKS);
    r = r < tile.end ? r : tile.end - 1;
    if (source) r = source[r];
    a_there[i] = r >= 0 && r < rows;
    a_row[i] = x.at(a_there[i] ? r : 0);
  }
  const Width along = {width, (int32_t)((width + N - 1) / N * N - width)};
  ChunkWords<T> a[AN], b[BN_CHUNKS];
  typename Four<T>::Wide b4[BLOCKS][N];
  auto fetch = [&](int32_t k0) {
#pragma unroll
    for (int i = 0; i < AN; ++i) a[i] = load_words(a_row[i], k0 + (int)threadIdx.x % CHUNKS * N, along);
    if (TURNED) {
#pragma unroll
      for (int i = 0; i < BN_CHUNKS; ++i) {
        int32_t n = n0 + threadIdx.x / CHUNKS + i * (THREADS / CHUNKS);
        n = n < out.width ? n : out.width - 1;
        b[i] = load_words(w + n * weights.stride, k0 + (int)threadIdx.x % CHUNKS * N, along);
      }
    } else {
      // a block: N of the width's numbers, 4 columns; the last columns are read so that they end with the row
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        const int q = threadIdx.x + i * THREADS;
        if (ALL_BLOCKS < THREADS && q >= ALL_BLOCKS) break;
        const int32_t n = n0 + q % (BN / 4) * 4, k = k0 + q / (BN / 4) * N;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const bool there = k + j < width;
          const T* const row = w + (int64_t)(there ? k + j : width - 1) * weights.stride;
          if (out.width < 4) {
#pragma unroll
            for (int l = 0; l < 4; ++l) b4[i][j][l] = l < out.width ? row[l] : (T)0.f;
          } else {
            b4[i][j] = *reinterpret_cast<const typename Four<T>::At*>(row + (n < out.width - 4 ? n : out.width - 4));
          }
          if (!there) b4[i][j] = (typename Four<T>::Wide)(T)0.f;
        }
      }
    }
  };
  auto put = [&]() {
#pragma unroll
    for (int i = 0; i < AN; ++i)
      lds_a[row_chunk(threadIdx.x / CHUNKS + i * (THREADS / CHUNKS), threadIdx.x % CHUNKS)] =
          a_there[i] ? a[i].words : words4{0, 0, 0, 0};
    if (TURNED) {
#pragma unroll
      for (int i = 0; i < BN_CHUNKS; ++i)
        lds_b[column_chunk(threadIdx.x / CHUNKS + i * (THREADS / CHUNKS), threadIdx.x % CHUNKS)] = b[i].words;
    } else {
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        const int q = threadIdx.x + i * THREADS;
        if (ALL_BLOCKS < THREADS && q >= ALL_BLOCKS) break;
        int32_t n = n0 + q % (BN / 4) * 4;
        n = (out.width < 4 || n < out.width - 4 ? n : out.width - 4) - n0;      // (several may put the same there)
#pragma unroll
        for (int l = 0; l < 4; ++l) {
          ChunkWords<T> u;
#pragma unroll
          for (int j = 0; j < N; ++j) u.wide[j] = b4[i][j][l];
          if (n + l >= 0) lds_b[column_chunk(n + l, q / (BN / 4))] = u.words;
        }
      }
    }
  };

  float4v sum[MT][NT] = {};
  fetch(0);
  for (int32_t k0 = 0; k0 < width; k0 += DEPTH) {
    if (k0 > 0) lds_barrier();
    put();
    lds_barrier();
    if (k0 + DEPTH < width) fetch(k0 + DEPTH);
#pragma unroll
    for (int k = 0; k < CHUNKS / 4; ++k) {
      ChunkWords<T> fa[MT], fb[NT];
#pragma unroll
      for (int m = 0; m < MT; ++m) fa[m].words = lds_a[row_chunk((wm * MT + m) * 16 + lane % 16, 4 * k + group)];
      // operand row 4 g + i of product n is column 16 g + 4 n + i
#pragma unroll
      for (int n = 0; n < NT; ++n)
        fb[n].words = lds_b[column_chunk(wn * WAVE_COLUMNS + lane % 16 / 4 * 16 + 4 * n + lane % 4, 4 * k + group)];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) sum[m][n] = product(fb[n], fa[m], sum[m][n]);
    }
  }

  float bias[LANE_COLUMNS];
  load_bias<T>(epilogue, tile.expert, c0, out, bias);
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t r = tile.first + (wm * MT + m) * 16 + lane % 16;
    float v[LANE_COLUMNS];
#pragma unroll
    for (int i = 0; i < LANE_COLUMNS; ++i) v[i] = sum[m][i / 4][i % 4] + bias[i];
    if (r < tile.end) {
      Columns<T> residual;
      if (epilogue.residual) residual.load(static_cast<const T*>(epilogue.residual) + r * epilogue.residual_stride, c0, out);
      finish<T>(epilogue, r, c0, n0 + (wn + 1) * WAVE_COLUMNS <= out.width, out, v, residual);
    }
  }
}

}  // namespace
}  // namespace ginex

using namespace ginex;

namespace {

template <typename T, int MT, int WM, int WN>
int32_t launch(const ginex_rows_t* x, const ginex_weights_t* w, const ginex_routing_t* route, bool by_slot, int64_t slots,
               const Epilogue& epilogue, hipStream_t st) {
  constexpr int BM = 16 * MT * WM, BN = WAVE_COLUMNS * WN;
  const int64_t tiles_n = ceil_div(w->out, BN);
  const int64_t tiles_m = route ? most_tiles(slots, route->experts, BM) : ceil_div(slots, BM);
  const auto kernel = w->turned ? k_linear<T, MT, WM, WN, true> : k_linear<T, MT, WM, WN, false>;
  // (a launch has fewer than 2^32 threads)
  const int64_t step = ((int64_t)1 << 23) / tiles_n / 8 * 8;
  for (int64_t m = 0; m < tiles_m; m += step) {
    const int64_t tiles = tiles_m - m < step ? tiles_m - m : step;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(tiles, 8) * 8 * tiles_n)), dim3(THREADS), 0, st, read_rows<T>(x),
                       x->rows, weights_of<T>(w), route && !by_slot ? route->source : nullptr,
                       route ? route->offsets : nullptr, w->experts, slots, (int32_t)w->width, Width::of<T>(w->out),
                       (uint32_t)m, (uint32_t)tiles, Divisor((uint32_t)tiles_n), epilogue);
    GINEX_LAUNCH_CHECK();
  }
  return GINEX_OK;
}

}  // namespace

extern "C" int32_t ginex_linear(const ginex_rows_t* x, const ginex_weights_t* weights, const void* bias, int32_t activation,
                                const ginex_rows_t* residual, const ginex_routing_t* route, int32_t by_slot,
                                const ginex_rows_t* y, const ginex_codes_t* kept, void* stream) {
  if (int32_t rc = check_rows("x", x, false)) return rc;
  if (int32_t rc = check_weights(weights)) return rc;
  if (int32_t rc = check_rows("y", y, true)) return rc;
  if (int32_t rc = check_activation(activation, GINEX_ACT_NONE)) return rc;
  if (x->type != weights->type) return fail(GINEX_ERR_ARG, "x and weights differ in type");
  if (x->type != y->type) return fail(GINEX_ERR_ARG, "x and y differ in type");
  if (x->width != weights->width)
    return fail(GINEX_ERR_ARG, "x is %lld wide, the weights take %lld", (long long)x->width, (long long)weights->width);
  if (y->width != weights->out)
    return fail(GINEX_ERR_ARG, "y is %lld wide, the weights give %lld", (long long)y->width, (long long)weights->out);
  if (int32_t rc = check_vector("bias", bias, x->type)) return rc;
  int64_t slots = x->rows;
  if (route) {
    if (int32_t rc = check_routing(route)) return rc;
    if (route->experts != weights->experts)
      return fail(GINEX_ERR_ARG, "weights of %d experts, a routing to %d", weights->experts, route->experts);
    slots = route->rows * route->top;
    const int64_t need = by_slot ? slots : route->rows;
    if (x->rows != need)
      return fail(GINEX_ERR_ARG, "x has %lld rows, the routing %lld %s", (long long)x->rows, (long long)need, by_slot ? "slots" : "rows");
  } else {
    if (weights->experts != 1) return fail(GINEX_ERR_ARG, "weights of %d experts without a routing", weights->experts);
    if (by_slot) return fail(GINEX_ERR_ARG, "rows by slot without a routing");
  }
  if (y->rows != slots) return fail(GINEX_ERR_ARG, "y has %lld rows, expected %lld", (long long)y->rows, (long long)slots);
  if (residual) {
    if (int32_t rc = check_rows("residual", residual, false)) return rc;
    if (int32_t rc = check_same("residual", residual, "y", y)) return rc;
    if (residual->rows != slots)
      return fail(GINEX_ERR_ARG, "residual has %lld rows, y %lld", (long long)residual->rows, (long long)slots);
  }
  if (kept) {
    if (int32_t rc = check_codes(kept)) return rc;
    if (int32_t rc = check_kept("y", y, kept)) return rc;
  }
  if (slots == 0) return GINEX_OK;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const Epilogue epilogue = {bias,
                             residual ? residual->data : nullptr,
                             residual ? residual->stride : 0,
                             y->data,
                             y->stride,
                             kept ? kept->codes : nullptr,
                             kept ? kept->scales : nullptr,
                             (int32_t)code_blocks(weights->out),
                             activation};
  if (slots <= FEW_ROWS) return linear_few(x, weights, route, by_slot != 0, slots, epilogue, st);
  if (resident_fits(weights, slots, route != nullptr))
    return linear_resident(x, weights, route, by_slot != 0, slots, epilogue, st);
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const int64_t groups = route ? route->experts : 1;
    const auto tiles = [&](int height) { return (slots / height + groups) * ceil_div(weights->out, 128); };
    if (weights->out <= WAVE_COLUMNS) {
      if (tiles(128) >= 1024) return launch<T, 2, 4, 1>(x, weights, route, by_slot, slots, epilogue, st);
      return launch<T, 1, 4, 1>(x, weights, route, by_slot, slots, epilogue, st);
    }
    if (tiles(128) >= 512) return launch<T, 2, 2, 2>(x, weights, route, by_slot, slots, epilogue, st);
    return launch<T, 1, 2, 2>(x, weights, route, by_slot, slots, epilogue, st);
  });
}
