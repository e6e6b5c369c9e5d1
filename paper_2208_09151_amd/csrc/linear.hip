// Linear layers with their epilogue, one for all rows or one per expert:
//
//   y[s] = f(x[source(s)] W_e + bias_e) + residual[s]
//
// A workgroup has a tile of rows and 64 columns a wave.  It goes through the width 128 bytes of a row at a time: rows and
// weights come from HBM into registers while the matrix cores work on the step before, and go to LDS as operands, with the
// width as the dense direction (weights that have it as the other one are turned over on the way, in registers; f32 is cut into
// its parts).  The columns are the matrix instruction's first operand and are dealt to its rows so that a lane ends up with 16
// neighbouring columns of one row: bias, activation, residual, codes and rounding are done in registers and stored in whole
// chunks.
//
// Bound by LDS and two barriers a step, which feed the matrix cores, where width and columns are many, by HBM where they are few:
// 50 000 x 1024 -> 1024 bf16 180 us, 583 TFLOP/s (198 where torch's product takes 144 on the same inputs; f32, with six products
// for an operand that is brought, 662 and 875); 152 000 slots of 8 experts, 256 -> 128 bf16 32 us, 3.6 TB/s of rows read and written.  The loads of a step are issued
// before the products of the one in front of it, with nothing between that depends on them (no branch, no arithmetic on what they
// bring), because a wave can only wait for its oldest loads: with the mending of ends right behind each load the first of these
// took 338 us.
#include "epilogue.hpp"
#include "parts.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;

// Where chunk c of row r is in LDS: a row has 8 chunks of 16 bits, or 4 of each part of f32.  8 lanes that read or write
// together use every bank once.  Those that read rows differ in the row's lowest three bits; those that read weights in bits 0, 1
// and 4 of the column.
template <int CHUNKS>
__device__ __forceinline__ int row_chunk(int r, int c) {
  return r * CHUNKS + (c ^ (CHUNKS == 8 ? r & 7 : r >> 1 & 3));
}
template <int CHUNKS>
__device__ __forceinline__ int column_chunk(int n, int c) {
  if (CHUNKS == 8) return n * CHUNKS + (c ^ (((n ^ n >> 2) & 3) | (n >> 4 & 1) << 2));
  return n * CHUNKS + (c ^ ((n >> 1 ^ n >> 2) & 1) ^ (n >> 3 & 2));
}

// WM x WN waves of 16 MT rows and 64 columns.  TURNED: the weights have the width as their dense direction.
template <typename T, int MT, int WM, int WN, bool TURNED>
__global__ __launch_bounds__(THREADS, 2) void k_linear(RowsOf<const T> x, int64_t rows, WeightsOf<T> weights,
                                                       const int32_t* __restrict__ source,
                                                       const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                                       int32_t width, Width out, uint32_t first_tile, uint32_t tiles,
                                                       Divisor tiles_n, Epilogue epilogue) {
  using K = typename Operand<T>::Kind;
  constexpr int N = Chunk<T>::N, UNIT = 8 * N, NT = 4, BM = 16 * MT * WM, BN = WAVE_COLUMNS * WN;
  constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, CHUNKS = UNIT / 8;        // of 8 numbers, a row's in LDS
  constexpr int FETCH = 8 / N;                                            // chunks of memory for one of LDS
  constexpr int AN = (BM * CHUNKS + THREADS - 1) / THREADS, BN_CHUNKS = BN * CHUNKS / THREADS;
  constexpr int ALL_BLOCKS = CHUNKS * BN / 4, BLOCKS = (ALL_BLOCKS + THREADS - 1) / THREADS;      // of 8 x 4 weights
  static_assert(WM * WN * WAVE == THREADS && BN_CHUNKS >= 1 && (BM * CHUNKS % THREADS == 0 || BM * CHUNKS < THREADS), "chunks of a thread");
  static_assert(ALL_BLOCKS % THREADS == 0 || ALL_BLOCKS < THREADS, "blocks of a thread");
  __shared__ words4 lds[(BM + BN) * CHUNKS * PARTS];
  words4* const lds_a = lds;
  words4* const lds_b = lds + BM * CHUNKS * PARTS;

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
#pragma unroll 1
    for (int m = 0; m < MT; ++m) {
      const int64_t r = tile.first + (wm * MT + m) * 16 + lane % 16;
      if (r < tile.end) clear_columns<T>(epilogue, r, c0, out);
    }
    return;
  }
  const T* const w = weights.of(tile.expert);

  // What a thread fetches: chunk t % CHUNKS of rows t / CHUNKS, ..  A row behind the end repeats the last one: its sums are not
  // written.
  const T* a_row[AN];
  bool a_there[AN];
#pragma unroll
  for (int i = 0; i < AN; ++i) {
    int64_t r = tile.first + threadIdx.x / CHUNKS + i * (THREADS / CHUNKS);
    r = r < tile.end ? r : tile.end - 1;
    if (source) r = source[r];
    a_there[i] = r >= 0 && r < rows;            // (without a source they are)
    a_row[i] = x.at(a_there[i] ? r : 0);
  }
  const Width along = {width, (int32_t)((width + N - 1) / N * N - width)};
  ChunkWords<T> a[AN][FETCH], b[TURNED ? BN_CHUNKS : 1][FETCH];
  typename Four<T>::Wide b4[TURNED ? 1 : BLOCKS][8];
  // Loads alone, which nothing looks at before put(): they are under way while the matrix cores work.
  const bool narrow = width < N, narrow_out = out.width < 4;         // (rows that are read element by element)
  auto fetch = [&](int32_t k0) {
    const int32_t k = k0 + (int)threadIdx.x % CHUNKS * 8;
#pragma unroll
    for (int i = 0; i < AN; ++i)
#pragma unroll
      for (int h = 0; h < FETCH; ++h) a[i][h] = narrow ? load_words(a_row[i], k + h * N, along) : read_words(a_row[i], k + h * N, along);
    if constexpr (TURNED) {
#pragma unroll
      for (int i = 0; i < BN_CHUNKS; ++i) {
        int32_t n = n0 + threadIdx.x / CHUNKS + i * (THREADS / CHUNKS);
        n = n < out.width ? n : out.width - 1;
#pragma unroll
        for (int h = 0; h < FETCH; ++h)
          b[i][h] = narrow ? load_words(w + n * weights.stride, k + h * N, along)
                           : read_words(w + n * weights.stride, k + h * N, along);
      }
    } else {
      // a block: 8 of the width's numbers, 4 columns, 0 where there are none (what is in LDS may leave no sum that is no number)
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        const int q = threadIdx.x + i * THREADS;
        if (ALL_BLOCKS < THREADS && q >= ALL_BLOCKS) break;
        int32_t n = n0 + q % (BN / 4) * 4;
        n = n < out.width ? n : out.width - 1;
        const int32_t k1 = k0 + q / (BN / 4) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const T* const row = w + (int64_t)(k1 + j < width ? k1 + j : width - 1) * weights.stride;
          b4[i][j] = narrow_out ? four_of(row, n, out.width) : four_read(row, n, out.width);
        }
      }
    }
  };
  // Eight numbers as they go to LDS.
  const auto put_eight = [&](words4* to, int stride, const ChunkWords<T>(&v)[FETCH]) {
    if constexpr (PARTS == 3) {
      ChunkWords<K> parts[PARTS];
      parts_of(v, parts);
#pragma unroll
      for (int z = 0; z < PARTS; ++z) to[z * stride] = parts[z].words;
    } else {
      *to = v[0].words;
    }
  };
  auto put = [&](int32_t k0) {
    const int32_t k = k0 + (int)threadIdx.x % CHUNKS * 8;
    if (k0 + UNIT > width && !narrow) {         // the row's end
#pragma unroll
      for (int h = 0; h < FETCH; ++h) {
#pragma unroll
        for (int i = 0; i < AN; ++i) a[i][h] = placed<T>(a[i][h], k + h * N, along);
        if constexpr (TURNED) {
#pragma unroll
          for (int i = 0; i < BN_CHUNKS; ++i) b[i][h] = placed<T>(b[i][h], k + h * N, along);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < AN; ++i) {
      if (BM * CHUNKS < THREADS && threadIdx.x >= BM * CHUNKS) break;
      if (source && !a_there[i]) {
#pragma unroll
        for (int h = 0; h < FETCH; ++h) a[i][h].words = words4{0, 0, 0, 0};
      }
      put_eight(lds_a + row_chunk<CHUNKS>(threadIdx.x / CHUNKS + i * (THREADS / CHUNKS), threadIdx.x % CHUNKS), BM * CHUNKS, a[i]);
    }
    if constexpr (TURNED) {
#pragma unroll
      for (int i = 0; i < BN_CHUNKS; ++i)
        put_eight(lds_b + column_chunk<CHUNKS>(threadIdx.x / CHUNKS + i * (THREADS / CHUNKS), threadIdx.x % CHUNKS), BN * CHUNKS, b[i]);
    } else {
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        const int q = threadIdx.x + i * THREADS;
        if (ALL_BLOCKS < THREADS && q >= ALL_BLOCKS) break;
        const int32_t n = q % (BN / 4) * 4, k1 = k0 + q / (BN / 4) * 8;
        if (n0 + BN > out.width && !narrow_out) {
          const int32_t at = n0 + n < out.width ? n0 + n : out.width - 1;
#pragma unroll
          for (int j = 0; j < 8; ++j) b4[i][j] = four_placed<T>(b4[i][j], at, out.width);
        }
        if (k0 + UNIT > width) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (k1 + j >= width) b4[i][j] = (typename Four<T>::Wide)(T)0.f;
        }
#pragma unroll
        for (int l = 0; l < 4; ++l) {
          ChunkWords<T> u[FETCH];
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j / N].wide[j % N] = b4[i][j][l];
          put_eight(lds_b + column_chunk<CHUNKS>(n + l, q / (BN / 4)), BN * CHUNKS, u);
        }
      }
    }
  };

  float4v sum[MT][NT] = {};
  fetch(0);
  for (int32_t k0 = 0; k0 < width; k0 += UNIT) {
    if (k0 > 0) lds_barrier();
    put(k0);
    lds_barrier();
    if (k0 + UNIT < width) fetch(k0 + UNIT);
    // operand row 4 g + i of product j is column 16 g + 4 j + i
    const auto column_of = [&](int t) { return wn * WAVE_COLUMNS + lane % 16 / 4 * 16 + t * 4 + lane % 4; };
#pragma unroll
    for (int k = 0; k < CHUNKS / 4; ++k) {
      ChunkWords<K> fa[MT][PARTS];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int z = 0; z < PARTS; ++z)
          fa[m][z].words = lds_a[z * BM * CHUNKS + row_chunk<CHUNKS>((wm * MT + m) * 16 + lane % 16, 4 * k + group)];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        ChunkWords<K> fb[PARTS];
#pragma unroll
        for (int z = 0; z < PARTS; ++z) fb[z].words = lds_b[z * BN * CHUNKS + column_chunk<CHUNKS>(column_of(t), 4 * k + group)];
        if constexpr (PARTS == 3) {
          products_of<K, MT>(fb, fa, &sum[0][t], NT);
        } else {
#pragma unroll
          for (int m = 0; m < MT; ++m) sum[m][t] = product(fb[0], fa[m][0], sum[m][t]);
        }
      }
    }
  }

  if constexpr (PARTS == 3) {
    if (any_none<MT * NT>(&sum[0][0])) {
#pragma unroll 1
      for (int m = 0; m < MT; ++m) {
        int64_t r = tile.first + (wm * MT + m) * 16 + lane % 16;
        r = r < tile.end ? r : tile.end - 1;
        r = source ? (int64_t)source[r] : r;
        const bool is = r >= 0 && r < rows;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          int32_t n = n0 + wn * WAVE_COLUMNS + lane % 16 / 4 * 16 + t * 4 + lane % 4;
          n = n < out.width ? n : out.width - 1;
          const float4v again = sums_again(x.at(is ? r : 0), is, w + (TURNED ? n * weights.stride : n), TURNED ? 1 : weights.stride,
                                           width, float4v{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int j = 0; j < MT; ++j)
            if (j == m) sum[j][t] = with_again(sum[j][t], again);
        }
      }
    }
  }
  // (a loop of one turn: what is in it is unrolled later and the row's end is looked at less often, 40 000 x 256 -> 256 bf16 with gelu
  // 20.3 instead of 21.3 us)
#pragma unroll
  for (int once = 0; once < 1; ++once) {
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
  // Few rows, or few workgroups of 16 of them: their waves share the width, where one workgroup of the others goes through it
  // alone (us of a call, few rows' way and tiles: f32, 512 rows, 1024 x 1024 26 and 39, 1024 rows 47 and 41; 2048 rows, 256 x 256
  // 11 and 14, 4096 21 and 16; bf16, 4096 rows, 1000 x 100 12 and 16, 8192 23 and 17; 512 rows, 1024 x 1024 13 and 16, 1024 rows
  // 25 and 16).
  if (slots <= GINEX_MAX_FEW_ROWS || few_groups(weights, route, slots) <= 512)
    return linear_few(x, weights, route, by_slot != 0, slots, epilogue, st);
  // Many rows of narrow layers: see resident_fits.
  if (resident_fits(weights, slots))
    return linear_resident(x, weights, route, by_slot != 0, slots, epilogue, st);
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const int64_t groups = route ? route->experts : 1;
    const auto tiles = [&](int height, int columns) { return (slots / height + groups) * ceil_div(weights->out, columns); };
    // Tiles as large as still leave every CU some (us of a call, tiles of 128, 64 and 32 rows x 128 columns: bf16, 16 000 rows, 256 x 256
    // 10.2, 10.2, 10.3; 40 000 18.5, 17.4, 20.8; 50 000, 1024 x 1024 180, 198, 260; 60 000, 256 x 256 21.1, 22.5, 27.6; f32, 3501 rows,
    // 1000 x 250 67, 50, 44; 250 x 1000 28, 24, 27; 177 000, 256 x 256 185, 179, 238; 50 000, 1024 x 1024 586, 617, 843).
    if (weights->out <= WAVE_COLUMNS) {
      if (tiles(128, 64) >= 1024) return launch<T, 2, 4, 1>(x, weights, route, by_slot, slots, epilogue, st);
      return launch<T, 1, 4, 1>(x, weights, route, by_slot, slots, epilogue, st);
    }
    if (tiles(128, 128) >= (sizeof(T) == 4 ? 3000 : 900)) return launch<T, 4, 2, 2>(x, weights, route, by_slot, slots, epilogue, st);
    if (tiles(64, 128) >= 400) return launch<T, 2, 2, 2>(x, weights, route, by_slot, slots, epilogue, st);
    return launch<T, 1, 2, 2>(x, weights, route, by_slot, slots, epilogue, st);
  });
}
