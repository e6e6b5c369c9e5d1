// Linear layers whose weights find room in LDS: many rows through 64 to 256 columns at once.
//
// Such a layer is bound by HBM: a row of 256 numbers through 256 columns is 256 products a number.  A workgroup puts the weights
// of its columns into LDS once, in the order in which the matrix instructions take them (a wave reads 1 KB in a row, no bank
// twice), and goes through tiles of rows, which come from HBM into the registers of the matrix instructions, a segment ahead of
// the products; no wave waits for another.  In 16 bits a wave has 16 rows and all of the workgroup's columns, so that one wave alone
// reads a row of up to 256 columns.  Of f32's three parts LDS has room for 64 columns of 256 numbers: four workgroups, which follow
// each other on one die, read a row for 256 columns, and each cuts it into its parts.  A layer per expert: the tiles of all experts
// are numbered, a workgroup has a range of them, and changes its weights where the expert changes.
//
// 177 000 x 256 -> 256 bf16 with gelu and residual 80 us: 52 for the rows, 10 for the residual and 18 for gelu on the vector unit, which
// the loads do not hide (relu: 2).  The 52 are a start of some 12 us and rounds of 32 768 rows of 7 each, the last as long as the
// others (196 608 rows 52.5, one more 58.8; 820 000 194, 4.3 TB/s).  820 000 x 256 -> 256 f32 700 us, 2.4 TB/s and 920 TFLOP/s of bf16
// products: the matrix cores, and the vector unit that cuts every row four times.
#include "epilogue.hpp"
#include "parts.hpp"

namespace ginex {
namespace {

constexpr int WAVES = 8, THREADS = WAVES * WAVE;
constexpr int MOST_LDS = 160 * 1024;

// NB x 64 columns, a chunk of columns and of width at least; rows are fetched S units ahead, MT x 16 of
// them to a wave.  A wave waits for the oldest of its loads alone, so none of them, and no store, stands behind a branch
// that depends on data or sizes: the compiler would have to wait for all.  RES: there is a residual.
template <typename T, int MT, int NB, int S, bool RES>
__global__ __launch_bounds__(THREADS, 2) void k_resident(RowsOf<const T> x, int64_t rows, WeightsOf<T> weights, int32_t turned,
                                                         const int32_t* __restrict__ source,
                                                         const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                                         int32_t width, Width out, int32_t workers, int32_t blocks,
                                                         int32_t across, Epilogue epilogue) {
  using O = Operand<T>;
  using K = typename O::Kind;
  constexpr int N = Chunk<T>::N, UNIT = 8 * N, NT = 4 * NB, PARTS = O::PARTS;
  extern __shared__ words4 lds[];
  const int32_t units = (width + UNIT - 1) / UNIT, all = NT * across, height = 16 * MT * WAVES / across;
  float* const lds_bias = reinterpret_cast<float*>(lds + units * all * PARTS * WAVE);
  // Workgroups go to the 8 dies in turn; those with the same rows follow each other on one die.
  const int32_t turn = blockIdx.x / 8, worker = turn / blocks * 8 + blockIdx.x % 8;
  const int32_t block0 = turn % blocks * across * NB * WAVE_COLUMNS;
  const int lane = lane_id(), group = lane / 16;
  // a wave's place: its columns, and among the waves that have those
  const int wave_of = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), wave = wave_of / across, part = wave_of % across;
  const int32_t n0 = block0 + part * NB * WAVE_COLUMNS;
  const Width along = {width, (int32_t)((width + N - 1) / N * N - width)};

  // A number that the compiler does not know: what depends on it is not computed in front of a loop and kept in registers.
  const auto anew = [](int32_t v) {
    asm volatile("" : "+v"(v));
    return v;
  };
  // Weights in the order in which the matrix instructions take them: operand row 4 g + i of product 4 b + j is column
  // 64 b + 16 g + 4 j + i.
  const auto put_weights = [&](int32_t expert) {
    const T* const w = weights.of(expert);
    const int32_t thread = anew(threadIdx.x);
    if (turned) {
#pragma unroll 4
      for (int32_t q = thread; q < units * all * WAVE; q += THREADS) {
        const int32_t l = q % WAVE, t = q / WAVE % all, k = q / WAVE / all;
        int32_t n = block0 + t / 4 * WAVE_COLUMNS + l % 16 / 4 * 16 + t % 4 * 4 + l % 4;
        n = n < out.width ? n : out.width - 1;
        ChunkWords<T> v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = load_words<true>(w + n * weights.stride, k * UNIT + (l / 16 * 2 + h) * N, along);
        ChunkWords<K> parts[PARTS];
        parts_of(v, parts);
#pragma unroll
        for (int z = 0; z < PARTS; ++z) lds[((k * all + t) * PARTS + z) * WAVE + l] = parts[z].words;
      }
    } else {
#pragma unroll 2
      for (int32_t q = thread; q < units * UNIT / 8 * (all * 4); q += THREADS) {
        const int32_t four = q % (all * 4), eight = q / (all * 4);     // columns 4 four .. + 3, numbers 8 eight .. + 7 of the width
        const int32_t n = block0 + four * 4;
        typename Four<T>::Wide raw[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int32_t at = eight * 8 + i;
          raw[i] = four_of<true>(w + (int64_t)(at < width ? at : width - 1) * weights.stride,
                                 n < out.width ? n : out.width - 1, out.width);
          if (at >= width) raw[i] = (typename Four<T>::Wide)(T)0.f;
        }
        // f32: a lane's unit; 16 bits: half of it
        constexpr int EIGHTS = UNIT / 8, HALVES = EIGHTS / 4;
        const int32_t t = four / 16 * 4 + four % 4, k = eight / EIGHTS, l = eight % EIGHTS / HALVES * 16 + four % 16 / 4 * 4;
        words4* const to = lds + (k * all + t) * PARTS * WAVE + l;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ChunkWords<T> v[2];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i / N].wide[i % N] = raw[i][j];
          if constexpr (sizeof(T) == 4) {
            ChunkWords<K> parts[PARTS];
            parts_of(v, parts);
#pragma unroll
            for (int z = 0; z < PARTS; ++z) to[z * WAVE + j] = parts[z].words;
          } else {
            to[eight % HALVES * WAVE + j] = v[0].words;
          }
        }
      }
    }
    for (int32_t c = thread; c < across * NB * WAVE_COLUMNS; c += THREADS)
      lds_bias[c] = epilogue.bias && block0 + c < out.width
                        ? (float)static_cast<const T*>(epilogue.bias)[(int64_t)expert * out.width + block0 + c] : 0.f;
  };

  // 16 MT rows a wave, `apart` rows from wave to wave and `stride` from tile to tile, `count` tiles up to row `end`.
  const auto go = [&](int32_t expert, int64_t first, int64_t apart, int64_t stride, int32_t count, int64_t end) {
    const auto row_of = [&](int32_t i, int m) {
      return first + (i < count ? i : count - 1) * stride + wave * apart + m * 16 + lane % 16;
    };
    int32_t from[MT];                 // where the rows of the tile that is fetched next come from
    const T* row[MT];                 // and of the one that is fetched now
    bool there[MT];
    ChunkWords<T> next[S][MT][2];
    const auto find = [&](int32_t i) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        int64_t r = row_of(i, m);
        r = r < end ? r : end - 1;
        from[m] = source ? source[r] : (int32_t)r;
      }
    };
    const auto take = [&]() {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        there[m] = (uint32_t)from[m] < (uint64_t)rows;
        row[m] = x.at(there[m] ? from[m] : 0);
      }
    };
    const auto fetch = [&](int32_t k, int s) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int32_t c = (k < units ? k : units - 1) * UNIT + (group * 2 + h) * N;
          next[s][m][h].wide = *reinterpret_cast<const typename Chunk<T>::At*>(row[m] + (c < width - N ? c : width - N));
        }
    };
    find(0);
    take();
    find(1);
#pragma unroll
    for (int s = 0; s < S; ++s) fetch(s, s);
    __syncthreads();                  // (nobody reads the weights before any more)
    put_weights(expert);
    __syncthreads();
    for (int32_t i = 0; i < count; ++i) {
      float4v sum[MT][NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        sum[0][t] = *reinterpret_cast<const float4v*>(lds_bias + (part * NB + t / 4) * WAVE_COLUMNS + group * LANE_COLUMNS + t % 4 * 4);
#pragma unroll
        for (int m = 1; m < MT; ++m) sum[m][t] = sum[0][t];
      }
      const int32_t c0 = n0 + group * LANE_COLUMNS;
      Columns<T> residual[MT][NB];
      for (int32_t k0 = 0; k0 < units; k0 += S) {
        // A unit's rows are fetched for the next segment, or the next tile, as soon as its products are under way.
        const bool last = k0 + S >= units;
        bool is[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) is[m] = there[m];
        if (last) {
          take();
          find(i + 2);
        }
        if (RES && k0 == 0) {
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const int64_t r = row_of(i, m);
            const T* const and_ = static_cast<const T*>(epilogue.residual) + (r < end ? r : end - 1) * epilogue.residual_stride;
#pragma unroll
            for (int b = 0; b < NB; ++b) residual[m][b].read(and_, c0 + b * WAVE_COLUMNS, out);
          }
        }
        // (the weights are read anew: they would be kept in registers through the loop, and spill)
        asm volatile("" ::: "memory");
        const words4* at = lds + (k0 * all + part * NT) * PARTS * WAVE + lane;
#pragma unroll
        for (int s = 0; s < S; ++s) {
          if (k0 + s < units) {
            ChunkWords<K> now[MT][PARTS];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              if (source) {
#pragma unroll
                for (int h = 0; h < 2; ++h) next[s][m][h].words = is[m] ? next[s][m][h].words : words4{0, 0, 0, 0};
              }
              if ((k0 + s + 1) * UNIT > width) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                  next[s][m][h] = placed<T>(next[s][m][h], anew((k0 + s) * UNIT + (group * 2 + h) * N), along);
              }
              parts_of(next[s][m], now[m]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              ChunkWords<K> w[PARTS];
#pragma unroll
              for (int z = 0; z < PARTS; ++z) w[z].words = at[(t * PARTS + z) * WAVE];
              products_of<K, MT>(w, now, &sum[0][t], NT);
            }
          }
          at += all * PARTS * WAVE;
          fetch((last ? 0 : k0 + S) + s, s);
        }
      }
      if constexpr (sizeof(T) == 4) {
        if (any_none<MT * NT>(&sum[0][0])) {
          const T* const w = weights.of(expert);
#pragma unroll 1
          for (int m = 0; m < MT; ++m) {
            int64_t r = row_of(i, m);
            r = r < end ? r : end - 1;
            r = source ? (int64_t)source[r] : r;
            const bool is = r >= 0 && r < rows;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              int32_t n = anew(n0 + t / 4 * WAVE_COLUMNS + lane % 16 / 4 * 16 + t % 4 * 4 + lane % 4);
              n = n < out.width ? n : out.width - 1;
              const float4v start =
                  *reinterpret_cast<const float4v*>(lds_bias + (part * NB + t / 4) * WAVE_COLUMNS + group * LANE_COLUMNS + t % 4 * 4);
              const float4v again = sums_again(x.at(is ? r : 0), is, w + (turned ? n * weights.stride : n),
                                               turned ? 1 : weights.stride, width, start);
#pragma unroll
              for (int j = 0; j < MT; ++j)
                if (j == m) sum[j][t] = with_again(sum[j][t], again);
            }
          }
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int64_t r = row_of(i, m);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          float v[LANE_COLUMNS];
#pragma unroll
          for (int j = 0; j < LANE_COLUMNS; ++j) v[j] = sum[m][b * 4 + j / 4][j % 4];
          const int32_t c = anew(c0) + b * WAVE_COLUMNS;
          finish_values<T>(epilogue, r, r < end, c, out, v);
          if (RES) {
            if (n0 + (b + 1) * WAVE_COLUMNS > out.width) residual[m][b].place(c, out);
#pragma unroll
            for (int j = 0; j < LANE_COLUMNS; ++j) v[j] += residual[m][b].of(j);
          }
          store_columns_masked<T>(epilogue, r, r < end, c, out, v);
        }
      }
    }
  };

  // one layer: every so many tiles are this workgroup's; a layer per expert: a range of them
  const uint32_t tiles = offsets ? count_tiles(offsets, experts, slots, height) : (uint32_t)((slots + height - 1) / height);
  uint32_t t = offsets ? (uint32_t)((uint64_t)tiles * worker / workers) : worker;
  const uint32_t upto = offsets ? (uint32_t)((uint64_t)tiles * (worker + 1) / workers) : tiles;
  while (t < upto) {
    // (neighbouring waves' rows on different CUs: the last ones are shared by all)
    TileRows tile = {0, (int64_t)worker * (16 * MT), slots};
    int64_t apart = (int64_t)workers * (16 * MT), stride = (int64_t)workers * height;
    int32_t count = (int32_t)((slots + stride - 1) / stride);
    if (offsets) {
      if (!find_tile(offsets, experts, slots, t, height, tile)) return;
      const uint32_t left = (uint32_t)((tile.end - tile.first + height - 1) / height);
      count = (int32_t)(left < upto - t ? left : upto - t);
      apart = 16 * MT;
      stride = height;
      t += count;
    }
    if (tile.expert == experts) {         // slots without an expert
      const int64_t until = tile.first + (int64_t)count * height < tile.end ? tile.first + (int64_t)count * height : tile.end;
      for (int64_t r = tile.first + wave * 16 + lane % 16; r < until; r += 16 * WAVES / across) {
#pragma unroll 1
        for (int b = 0; b < NB; ++b) clear_columns<T>(epilogue, r, anew(n0 + b * WAVE_COLUMNS + group * LANE_COLUMNS), out);
      }
    } else {
      go(tile.expert, tile.first, apart, stride, count, tile.end);
    }
    if (!offsets) return;
  }
}

struct Fit {
  int32_t nb, across, blocks, units;
  int64_t lds;
};
Fit fit_of(int64_t width, int64_t out, int bytes) {
  Fit f;
  const int64_t parts = bytes == 4 ? Operand<float>::PARTS : Operand<bf16>::PARTS;
  const int64_t units = ceil_div(width * bytes, 128), groups = ceil_div(out, WAVE_COLUMNS);
  // columns of 64 of a workgroup: what LDS has room for, 4 at most; of a wave: what its registers have
  int64_t most = (MOST_LDS - 1024) / (units * parts * 4 * 1024);
  most = most < 4 ? most : 4;
  f.units = (int32_t)units;
  f.blocks = most > 0 ? (int32_t)ceil_div(groups, most) : 1 << 30;
  const int32_t columns = (int32_t)ceil_div(groups, f.blocks);
  f.across = bytes == 4 ? (columns < 3 ? columns : 4) : 1;
  f.nb = bytes == 4 ? 1 : (columns < 3 ? columns : 4);
  f.lds = units * parts * f.across * f.nb * 4 * 1024 + f.across * f.nb * WAVE_COLUMNS * sizeof(float);
  if (f.lds > MOST_LDS) f.blocks = 1 << 30;
  return f;
}

}  // namespace

// Where the rows are many enough to pay for the weights' way into LDS (us of a call, this and tiles: bf16, 256 x 256, 60 000 rows
// 25.5 and 21.1, 100 000 42.5 and 39.6, 177 000 56.5 and 61.6, 820 000 200 and 268; 8 experts, 152 000 slots, 256 x 128 41 and 34; 32
// experts, 600 000 slots, 128 x 128 81 and 94; f16, 300 000 x 100, 47 out 30 and 39; f32, 128 x 128, 60 000 rows 28.6 and 25.0, 152 000
// slots of 8 experts, 256 x 128 88 and 100; 820 000, 256 x 256 710 and 739), and with each expert's anew: bf16 and f32, 162 000 slots,
// 256 x 128, of 256 experts 65 and 54, 129 and 137, of 1024 117 and 72, 232 and 151; 600 000, 128 x 128, of 256 99 and 117, 238 and 263.
bool resident_fits(const ginex_weights_t* w, int64_t slots) {
  const int bytes = element_bytes(w->type);
  const Fit f = fit_of(w->width, w->out, bytes);
  return w->width >= 16 / bytes && w->out >= 16 / bytes && f.blocks <= (bytes == 4 ? 4 : 2) &&
         slots >= (bytes == 4 ? (1 << 17) + 512 * (int64_t)w->experts : 160000 + 400 * (int64_t)w->experts);
}

int32_t linear_resident(const ginex_rows_t* x, const ginex_weights_t* w, const ginex_routing_t* route, bool by_slot,
                        int64_t slots, const Epilogue& epilogue, hipStream_t st) {
  Fit f = fit_of(w->width, w->out, element_bytes(x->type));
  // as many workgroups as are on the GPU at a time, those with the same rows together
  int32_t workers = 256 * (f.lds <= MOST_LDS / 2 ? 2 : 1) / f.blocks;
  workers = (workers + 7) / 8 * 8;
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const auto with = [&](auto nb, auto s) -> int32_t {
      constexpr int MT = sizeof(T) == 4 ? 2 : 1, NB = decltype(nb)::value, S = decltype(s)::value;
      const auto kernel = epilogue.residual ? k_resident<T, MT, NB, S, true> : k_resident<T, MT, NB, S, false>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(workers * f.blocks)), dim3(THREADS), (unsigned)f.lds, st,
                         read_rows<T>(x), x->rows, weights_of<T>(w), w->turned, route && !by_slot ? route->source : nullptr,
                         route ? route->offsets : nullptr, w->experts, slots, (int32_t)w->width, Width::of<T>(w->out), workers,
                         f.blocks, f.across, epilogue);
      GINEX_LAUNCH_CHECK();
      return GINEX_OK;
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    const auto with_columns = [&](auto nb) -> int32_t {
      return f.units == 1 ? with(nb, one) : f.units <= 3 ? with(nb, two) : with(nb, four);
    };
    if constexpr (sizeof(T) == 4) return with_columns(one);
    else return f.nb == 1 ? with_columns(one) : f.nb == 2 ? with_columns(two) : with_columns(four);
  });
}

}  // namespace ginex
