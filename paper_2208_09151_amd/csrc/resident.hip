// Linear layers whose weights find room in LDS: many rows through 64 to 256 columns at once.
//
// Such a layer is bound by HBM: a row of 256 numbers through 256 columns is 256 products a number.  A workgroup puts the weights
// of its columns into LDS once, in the order in which the matrix instructions take them (a wave reads 1 KB in a row, no bank
// twice), and goes through tiles of 128 rows.  A wave has 16 of them and all columns, so a row is read by one wave alone, from
// HBM into the registers of the matrix instructions, a segment ahead of the products, and no wave waits for another.  A layer
// per expert: the tiles of all experts are numbered, a workgroup has a range of them, and changes its weights where the expert
// changes.
#include "epilogue.hpp"

namespace ginex {
namespace {

constexpr int WAVES = 8, THREADS = WAVES * WAVE, HEIGHT = 16 * WAVES;
constexpr int MOST_LDS = 160 * 1024;

// NB x 64 columns, a chunk of columns and of width at least; rows are fetched S steps (64 bytes of every row) at a time.
template <typename T, int NB, int S>
__global__ __launch_bounds__(THREADS, 2) void k_resident(RowsOf<const T> x, int64_t rows, WeightsOf<T> weights, int32_t turned,
                                                         const int32_t* __restrict__ source,
                                                         const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                                         int32_t width, Width out, int32_t workers, int32_t blocks,
                                                         Epilogue epilogue) {
  constexpr int N = Chunk<T>::N, STEP = 4 * N, NT = 4 * NB;
  extern __shared__ words4 lds[];
  const int32_t steps = (width + STEP - 1) / STEP;
  float* const lds_bias = reinterpret_cast<float*>(lds + steps * NT * WAVE);
  // Workgroups go to the 8 dies in turn; those with the same rows follow each other on one die.
  const int32_t turn = blockIdx.x / 8, worker = turn / blocks * 8 + blockIdx.x % 8;
  const int32_t n0 = turn % blocks * NB * WAVE_COLUMNS;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), group = lane / 16;
  const Width along = {width, (int32_t)((width + N - 1) / N * N - width)};

  // A number that the compiler does not know: what depends on it is not computed in front of a loop and kept in registers.
  const auto anew = [](int32_t v) {
    asm volatile("" : "+v"(v));
    return v;
  };
  const auto put_weights = [&](int32_t expert) {
    const T* const w = weights.of(expert);
    const int32_t thread = anew(threadIdx.x);
    if (turned) {
#pragma unroll 4
      for (int32_t q = thread; q < steps * NT * WAVE; q += THREADS) {
        const int32_t l = q % WAVE, t = q / WAVE % NT, k = q / WAVE / NT;
        // operand row 4 g + i of product 4 b + j is column 64 b + 16 g + 4 j + i
        int32_t n = n0 + t / 4 * WAVE_COLUMNS + l % 16 / 4 * 16 + t % 4 * 4 + l % 4;
        n = n < out.width ? n : out.width - 1;
        lds[q] = load_words<true>(w + n * weights.stride, k * STEP + l / 16 * N, along).words;
      }
    } else {
#pragma unroll 2
      for (int32_t q = thread; q < steps * 4 * (NT * 4); q += THREADS) {
        const int32_t four = q % (NT * 4), k = q / (NT * 4);         // columns 4 four .. + 3, chunk k of the width
        const int32_t n = n0 + four * 4;
        typename Four<T>::Wide raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int32_t at = k * N + i;
          raw[i] = four_of<true>(w + (int64_t)(at < width ? at : width - 1) * weights.stride, n < out.width ? n : out.width - 1,
                           out.width);
          if (at >= width) raw[i] = (typename Four<T>::Wide)(T)0.f;
        }
        const int32_t t = four / 16 * 4 + four % 4, l = k % 4 * 16 + four % 16 / 4 * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ChunkWords<T> u;
#pragma unroll
          for (int i = 0; i < N; ++i) u.wide[i] = raw[i][j];
          lds[(k / 4 * NT + t) * WAVE + l + j] = u.words;
        }
      }
    }
    for (int32_t c = thread; c < NB * WAVE_COLUMNS; c += THREADS)
      lds_bias[c] = epilogue.bias && n0 + c < out.width
                        ? (float)static_cast<const T*>(epilogue.bias)[(int64_t)expert * out.width + n0 + c] : 0.f;
  };

  // Rows first + i stride + 0 .. 127 for i < count, up to end.
  const auto go = [&](int64_t first, int64_t stride, int32_t count, int64_t end) {
    const auto row_of = [&](int32_t i) { return first + (i < count ? i : count - 1) * stride + wave * 16 + lane % 16; };
    const auto source_of = [&](int32_t i) {
      int64_t r = row_of(i);
      r = r < end ? r : end - 1;
      return source ? (int64_t)source[r] : r;
    };
    ChunkWords<T> next[S];
    const auto fetch = [&](const T* row, int32_t k0) {
      const T* const from = row + k0 * STEP + group * N;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        if ((k0 + s + 1) * STEP <= width) next[s].wide = *reinterpret_cast<const typename Chunk<T>::At*>(from + s * STEP);
        else if (k0 + s < steps) next[s] = load_words<true>(row, anew((k0 + s) * STEP + group * N), along);
      }
    };
    int64_t r0 = source_of(0), r1 = source_of(1);
    bool there = r0 >= 0 && r0 < rows;
    const T* row = x.at(there ? r0 : 0);
    fetch(row, 0);
    for (int32_t i = 0; i < count; ++i) {
      float4v sum[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
        sum[t] = *reinterpret_cast<const float4v*>(lds_bias + t / 4 * WAVE_COLUMNS + group * LANE_COLUMNS + t % 4 * 4);
      const int64_t r = row_of(i);
      const bool mine = r < end;
      Columns<T> residual[NB];
      const int32_t c0 = n0 + group * LANE_COLUMNS;
      for (int32_t k0 = 0; k0 < steps; k0 += S) {
        ChunkWords<T> now[S];
#pragma unroll
        for (int s = 0; s < S; ++s) now[s].words = there ? next[s].words : words4{0, 0, 0, 0};
        if (k0 + S < steps) {
          fetch(row, k0 + S);
        } else {
          there = r1 >= 0 && r1 < rows;
          row = x.at(there ? r1 : 0);
          fetch(row, 0);
          r1 = source_of(i + 2);
          if (epilogue.residual) {
            const T* const and_ = static_cast<const T*>(epilogue.residual) + (mine ? r : end - 1) * epilogue.residual_stride;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              if (n0 + (b + 1) * WAVE_COLUMNS <= out.width) residual[b].load_whole(and_ + c0 + b * WAVE_COLUMNS);
              else residual[b].template load<true>(and_, anew(c0 + b * WAVE_COLUMNS), out);
            }
          }
        }
        // (the weights are read anew: they would be kept in registers through the loop, and spill)
        asm volatile("" ::: "memory");
        const words4* const at = lds + k0 * NT * WAVE + lane;
        const auto step = [&](int s) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            ChunkWords<T> w;
            w.words = at[(s * NT + t) * WAVE];
            sum[t] = product(w, now[s], sum[t]);
          }
        };
        if (k0 + S <= steps) {
#pragma unroll
          for (int s = 0; s < S; ++s) step(s);
        } else {
#pragma unroll
          for (int s = 0; s < S; ++s)
            if (k0 + s < steps) step(s);
        }
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float v[LANE_COLUMNS];
#pragma unroll
        for (int j = 0; j < LANE_COLUMNS; ++j) v[j] = sum[b * 4 + j / 4][j % 4];
        if (mine) finish<T>(epilogue, r, anew(c0) + b * WAVE_COLUMNS, n0 + (b + 1) * WAVE_COLUMNS <= out.width, out, v, residual[b]);
      }
    }
  };

  // one layer: every so many tiles are this workgroup's; a layer per expert: a range of them
  const uint32_t tiles = offsets ? count_tiles(offsets, experts, slots, HEIGHT) : (uint32_t)((slots + HEIGHT - 1) / HEIGHT);
  uint32_t t = offsets ? (uint32_t)((uint64_t)tiles * worker / workers) : worker;
  const uint32_t upto = offsets ? (uint32_t)((uint64_t)tiles * (worker + 1) / workers) : tiles;
  while (t < upto) {
    TileRows tile = {0, (int64_t)t * HEIGHT, slots};
    int64_t stride = (int64_t)workers * HEIGHT;
    int32_t count = (int32_t)((tiles - t + workers - 1) / workers);
    if (offsets) {
      if (!find_tile(offsets, experts, slots, t, HEIGHT, tile)) return;
      const uint32_t left = (uint32_t)((tile.end - tile.first + HEIGHT - 1) / HEIGHT);
      count = (int32_t)(left < upto - t ? left : upto - t);
      stride = HEIGHT;
    }
    t = offsets ? t + count : upto;
    if (tile.expert == experts) {         // slots without an expert
      for (int32_t i = 0; i < count; ++i) {
        const int64_t r = tile.first + (int64_t)i * HEIGHT + wave * 16 + lane % 16;
        if (r >= tile.end) continue;
#pragma unroll 1
        for (int b = 0; b < NB; ++b) clear_columns<T>(epilogue, r, anew(n0 + b * WAVE_COLUMNS + group * LANE_COLUMNS), out);
      }
      continue;
    }
    __syncthreads();                      // (nobody reads the weights before any more)
    put_weights(tile.expert);
    __syncthreads();
    go(tile.first, stride, count, tile.end);
  }
}

struct Fit {
  int32_t nb, blocks, steps;
  int64_t lds;
};
Fit fit_of(int64_t width, int64_t out, int bytes) {
  Fit f;
  const int64_t steps = ceil_div(width * bytes, 64), groups = ceil_div(out, WAVE_COLUMNS);
  int64_t most = (MOST_LDS - 1024) / (steps * 4 * 1024);
  const int64_t columns = bytes == 4 ? 2 : 4;         // sums and rows of more would not find room in the registers
  most = most < columns ? most : columns;
  f.steps = (int32_t)steps;
  f.blocks = most > 0 ? (int32_t)ceil_div(groups, most) : 1 << 30;
  f.nb = (int32_t)ceil_div(groups, f.blocks);
  f.lds = steps * f.nb * 4 * 1024 + f.nb * WAVE_COLUMNS * sizeof(float);
  return f;
}

}  // namespace

bool resident_fits(const ginex_weights_t* w, int64_t slots, bool routed) {
  const Fit f = fit_of(w->width, w->out, element_bytes(w->type));
  const int chunk = 16 / element_bytes(w->type);
  return w->width >= chunk && w->out >= chunk && f.blocks <= 2 && slots >= 32 * HEIGHT;
}

int32_t linear_resident(const ginex_rows_t* x, const ginex_weights_t* w, const ginex_routing_t* route, bool by_slot,
                        int64_t slots, const Epilogue& epilogue, hipStream_t st) {
  const Fit f = fit_of(w->width, w->out, element_bytes(x->type));
  const int32_t workers = 256 * (f.lds <= MOST_LDS / 2 ? 2 : 1);
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const auto with_segment = [&](auto nb, auto s) -> int32_t {
      constexpr int NB = decltype(nb)::value, S = decltype(s)::value;
      hipLaunchKernelGGL((k_resident<T, NB, S>), dim3((unsigned)(workers * f.blocks)), dim3(THREADS), (unsigned)f.lds, st,
                         read_rows<T>(x), x->rows, weights_of<T>(w), w->turned, route && !by_slot ? route->source : nullptr,
                         route ? route->offsets : nullptr, w->experts, slots, (int32_t)w->width, Width::of<T>(w->out), workers,
                         f.blocks, epilogue);
      GINEX_LAUNCH_CHECK();
      return GINEX_OK;
    };
    const auto with_columns = [&](auto nb) -> int32_t {
      if (f.steps <= 2) return with_segment(nb, std::integral_constant<int, 2>{});
      if (decltype(nb)::value == 4 || f.steps <= 4) return with_segment(nb, std::integral_constant<int, 4>{});
      return with_segment(nb, std::integral_constant<int, decltype(nb)::value == 4 ? 4 : 8>{});
    };
    if (f.nb == 1) return with_columns(std::integral_constant<int, 1>{});
    if (f.nb == 2) return with_columns(std::integral_constant<int, 2>{});
    if constexpr (sizeof(T) == 2) {
      if (f.nb == 3) return with_columns(std::integral_constant<int, 3>{});
      return with_columns(std::integral_constant<int, 4>{});
    }
    return fail(GINEX_ERR_ARG, "linear: %d columns of 64", f.nb);
  });
}

}  // namespace ginex
