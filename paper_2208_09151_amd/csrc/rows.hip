// Rows to their experts' slots and back, and the gradients of both.
//
//   dispatch            out[slot(r,j)] = x[r]
//   combine             y[r]  = sum_j w(r,j) z[slot(r,j)]         (w = 1: dispatch's gradient)
//   combine, backward   dz[slot(r,j)] = w(r,j) dy[r],  dw(r,j) = <dy[r], z[slot(r,j)]>
//
// All of it is rows moved once, bound by HBM.  Work is laid out by row r, not by slot, so that x, y and dy
// are read or written once whatever the number of choices, and a row's sum stays in registers.  A slot and an
// offset are checked against the slots that exist before anything is computed from them: a routing that was
// not made by ginex_route cannot reach memory outside the arrays.
//
// Measured (bytes that have to move, over the time of a call among others, inputs of 4 to 10 calls in turn, so that none are
// in the caches of 256 MB; a plain copy reaches 6.2 TB/s):
//   rows x width, slots a row     dispatch        combine         its gradient
//   820 000 x 256 f32, 2          413 us 6.1      429 us 5.9      776 us 5.4 TB/s
//   820 000 x 256 bf16, 2         216    5.9      220    5.8      409    5.2
//   177 000 x 128 f32, 2           49    5.6       50    5.5       85    5.4   (all of it in the caches: 40, 41, 80)
//   41 017 x 250 f32, 8            87    4.3       71    5.2      170    4.1   (slots that share lines)
//   41 017 x 256 f32, 8            73    5.2       71    5.4      154    4.7
#include "train.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;

// The workgroup's place: workgroups go to the 8 dies in turn, and `together` gives a die an eighth of all beside each other.
__device__ __forceinline__ uint32_t place_of(bool together) {
  return together ? blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8 : blockIdx.x;
}

// Rows from offsets[experts] on are cleared, chunk by chunk, by all threads of the launch.
template <typename T>
__device__ __forceinline__ void clear_rest(RowsOf<T> out, Width width, Divisor cpr, const int64_t* __restrict__ end,
                                           int64_t slots, int64_t thread, int64_t threads) {
  constexpr int N = Chunk<T>::N;
  const float zero[N] = {};
  for (int64_t s = first_free_chunk(*end, slots, cpr.d) + thread; s < slots * cpr.d; s += threads) {
    const int64_t row = s / cpr.d;
    store_chunk(out.at(row), (int32_t)(s - row * cpr.d) * N, width, zero);
  }
}

// The slots of K of a row's choices from j0 on, -1 where there is none.
template <int K>
__device__ __forceinline__ void slots_of_row(const int32_t* __restrict__ slot, int64_t r, int32_t j0, int32_t top,
                                             int64_t slots, int32_t (&s)[K]) {
#pragma unroll
  for (int i = 0; i < K; ++i) s[i] = slot[r * top + (j0 + i < top ? j0 + i : j0)];
#pragma unroll
  for (int i = 0; i < K; ++i) s[i] = j0 + i < top && s[i] < slots ? s[i] : -1;
}

// A thread moves one chunk of row `first + t / cpr` to the row's slots, K of them at a time.  Chunks are numbered through
// all rows, so that no lane idles for a width that is no power of two.
template <typename T, int K, bool KEEP>
__global__ __launch_bounds__(THREADS) void k_dispatch(RowsOf<const T> x, RowsOf<T> out, const int32_t* __restrict__ slot,
                                                      const int64_t* __restrict__ end, int32_t top, int64_t first,
                                                      uint32_t chunks, Divisor cpr, Width width, int64_t slots,
                                                      bool clear, bool together) {
  constexpr int N = Chunk<T>::N;
  const uint32_t t = place_of(together) * THREADS + threadIdx.x;
  if (t < chunks) {
    const uint32_t row = cpr.of(t);
    const int32_t c = (int32_t)(t - row * cpr.d) * N;
    const int64_t r = first + row;
    const ChunkWords<T> v = load_words(x.at(r), c, width);
    for (int32_t j = 0; j < top; j += K) {
      int32_t s[K];
      slots_of_row<K>(slot, r, j, top, slots, s);
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (s[i] >= 0) store_words<KEEP>(out.at(s[i]), c, width, v);
    }
  }
  if (clear) clear_rest(out, width, cpr, end, slots, t, (int64_t)gridDim.x * THREADS);
}

// K slots of a row are read together; a choice without a slot reads slot 0 and counts for nothing.  (One after the other:
// 491 us instead of 433, 820 000 x 256 f32; eight together for eight choices: 29 -> 34 us, 41 017 x 256 bf16.)
template <typename T, bool WEIGHTED, int K>
__global__ __launch_bounds__(THREADS) void k_combine(RowsOf<const T> z, RowsOf<T> y, const int32_t* __restrict__ slot,
                                                     const float* __restrict__ weights, int32_t top, int64_t first,
                                                     uint32_t chunks, Divisor cpr, Width width, int64_t slots) {
  constexpr int N = Chunk<T>::N;
  const uint32_t t = blockIdx.x * THREADS + threadIdx.x;
  if (t >= chunks) return;
  const uint32_t row = cpr.of(t);
  const int32_t c = (int32_t)(t - row * cpr.d) * N;
  const int64_t r = first + row;
  float sum[N] = {};
  for (int32_t j = 0; j < top; j += K) {
    int32_t s[K];
    float v[K][N], w[K];
    slots_of_row<K>(slot, r, j, top, slots, s);
#pragma unroll
    for (int i = 0; i < K; ++i) {
      w[i] = WEIGHTED ? weights[r * top + (j + i < top ? j + i : j)] : 1.f;
      load_chunk(z.at(s[i] >= 0 ? s[i] : 0), c, width, v[i]);
    }
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float next = WEIGHTED ? fmaf(w[i], v[i][n], sum[n]) : sum[n] + v[i][n];
        sum[n] = s[i] >= 0 ? next : sum[n];
      }
  }
  store_chunk(y.at(r), c, width, sum);
}

// The sum of a group's lanes, in the last of them: lane by lane inside rows of 16 (DPP), then across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ float from_lane(float v) {
  return __uint_as_float(dpp_or_zero<CTRL, ROWS>(__float_as_uint(v)));
}
__device__ __forceinline__ float sum_to_last(float v, int32_t group) {
  if (group > 1) v += from_lane<0x111, 0xF>(v);     // row_shr:1
  if (group > 2) v += from_lane<0x112, 0xF>(v);
  if (group > 4) v += from_lane<0x114, 0xF>(v);
  if (group > 8) v += from_lane<0x118, 0xF>(v);
  if (group > 16) v += from_lane<0x142, 0xA>(v);    // row_bcast:15
  if (group > 32) v += from_lane<0x143, 0xC>(v);    // row_bcast:31
  return v;
}

// `group` lanes share a row: they walk its chunks and add up their products at the end.  (Two rows to a group: 774 -> 934
// us; one choice after the other: 780 -> 878; eight together: 152 -> 171.)  BLOCK > THREADS: the whole workgroup does.
template <typename T, int K, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_combine_backward(RowsOf<const T> dy, RowsOf<const T> z, RowsOf<T> dz,
                                                              const int32_t* __restrict__ slot,
                                                              const float* __restrict__ weights,
                                                              const int64_t* __restrict__ end,
                                                              float* __restrict__ dweights, int64_t first, int64_t rows,
                                                              int32_t top, int32_t shift, Divisor cpr, Width width,
                                                              int64_t slots, bool together) {
  constexpr int N = Chunk<T>::N;
  constexpr bool WHOLE = BLOCK > THREADS;
  const int64_t t = (int64_t)place_of(together) * BLOCK + threadIdx.x;
  const int32_t group = 1 << shift;
  const bool has_row = t >> shift < rows;
  const int64_t r = first + (has_row ? t >> shift : rows - 1);       // (all lanes take part in the sums)
  const int lane = (int)(t & (group - 1));
  for (int32_t j = 0; j < top; j += K) {
    int32_t s[K];
    float w[K], dot[K] = {};
    slots_of_row<K>(slot, r, j, top, slots, s);
#pragma unroll
    for (int i = 0; i < K; ++i) w[i] = weights[r * top + (j + i < top ? j + i : j)];
    for (int32_t c = lane * N; c < width.width; c += group * N) {
      float g[N], v[K][N];
      load_chunk(dy.at(r), c, width, g);
#pragma unroll
      for (int i = 0; i < K; ++i) load_chunk(z.at(s[i] >= 0 ? s[i] : 0), c, width, v[i]);
#pragma unroll
      for (int i = 0; i < K; ++i) {
        if (s[i] < 0 || !has_row) continue;
        float scaled[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
          dot[i] = fmaf(g[n], v[i][n], dot[i]);
          scaled[n] = w[i] * g[n];
        }
        store_chunk(dz.at(s[i]), c, width, scaled);
      }
    }
    if constexpr (WHOLE) {
      __shared__ float sums[K][BLOCK / WAVE];
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const float sum = sum_to_last(dot[i], WAVE);
        if (lane % WAVE == WAVE - 1) sums[i][lane / WAVE] = s[i] >= 0 ? sum : 0.f;
      }
      __syncthreads();
      if (has_row && lane < K && j + lane < top) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < BLOCK / WAVE; ++w) sum += sums[lane][w];
        dweights[r * top + j + lane] = sum;
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const float sum = sum_to_last(dot[i], group);
        if (has_row && lane == group - 1 && j + i < top) dweights[r * top + j + i] = s[i] >= 0 ? sum : 0.f;
      }
    }
  }
  if (first == 0) clear_rest(dz, width, cpr, end, slots, t, (int64_t)gridDim.x * BLOCK);
}

// How many of a row's choices are in flight together.
template <typename Go>
int32_t with_choices(int32_t top, Go go) {
  if (top == 1) return go(std::integral_constant<int, 1>{});
  if (top == 2) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}

// Whether every row begins and ends with a line of 128 bytes.  Where lines are shared by the slots of different rows,
// a dispatch stores through the caches, which put them together (41 017 x 8 slots of 1000 bytes: 123 -> 96 us); whole
// lines go past them (177 000 x 2 slots of 512 bytes: 45 -> 41).  And neighbouring rows, whose slots are neighbours as well,
// go to one die, as its caches are the dies' own (`together`; dispatch of 820 000 x 100 f16, 2 slots a row: 138 -> 107 us, 300 000
// x 333 f16 135 -> 121, 41 017 x 250 f32, 8: 95 and 96; combine's gradient 239 -> 218, 281 and 286, 170 and 168; where lines
// are whole, 820 000 x 256 f32, 2: 412 -> 472 and 778 -> 837).
bool whole_lines(const ginex_rows_t* r) {
  const int64_t bytes = element_bytes(r->type);
  return r->width * bytes % 128 == 0 && r->stride * bytes % 128 == 0 && reinterpret_cast<uintptr_t>(r->data) % 128 == 0;
}

unsigned blocks_of(int64_t threads, int64_t each, bool together) {
  const int64_t blocks = ceil_div(threads, each);
  return (unsigned)(together ? ceil_div(blocks, 8) * 8 : blocks);
}

// Rows of a launch: chunks are numbered in 31 bits.
int64_t rows_a_launch(int64_t chunks_a_row) { return (((int64_t)1 << 31) - THREADS) / chunks_a_row; }

int32_t check_slots(const char* what, const ginex_rows_t* r, const ginex_routing_t* route) {
  const int64_t slots = route->rows * route->top;
  if (r->rows != slots) return fail(GINEX_ERR_ARG, "%s has %lld rows, the routing %lld slots", what, (long long)r->rows, (long long)slots);
  return GINEX_OK;
}

int32_t check_sources(const char* what, const ginex_rows_t* r, const ginex_routing_t* route) {
  if (r->rows != route->rows)
    return fail(GINEX_ERR_ARG, "%s has %lld rows, the routing %lld", what, (long long)r->rows, (long long)route->rows);
  return GINEX_OK;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

extern "C" int32_t ginex_dispatch(const ginex_routing_t* route, const ginex_rows_t* x, const ginex_rows_t* out,
                                  void* stream) {
  if (int32_t rc = check_routing(route)) return rc;
  if (int32_t rc = check_rows("x", x, false)) return rc;
  if (int32_t rc = check_rows("out", out, true)) return rc;
  if (int32_t rc = check_same("x", x, "out", out)) return rc;
  if (int32_t rc = check_sources("x", x, route)) return rc;
  if (int32_t rc = check_slots("out", out, route)) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(x->type, [&](auto t) -> int32_t {
    return with_choices(route->top, [&](auto k) -> int32_t {
      using T = decltype(t);
      constexpr int K = decltype(k)::value;
      const int64_t cpr = ceil_div(x->width, Chunk<T>::N), step = rows_a_launch(cpr);
      for (int64_t r = 0; r < x->rows; r += step) {
        const int64_t chunks = (x->rows - r < step ? x->rows - r : step) * cpr;
        const bool shared = !whole_lines(out);
        const auto kernel = shared ? k_dispatch<T, K, true> : k_dispatch<T, K, false>;
        hipLaunchKernelGGL(kernel, dim3(blocks_of(chunks, THREADS, shared)), dim3(THREADS), 0, st,
                           read_rows<T>(x), rows_of<T>(out), route->slot, route->offsets + route->experts, route->top, r,
                           (uint32_t)chunks, Divisor((uint32_t)cpr), Width::of<T>(x->width), out->rows, r == 0, shared);
        GINEX_LAUNCH_CHECK();
      }
      return GINEX_OK;
    });
  });
}

extern "C" int32_t ginex_combine(const ginex_routing_t* route, const ginex_rows_t* z, const float* weights,
                                 const ginex_rows_t* y, void* stream) {
  if (int32_t rc = check_routing(route)) return rc;
  if (int32_t rc = check_rows("z", z, false)) return rc;
  if (int32_t rc = check_rows("y", y, true)) return rc;
  if (int32_t rc = check_same("z", z, "y", y)) return rc;
  if (int32_t rc = check_slots("z", z, route)) return rc;
  if (int32_t rc = check_sources("y", y, route)) return rc;
  if (reinterpret_cast<uintptr_t>(weights) % 4) return fail(GINEX_ERR_ARG, "weights: misaligned");
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(y->type, [&](auto t) -> int32_t {
    return with_choices(route->top, [&](auto k) -> int32_t {
      using T = decltype(t);
      constexpr int K = decltype(k)::value;
      const int64_t cpr = ceil_div(y->width, Chunk<T>::N), step = rows_a_launch(cpr);
      const auto kernel = weights ? k_combine<T, true, K> : k_combine<T, false, K>;
      for (int64_t r = 0; r < y->rows; r += step) {
        const int64_t chunks = (y->rows - r < step ? y->rows - r : step) * cpr;
        hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(chunks, THREADS)), dim3(THREADS), 0, st, read_rows<T>(z),
                           rows_of<T>(y), route->slot, weights, route->top, r, (uint32_t)chunks, Divisor((uint32_t)cpr),
                           Width::of<T>(y->width), z->rows);
        GINEX_LAUNCH_CHECK();
      }
      return GINEX_OK;
    });
  });
}

extern "C" int32_t ginex_combine_backward(const ginex_routing_t* route, const ginex_rows_t* dy, const ginex_rows_t* z,
                                          const float* weights, const ginex_rows_t* dz, float* dweights, void* stream) {
  if (int32_t rc = check_routing(route)) return rc;
  if (int32_t rc = check_rows("dy", dy, false)) return rc;
  if (int32_t rc = check_rows("z", z, false)) return rc;
  if (int32_t rc = check_rows("dz", dz, true)) return rc;
  if (int32_t rc = check_same("dy", dy, "z", z)) return rc;
  if (int32_t rc = check_same("dy", dy, "dz", dz)) return rc;
  if (int32_t rc = check_sources("dy", dy, route)) return rc;
  if (int32_t rc = check_slots("z", z, route)) return rc;
  if (int32_t rc = check_slots("dz", dz, route)) return rc;
  if (route->rows > 0 && (!weights || !dweights)) return fail(GINEX_ERR_ARG, "null weights or their gradient");
  if ((reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(dweights)) % 4)
    return fail(GINEX_ERR_ARG, "weights: misaligned");
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(dy->type, [&](auto t) -> int32_t {
    return with_choices(route->top, [&](auto k) -> int32_t {
      using T = decltype(t);
      constexpr int K = decltype(k)::value;
      const int64_t cpr = ceil_div(dy->width, Chunk<T>::N);
      // a workgroup to a row where rows are long and few (f32, 2 slots a row, a wave and a workgroup: 64 rows of 1024 5.9 and
      // 3.8 us, of 8192 27 and 5.3, 1024 rows of 8192 47 and 28; but 1024 rows of 512 4.8 and 8.7, of 1024 6.3 and 9.0)
      constexpr int WHOLE = 1024;
      const bool whole = cpr > WAVE && dy->rows <= cpr;
      int32_t shift = 0;
      while (1 << shift < (whole ? WHOLE : WAVE) && (whole || 1 << shift < cpr)) ++shift;
      const auto kernel = whole ? k_combine_backward<T, K, WHOLE> : k_combine_backward<T, K, THREADS>;
      const int threads = whole ? WHOLE : THREADS;
      const bool shared = !whole_lines(dz);
      // (a launch has fewer than 2^32 threads)
      const int64_t step = ((int64_t)1 << 31) >> shift;
      for (int64_t r = 0; r < dy->rows; r += step) {
        const int64_t rows = dy->rows - r < step ? dy->rows - r : step;
        hipLaunchKernelGGL(kernel, dim3(blocks_of(rows << shift, threads, shared)), dim3((unsigned)threads), 0, st,
                           read_rows<T>(dy), read_rows<T>(z), rows_of<T>(dz), route->slot, weights,
                           route->offsets + route->experts, dweights, r, rows, route->top, shift, Divisor((uint32_t)cpr),
                           Width::of<T>(dy->width), dz->rows, shared);
        GINEX_LAUNCH_CHECK();
      }
      return GINEX_OK;
    });
  });
}
