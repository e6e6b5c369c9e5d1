// Rows to their experts' slots and back, and the gradients of both.
//
//   dispatch            out[slot(r,j)] = x[r]
//   combine             y[r]  = sum_j w(r,j) z[slot(r,j)]         (w = 1: dispatch's gradient)
//   combine, backward   dz[slot(r,j)] = w(r,j) dy[r],  dw(r,j) = <dy[r], z[slot(r,j)]>
//
// All of it is rows moved once.  Work is laid out by row r, not by slot, so that x, y and dy are read or
// written once whatever the number of choices, and a row's sum stays in registers.  A slot is checked
// against the slots that exist before it is used: a routing that was not made by ginex_route cannot reach
// memory outside the arrays.
#include "train.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;
constexpr int CHOICES = 4;       // of a row, in flight together

// Rows from offsets[experts] on are cleared, chunk by chunk, by all threads of the launch.
template <typename T>
__device__ __forceinline__ void clear_rest(RowsOf<T> out, int32_t width, Divisor cpr, const int64_t* __restrict__ end,
                                           int64_t slots, int64_t thread, int64_t threads) {
  constexpr int N = Chunk<T>::N;
  const float zero[N] = {};
  int64_t kept = *end;
  kept = kept < 0 ? 0 : kept;
  for (int64_t s = kept * cpr.d + thread; s < slots * cpr.d; s += threads) {
    const int64_t row = s / cpr.d;
    const int32_t c = (int32_t)(s - row * cpr.d) * N;
    store_chunk(out.at(row, c), width - c, zero);
  }
}

// A thread moves one chunk of row `first + t / cpr` to the row's slots.
template <typename T>
__global__ __launch_bounds__(THREADS) void k_dispatch(RowsOf<T> x, RowsOf<T> out, const int32_t* __restrict__ slot,
                                                      const int64_t* __restrict__ end, int32_t top, int64_t first,
                                                      uint32_t chunks, Divisor cpr, int32_t width, int64_t slots,
                                                      bool clear) {
  constexpr int N = Chunk<T>::N;
  const uint32_t t = blockIdx.x * THREADS + threadIdx.x;
  if (t < chunks) {
    const uint32_t row = cpr.of(t);
    const int32_t c = (int32_t)(t - row * cpr.d) * N;
    const int64_t r = first + row;
    float v[N];
    load_chunk(x.at(r, c), width - c, v);
    for (int j = 0; j < top; ++j) {
      const int32_t s = slot[r * top + j];
      if (s >= 0 && s < slots) store_chunk(out.at(s, c), width - c, v);
    }
  }
  if (clear) clear_rest(out, width, cpr, end, slots, t, (int64_t)gridDim.x * THREADS);
}

template <typename T, bool WEIGHTED>
__global__ __launch_bounds__(THREADS) void k_combine(RowsOf<T> z, RowsOf<T> y, const int32_t* __restrict__ slot,
                                                     const float* __restrict__ weights, int32_t top, int64_t first,
                                                     uint32_t chunks, Divisor cpr, int32_t width, int64_t slots) {
  constexpr int N = Chunk<T>::N;
  const uint32_t t = blockIdx.x * THREADS + threadIdx.x;
  if (t >= chunks) return;
  const uint32_t row = cpr.of(t);
  const int32_t c = (int32_t)(t - row * cpr.d) * N;
  const int64_t r = first + row;
  float sum[N] = {};
  for (int j0 = 0; j0 < top; j0 += CHOICES) {
    float v[CHOICES][N], w[CHOICES];
#pragma unroll
    for (int i = 0; i < CHOICES; ++i) {
      const bool in = j0 + i < top;
      const int32_t s = in ? slot[r * top + j0 + i] : -1;
      const bool has = s >= 0 && s < slots;
      w[i] = has ? (WEIGHTED ? weights[r * top + j0 + i] : 1.f) : 0.f;
      if (has) {
        load_chunk(z.at(s, c), width - c, v[i]);
      } else {
#pragma unroll
        for (int n = 0; n < N; ++n) v[i][n] = 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < CHOICES; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) sum[n] = WEIGHTED ? fmaf(w[i], v[i][n], sum[n]) : sum[n] + v[i][n];
  }
  store_chunk(y.at(r, c), width - c, sum);
}

// GROUP lanes share a row: they walk its chunks and add up their products at the end.
template <typename T>
__global__ __launch_bounds__(THREADS) void k_combine_backward(RowsOf<T> dy, RowsOf<T> z, RowsOf<T> dz,
                                                              const int32_t* __restrict__ slot,
                                                              const float* __restrict__ weights,
                                                              const int64_t* __restrict__ end,
                                                              float* __restrict__ dweights, int64_t rows, int32_t top,
                                                              int32_t group, Divisor cpr, int32_t width, int64_t slots) {
  constexpr int N = Chunk<T>::N;
  const int64_t t = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  const int64_t r = t / group;
  const int lane = (int)(t & (group - 1));
  if (r < rows) {
    for (int j0 = 0; j0 < top; j0 += CHOICES) {
      int32_t s[CHOICES];
      float w[CHOICES], dot[CHOICES] = {};
#pragma unroll
      for (int i = 0; i < CHOICES; ++i) {
        s[i] = j0 + i < top ? slot[r * top + j0 + i] : -1;
        s[i] = s[i] < slots ? s[i] : -1;
        w[i] = s[i] >= 0 ? weights[r * top + j0 + i] : 0.f;
      }
      for (int32_t c = lane * N; c < width; c += group * N) {
        float g[N];
        load_chunk(dy.at(r, c), width - c, g);
#pragma unroll
        for (int i = 0; i < CHOICES; ++i) {
          if (s[i] < 0) continue;
          float v[N];
          load_chunk(z.at(s[i], c), width - c, v);
          float scaled[N];
#pragma unroll
          for (int n = 0; n < N; ++n) {
            dot[i] = fmaf(g[n], v[n], dot[i]);
            scaled[n] = w[i] * g[n];
          }
          store_chunk(dz.at(s[i], c), width - c, scaled);
        }
      }
      // (the lanes of a group are neighbours, and all of them are here: a group has one row)
#pragma unroll
      for (int i = 0; i < CHOICES; ++i) {
        for (int step = group / 2; step > 0; step /= 2) dot[i] += __shfl_xor(dot[i], step, WAVE);
        if (lane == 0 && j0 + i < top) dweights[r * top + j0 + i] = s[i] >= 0 ? dot[i] : 0.f;
      }
    }
  }
  clear_rest(dz, width, cpr, end, slots, t, (int64_t)gridDim.x * THREADS);
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
    using T = decltype(t);
    const int64_t cpr = ceil_div(x->width, Chunk<T>::N), step = rows_a_launch(cpr);
    for (int64_t r = 0; r < x->rows; r += step) {
      const int64_t chunks = (x->rows - r < step ? x->rows - r : step) * cpr;
      hipLaunchKernelGGL(k_dispatch<T>, dim3((unsigned)ceil_div(chunks, THREADS)), dim3(THREADS), 0, st, rows_of<T>(x),
                         rows_of<T>(out), route->slot, route->offsets + route->experts, route->top, r, (uint32_t)chunks,
                         Divisor((uint32_t)cpr), (int32_t)x->width, out->rows, r == 0);
      GINEX_LAUNCH_CHECK();
    }
    return GINEX_OK;
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
    using T = decltype(t);
    const int64_t cpr = ceil_div(y->width, Chunk<T>::N), step = rows_a_launch(cpr);
    const auto kernel = weights ? k_combine<T, true> : k_combine<T, false>;
    for (int64_t r = 0; r < y->rows; r += step) {
      const int64_t chunks = (y->rows - r < step ? y->rows - r : step) * cpr;
      hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(chunks, THREADS)), dim3(THREADS), 0, st, rows_of<T>(z),
                         rows_of<T>(y), route->slot, weights, route->top, r, (uint32_t)chunks, Divisor((uint32_t)cpr),
                         (int32_t)y->width, z->rows);
      GINEX_LAUNCH_CHECK();
    }
    return GINEX_OK;
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
  if (route->rows == 0) return GINEX_OK;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(dy->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const int64_t cpr = ceil_div(dy->width, Chunk<T>::N);
    int32_t group = 1;
    while (group < WAVE && group < cpr) group *= 2;
    const int64_t blocks = ceil_div(dy->rows * group, THREADS);
    hipLaunchKernelGGL(k_combine_backward<T>, dim3((unsigned)blocks), dim3(THREADS), 0, st, rows_of<T>(dy), rows_of<T>(z),
                       rows_of<T>(dz), route->slot, weights, route->offsets + route->experts, dweights, dy->rows,
                       route->top, group, Divisor((uint32_t)cpr), (int32_t)dy->width, dz->rows);
    GINEX_LAUNCH_CHECK();
    return GINEX_OK;
  });
}
