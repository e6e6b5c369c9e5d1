// Layer norm and its gradients:
//
//   y = (x - mean) rstd weight + bias,   rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   dx = rstd (a - mean(a) - unit mean(a unit)),   a = dy weight,  unit = (x - mean) rstd
//   dweight = sum over the rows of dy unit,  dbias = sum over the rows of dy
//
// Bound by HBM: a row is read once into registers, by as many lanes as it has chunks of 16 bytes (a power of two, up to a
// wave with 4 chunks a lane, then a workgroup), and only rows beyond 16 KB are read again.  A mean in f32 is off by up to half
// its last place, which counts where rows lie far from 0: the mean of what is left after it is taken away is added up along
// with the squares, and taken away as well, in the backward pass too.  There a lane keeps the sums of its columns over the
// rows of its workgroup in registers; each workgroup leaves one part, and a second launch adds the parts up in their order.
//
// 820 000 x 256 f32: 334 us (5.0 TB/s) and 479 (5.3) with 4.6 for the parts; 3501 x 333 bf16 5.2 and 7.8 + 5.1, latency.
#include "joins.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / WAVE;

// The sum over `group` lanes (a power of two) in all of them.
__device__ __forceinline__ float sum_of_group(float v, int32_t group) {
  if (group > 1) v += __uint_as_float(dpp_or_zero<0xB1, 0xF>(__float_as_uint(v)));      // quad_perm [1, 0, 3, 2]
  if (group > 2) v += __uint_as_float(dpp_or_zero<0x4E, 0xF>(__float_as_uint(v)));      // quad_perm [2, 3, 0, 1]
  if (group > 4) v += __uint_as_float(dpp_or_zero<0x141, 0xF>(__float_as_uint(v)));     // row_half_mirror
  if (group > 8) v += __uint_as_float(dpp_or_zero<0x140, 0xF>(__float_as_uint(v)));     // row_mirror
  if (group > 16) v += __shfl_xor(v, 16, WAVE);
  if (group > 32) v += __shfl_xor(v, 32, WAVE);
  return v;
}

// The sums of K numbers over the lanes of a row: a group of lanes, or (WHOLE) the workgroup, whose waves meet in `room`,
// one of two that take turns so that no wave writes what another has still to read.
template <int K, bool WHOLE>
__device__ __forceinline__ void sums_of_row(float (&v)[K], int32_t group, float (*room)[WAVES][4], int turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = sum_of_group(v[k], WHOLE ? WAVE : group);
  if (!WHOLE) return;
  float(*const at)[4] = room[turn];
  if (lane_id() == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) at[threadIdx.x / WAVE][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v[k] += at[w][k];
  }
}

__device__ __forceinline__ float rstd_of(float variance, float eps) {
  return 1.f / sqrtf((variance < 0.f ? 0.f : variance) + eps);       // (a NaN stays one)
}

template <typename T>
__device__ __forceinline__ void load_vector(const T* v, int32_t c, Width width, float none, float (&to)[Chunk<T>::N]) {
  if (v) {
    load_chunk(v, c, width, to);
    return;
  }
#pragma unroll
  for (int i = 0; i < Chunk<T>::N; ++i) to[i] = none;
}

// K chunks a lane, in registers; a group of lanes or the workgroup to a row.
template <typename T, int K, bool WHOLE>
__global__ __launch_bounds__(THREADS) void k_norm(RowsOf<const T> x, RowsOf<T> y, const T* __restrict__ weight,
                                                  const T* __restrict__ bias, int64_t rows, int32_t shift, Width width,
                                                  float per_width, float eps, float* __restrict__ stats) {
  constexpr int N = Chunk<T>::N;
  __shared__ float room[2][WAVES][4];
  const int32_t group = WHOLE ? THREADS : 1 << shift;
  const int64_t at = WHOLE ? (int64_t)blockIdx.x : ((int64_t)blockIdx.x * THREADS + threadIdx.x) >> shift;
  const int64_t r = at < rows ? at : rows - 1;        // (all lanes take part in the sums)
  const int32_t lane = threadIdx.x & (group - 1);
  float v[K][N];
#pragma unroll
  for (int k = 0; k < K; ++k) load_chunk(x.at(r), (lane + k * group) * N, width, v[k]);
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) sum[0] += v[k][i];
  float one[1] = {sum[0]};
  sums_of_row<1, WHOLE>(one, group, room, 0);
  const float mean = one[0] * per_width;
  sum[0] = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[k][i] = (lane + k * group) * N + i < width.width ? v[k][i] - mean : 0.f;
      sum[0] += v[k][i];
      sum[1] = fmaf(v[k][i], v[k][i], sum[1]);
    }
  sums_of_row<2, WHOLE>(sum, group, room, 1);
  const float rest = sum[0] * per_width, rstd = rstd_of(fmaf(-rest, rest, sum[1] * per_width), eps);
  if (at >= rows) return;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int32_t c = (lane + k * group) * N;
    if (c >= width.width) continue;
    float w[N], b[N];
    load_vector(weight, c, width, 1.f, w);
    load_vector(bias, c, width, 0.f, b);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = fmaf((v[k][i] - rest) * rstd, w[i], b[i]);
    store_chunk(y.at(r), c, width, w);
  }
  if (stats && lane == 0) *reinterpret_cast<float2*>(stats + 2 * r) = make_float2(mean + rest, rstd);
}

// Rows of any width, read again from the caches.
template <typename T>
__global__ __launch_bounds__(THREADS) void k_norm_long(RowsOf<const T> x, RowsOf<T> y, const T* __restrict__ weight,
                                                       const T* __restrict__ bias, Width width, float per_width, float eps,
                                                       float* __restrict__ stats) {
  constexpr int N = Chunk<T>::N, STEP = THREADS * N;
  __shared__ float room[2][WAVES][4];
  const int64_t r = blockIdx.x;
  const T* const row = x.at(r);
  float one[1] = {0.f};
  for (int32_t c = threadIdx.x * N; c < width.width; c += STEP) {
    float v[N];
    load_chunk(row, c, width, v);
#pragma unroll
    for (int i = 0; i < N; ++i) one[0] += v[i];
  }
  sums_of_row<1, true>(one, THREADS, room, 0);
  const float mean = one[0] * per_width;
  float sum[2] = {0.f, 0.f};
  for (int32_t c = threadIdx.x * N; c < width.width; c += STEP) {
    float v[N];
    load_chunk(row, c, width, v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = c + i < width.width ? v[i] - mean : 0.f;
      sum[0] += d;
      sum[1] = fmaf(d, d, sum[1]);
    }
  }
  sums_of_row<2, true>(sum, THREADS, room, 1);
  const float rest = sum[0] * per_width, rstd = rstd_of(fmaf(-rest, rest, sum[1] * per_width), eps);
  for (int32_t c = threadIdx.x * N; c < width.width; c += STEP) {
    float v[N], w[N], b[N];
    load_chunk(row, c, width, v);
    load_vector(weight, c, width, 1.f, w);
    load_vector(bias, c, width, 0.f, b);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = fmaf(((v[i] - mean) - rest) * rstd, w[i], b[i]);
    store_chunk(y.at(r), c, width, w);
  }
  if (stats && threadIdx.x == 0) *reinterpret_cast<float2*>(stats + 2 * r) = make_float2(mean + rest, rstd);
}

// part NULL: dx alone.
template <typename T, int K, bool WHOLE>
__global__ __launch_bounds__(THREADS) void k_norm_backward(RowsOf<const T> dy, RowsOf<const T> x,
                                                           const float* __restrict__ stats, const T* __restrict__ weight,
                                                           RowsOf<T> dx, int64_t rows, int32_t shift, Width width,
                                                           float per_width, float* __restrict__ part) {
  constexpr int N = Chunk<T>::N;
  __shared__ float room[2][WAVES][4];
  __shared__ float sums[THREADS][N + 1];
  const int32_t group = WHOLE ? THREADS : 1 << shift;
  const int32_t lane = threadIdx.x & (group - 1);
  const int64_t first = WHOLE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (THREADS >> shift) + (threadIdx.x >> shift);
  const int64_t step = WHOLE ? (int64_t)gridDim.x : (int64_t)gridDim.x * (THREADS >> shift);
  float w[K][N], dw[K][N] = {}, db[K][N] = {};
#pragma unroll
  for (int k = 0; k < K; ++k) load_vector(weight, (lane + k * group) * N, width, 1.f, w[k]);
  int turn = 0;
  // every group of a wave goes round as often: a row behind the end is the last one again, and is not counted
  const int64_t rounds = (rows + step - 1) / step;
  for (int64_t i = 0; i < rounds; ++i) {
    const int64_t at = first + i * step;
    const bool there = at < rows;
    const int64_t r = there ? at : rows - 1;
    const float2 of_row = *reinterpret_cast<const float2*>(stats + 2 * r);
    float u[K][N], g[K][N];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      load_chunk(x.at(r), (lane + k * group) * N, width, u[k]);
      load_chunk(dy.at(r), (lane + k * group) * N, width, g[k]);
    }
    float sum[3] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        u[k][n] = (lane + k * group) * N + n < width.width ? u[k][n] - of_row.x : 0.f;
        const float a = g[k][n] * w[k][n];
        sum[0] += a;
        sum[1] = fmaf(a, u[k][n], sum[1]);
        sum[2] += u[k][n];
      }
    sums_of_row<3, WHOLE>(sum, group, room, turn);
    turn ^= 1;
    const float mean_a = sum[0] * per_width, rest = sum[2] * per_width;
    const float mean_au = of_row.y * fmaf(-rest, mean_a, sum[1] * per_width);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int32_t c = (lane + k * group) * N;
      float d[N];
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float unit = (u[k][n] - rest) * of_row.y;
        d[n] = of_row.y * (fmaf(g[k][n], w[k][n], -mean_a) - unit * mean_au);
        dw[k][n] += there ? g[k][n] * unit : 0.f;
        db[k][n] += there ? g[k][n] : 0.f;
      }
      if (there && c < width.width) store_chunk(dx.at(r), c, width, d);
    }
  }
  if (!part) return;
  float* const to = part + (int64_t)blockIdx.x * 2 * width.width;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if (WHOLE) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const int32_t c = (lane + k * group) * N + n;
          if (c < width.width) to[b * width.width + c] = b ? db[k][n] : dw[k][n];
        }
        continue;
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < N; ++n) sums[threadIdx.x][n] = b ? db[k][n] : dw[k][n];
      __syncthreads();
      for (int32_t q = threadIdx.x; q < group * N; q += THREADS) {
        const int32_t c = k * group * N + q;
        if (c >= width.width) break;
        float total = 0.f;
        for (int32_t s = 0; s < THREADS >> shift; ++s) total += sums[(s << shift) + q / N][q % N];
        to[b * width.width + c] = total;
      }
    }
}

template <typename T>
__global__ __launch_bounds__(THREADS) void k_norm_backward_long(RowsOf<const T> dy, RowsOf<const T> x,
                                                                const float* __restrict__ stats,
                                                                const T* __restrict__ weight, RowsOf<T> dx, Width width,
                                                                float per_width) {
  constexpr int N = Chunk<T>::N, STEP = THREADS * N;
  __shared__ float room[2][WAVES][4];
  const int64_t r = blockIdx.x;
  const float2 of_row = *reinterpret_cast<const float2*>(stats + 2 * r);
  float sum[3] = {};
  for (int32_t c = threadIdx.x * N; c < width.width; c += STEP) {
    float u[N], g[N], w[N];
    load_chunk(x.at(r), c, width, u);
    load_chunk(dy.at(r), c, width, g);
    load_vector(weight, c, width, 1.f, w);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float d = c + n < width.width ? u[n] - of_row.x : 0.f, a = g[n] * w[n];
      sum[0] += a;
      sum[1] = fmaf(a, d, sum[1]);
      sum[2] += d;
    }
  }
  sums_of_row<3, true>(sum, THREADS, room, 0);
  const float mean_a = sum[0] * per_width, rest = sum[2] * per_width;
  const float mean_au = of_row.y * fmaf(-rest, mean_a, sum[1] * per_width);
  for (int32_t c = threadIdx.x * N; c < width.width; c += STEP) {
    float u[N], g[N], w[N];
    load_chunk(x.at(r), c, width, u);
    load_chunk(dy.at(r), c, width, g);
    load_vector(weight, c, width, 1.f, w);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float unit = ((u[n] - of_row.x) - rest) * of_row.y;
      w[n] = of_row.y * (fmaf(g[n], w[n], -mean_a) - unit * mean_au);
    }
    store_chunk(dx.at(r), c, width, w);
  }
}

// What is left of long rows when their means, as they were rounded, are taken away: rests[r] is the mean of that.  Without it dweight
// of rows at 10 000 +- 0.1 was off by 0.3 % of itself.  12 us of the 103 that the gradients of 3000 x 6000 f32 take, 74 of 628 for
// 13 120 x 16 000 bf16.
template <typename T>
__global__ __launch_bounds__(THREADS) void k_norm_rests(RowsOf<const T> x, const float* __restrict__ stats, Width width,
                                                        float per_width, float* __restrict__ rests) {
  constexpr int N = Chunk<T>::N, STEP = THREADS * N;
  __shared__ float room[2][WAVES][4];
  const int64_t r = blockIdx.x;
  const float mean = stats[2 * r];
  float sum[1] = {};
  for (int32_t c = threadIdx.x * N; c < width.width; c += STEP) {
    float u[N];
    load_chunk(x.at(r), c, width, u);
#pragma unroll
    for (int n = 0; n < N; ++n) sum[0] += c + n < width.width ? u[n] - mean : 0.f;
  }
  sums_of_row<1, true>(sum, THREADS, room, 0);
  if (threadIdx.x == 0) rests[r] = sum[0] * per_width;
}

// Columns of long rows: a thread's chunk over every gridDim.y-th row.
template <typename T>
__global__ __launch_bounds__(THREADS) void k_norm_columns(RowsOf<const T> dy, RowsOf<const T> x,
                                                          const float* __restrict__ stats, const float* __restrict__ rests,
                                                          int64_t rows, Width width, float* __restrict__ part) {
  constexpr int N = Chunk<T>::N;
  const int32_t c = (blockIdx.x * THREADS + threadIdx.x) * N;
  if (c >= width.width) return;
  float dw[N] = {}, db[N] = {};
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const float2 of_row = *reinterpret_cast<const float2*>(stats + 2 * r);
    const float rest = rests[r];
    float u[N], g[N];
    load_chunk(x.at(r), c, width, u);
    load_chunk(dy.at(r), c, width, g);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      dw[n] = fmaf(g[n], ((u[n] - of_row.x) - rest) * of_row.y, dw[n]);
      db[n] += g[n];
    }
  }
  float* const to = part + (int64_t)blockIdx.y * 2 * width.width;
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (c + n < width.width) {
      to[c + n] = dw[n];
      to[width.width + c + n] = db[n];
    }
}

// How a row is dealt to lanes: 2^shift of them with K chunks each, the workgroup, or (long) again and again.
struct Deal {
  int32_t shift, k;
  bool whole, is_long;
};
Deal deal_of(int64_t width, int chunk) {
  const int64_t cpr = ceil_div(width, chunk);
  Deal d = {0, 1, false, false};
  while (d.shift < 6 && 1 << d.shift < cpr) ++d.shift;
  int64_t lanes = 1 << d.shift;
  if (cpr > 4 * WAVE) {
    d.whole = true;
    lanes = THREADS;
  }
  while (d.k < 4 && d.k * lanes < cpr) d.k *= 2;
  d.is_long = d.k * lanes < cpr;
  return d;
}

constexpr int64_t MOST_PARTS = 1024;
int64_t parts_of_norm(int64_t rows, const Deal& d) {
  if (d.is_long) return rows < 64 ? (rows > 0 ? rows : 1) : 64;
  const int64_t groups = d.whole ? rows : ceil_div(rows, THREADS >> d.shift);
  return groups < 1 ? 1 : (groups < MOST_PARTS ? groups : MOST_PARTS);
}
// Parts, and behind them a number for each of long rows.
size_t norm_space(int64_t rows, int64_t width) {
  int64_t parts = 0, rests = 0;
  for (int chunk = 4; chunk <= 8; chunk += 4) {
    const Deal d = deal_of(width, chunk);
    const int64_t p = parts_of_norm(rows, d);
    parts = p > parts ? p : parts;
    rests = d.is_long ? rows : rests;
  }
  return (size_t)(parts * 2 * width + rests) * sizeof(float) + 256;
}

template <typename Go>
int32_t with_deal(const Deal& d, Go go) {
  if (d.whole) {
    if (d.k == 2) return go(std::integral_constant<int, 2>{}, std::true_type{});
    return go(std::integral_constant<int, 4>{}, std::true_type{});
  }
  if (d.k == 1) return go(std::integral_constant<int, 1>{}, std::false_type{});
  if (d.k == 2) return go(std::integral_constant<int, 2>{}, std::false_type{});
  return go(std::integral_constant<int, 4>{}, std::false_type{});
}

}  // namespace
}  // namespace ginex

using namespace ginex;

extern "C" int32_t ginex_layer_norm(const ginex_rows_t* x, const void* weight, const void* bias, float eps,
                                    const ginex_rows_t* y, float* stats, void* stream) {
  if (int32_t rc = check_rows("x", x, false)) return rc;
  if (int32_t rc = check_rows("y", y, true)) return rc;
  if (int32_t rc = check_same("x", x, "y", y)) return rc;
  if (x->rows != y->rows) return fail(GINEX_ERR_ARG, "x has %lld rows, y %lld", (long long)x->rows, (long long)y->rows);
  if (int32_t rc = check_vector("weight", weight, x->type)) return rc;
  if (int32_t rc = check_vector("bias", bias, x->type)) return rc;
  if (!(eps >= 0.f)) return fail(GINEX_ERR_ARG, "eps=%g", (double)eps);
  if (reinterpret_cast<uintptr_t>(stats) % 8) return fail(GINEX_ERR_ARG, "stats: not aligned to 8 bytes");
  if (x->rows == 0) return GINEX_OK;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const float per_width = (float)(1.0 / (double)x->width);
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const T* const w = static_cast<const T*>(weight);
    const T* const b = static_cast<const T*>(bias);
    const Deal deal = deal_of(x->width, Chunk<T>::N);
    const Width width = Width::of<T>(x->width);
    // (a launch has fewer than 2^32 threads)
    const int64_t step = deal.whole ? (int64_t)1 << 23 : ((int64_t)1 << 31) >> deal.shift;
    for (int64_t r = 0; r < x->rows; r += step) {
      const int64_t rows = x->rows - r < step ? x->rows - r : step;
      const RowsOf<const T> from = {read_rows<T>(x).data + r * x->stride, x->stride};
      const RowsOf<T> to = {rows_of<T>(y).data + r * y->stride, y->stride};
      float* const of_rows = stats ? stats + 2 * r : nullptr;
      if (deal.is_long) {
        hipLaunchKernelGGL(k_norm_long<T>, dim3((unsigned)rows), dim3(THREADS), 0, st, from, to, w, b, width, per_width, eps,
                           of_rows);
      } else {
        with_deal(deal, [&](auto k, auto whole) -> int32_t {
          constexpr int K = decltype(k)::value;
          constexpr bool WHOLE = decltype(whole)::value;
          const int64_t blocks = WHOLE ? rows : ceil_div(rows, THREADS >> deal.shift);
          hipLaunchKernelGGL((k_norm<T, K, WHOLE>), dim3((unsigned)blocks), dim3(THREADS), 0, st, from, to, w, b, rows,
                             deal.shift, width, per_width, eps, of_rows);
          return GINEX_OK;
        });
      }
      GINEX_LAUNCH_CHECK();
    }
    return GINEX_OK;
  });
}

extern "C" size_t ginex_layer_norm_backward_workspace_bytes(int64_t rows, int64_t width) {
  if (rows < 0 || rows >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "rows=%lld", (long long)rows), 0;
  if (width < 1 || width > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "width=%lld (1..%d)", (long long)width, GINEX_MAX_WIDTH), 0;
  return norm_space(rows, width);
}

extern "C" int32_t ginex_layer_norm_backward(const ginex_rows_t* dy, const ginex_rows_t* x, const float* stats,
                                             const void* weight, const ginex_rows_t* dx, float* dweight, float* dbias,
                                             void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_rows("dy", dy, false)) return rc;
  if (int32_t rc = check_rows("x", x, false)) return rc;
  if (int32_t rc = check_rows("dx", dx, true)) return rc;
  if (int32_t rc = check_same("dy", dy, "x", x)) return rc;
  if (int32_t rc = check_same("dx", dx, "x", x)) return rc;
  if (dy->rows != x->rows || dx->rows != x->rows)
    return fail(GINEX_ERR_ARG, "rows: dy %lld, x %lld, dx %lld", (long long)dy->rows, (long long)x->rows, (long long)dx->rows);
  if (int32_t rc = check_vector("weight", weight, x->type)) return rc;
  if ((x->rows > 0 && !stats) || reinterpret_cast<uintptr_t>(stats) % 8)
    return fail(GINEX_ERR_ARG, "stats: null or not aligned to 8 bytes");
  if (!dweight != !dbias) return fail(GINEX_ERR_ARG, "dweight and dbias go together");
  if ((reinterpret_cast<uintptr_t>(dweight) | reinterpret_cast<uintptr_t>(dbias)) % 4)
    return fail(GINEX_ERR_ARG, "dweight, dbias: misaligned");
  const size_t need = norm_space(x->rows, x->width);
  if (dweight) {
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(GINEX_ERR_ARG, "workspace: null or misaligned");
    if (ws_bytes < need) return fail(GINEX_ERR_WORKSPACE, "workspace: need %zu bytes, got %zu", need, ws_bytes);
  }
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const float per_width = (float)(1.0 / (double)x->width);
  float* const part = dweight ? static_cast<float*>(ws) : nullptr;
  const Deal deal = deal_of(x->width, 16 / element_bytes(x->type));
  const int64_t parts = x->rows > 0 ? parts_of_norm(x->rows, deal) : 0;
  if (x->rows > 0) {
    const int32_t rc = with_type(x->type, [&](auto t) -> int32_t {
      using T = decltype(t);
      const T* const w = static_cast<const T*>(weight);
      const Width width = Width::of<T>(x->width);
      if (!deal.is_long) {
        with_deal(deal, [&](auto k, auto whole) -> int32_t {
          hipLaunchKernelGGL((k_norm_backward<T, decltype(k)::value, decltype(whole)::value>), dim3((unsigned)parts),
                             dim3(THREADS), 0, st, read_rows<T>(dy), read_rows<T>(x), stats, w, rows_of<T>(dx), x->rows,
                             deal.shift, width, per_width, part);
          return GINEX_OK;
        });
        GINEX_LAUNCH_CHECK();
        return GINEX_OK;
      }
      const int64_t step = (int64_t)1 << 23;
      // (the columns first: dx may be dy)
      if (part) {
        float* const rests = part + parts * 2 * x->width;
        for (int64_t r = 0; r < x->rows; r += step) {
          const int64_t rows = x->rows - r < step ? x->rows - r : step;
          hipLaunchKernelGGL(k_norm_rests<T>, dim3((unsigned)rows), dim3(THREADS), 0, st,
                             RowsOf<const T>{read_rows<T>(x).data + r * x->stride, x->stride}, stats + 2 * r, width, per_width,
                             rests + r);
          GINEX_LAUNCH_CHECK();
        }
        hipLaunchKernelGGL(k_norm_columns<T>, dim3((unsigned)ceil_div(x->width, THREADS * Chunk<T>::N), (unsigned)parts),
                           dim3(THREADS), 0, st, read_rows<T>(dy), read_rows<T>(x), stats, rests, x->rows, width, part);
        GINEX_LAUNCH_CHECK();
      }
      for (int64_t r = 0; r < x->rows; r += step) {
        const int64_t rows = x->rows - r < step ? x->rows - r : step;
        hipLaunchKernelGGL(k_norm_backward_long<T>, dim3((unsigned)rows), dim3(THREADS), 0, st,
                           RowsOf<const T>{read_rows<T>(dy).data + r * dy->stride, dy->stride},
                           RowsOf<const T>{read_rows<T>(x).data + r * x->stride, x->stride}, stats + 2 * r, w,
                           RowsOf<T>{rows_of<T>(dx).data + r * dx->stride, dx->stride}, width, per_width);
        GINEX_LAUNCH_CHECK();
      }
      return GINEX_OK;
    });
    if (rc) return rc;
  }
  if (part)
    GINEX_HIP(join_async(part, nullptr, 1, 0, 1, parts, 2 * (int32_t)x->width, (int32_t)x->width, dweight, dbias, st));
  return GINEX_OK;
}
