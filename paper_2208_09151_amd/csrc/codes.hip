// Activations kept in 8 bits: compress (with the activation in the same pass), restore, and the
// activation's gradient from the codes.
//
// Elementwise, bound by HBM; gelu in 16 bits by the vector unit as well, some 40 instructions an element.  A
// thread has two chunks of 16 bytes of the wide side and their 4 (f32) or 8 codes; 8 or 4 neighbouring lanes
// share a block of 32 channels and find its largest magnitude by exchanging lanes.  Chunks are numbered
// through all rows, padded to whole blocks, so that no lane idles for a width that is no power of two.
//
// Measured (bytes that have to move, over the time of a call among others, inputs and outputs of 4 to 10 calls in turn, so
// that none are in the caches of 256 MB; a plain copy reaches 6.2 TB/s, what writes more than it reads somewhat more):
//                        compress       with silu      with gelu      restore        silu's gradient  gelu's
//   820 000 x 256 f32    171 us 6.2     302 us 6.3     302 us 6.3     161 us 6.5     309 us 6.1       307 us 6.2 TB/s
//   820 000 x 256 bf16   108    5.9     170    6.2     180    5.9      99    6.4     177    6.0       186    5.7
//   300 000 x 333 f16     54    5.7      92    5.5     103    4.9      60    5.2      89    5.7        99    5.1
// (Codes that are still in the caches: restore of the first 145 us.)
#include "activations.hpp"
#include "codes.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;
// Chunks of a thread, their loads issued together (compress, 820 000 x 256 f32: 179 us with one, 175 with two, 174 with four;
// silu 313, 309 and 322; 300 000 x 333 f16: 57, 49 and 49, silu's gradient 90, 83 and 87).
constexpr int UNROLL = 2;

// The codes of a chunk, as one word of N bytes.
template <int N>
struct Word;
template <>
struct Word<4> {
  typedef uint32_t type;
};
template <>
struct Word<8> {
  typedef uint64_t type;
};

// The largest of the 4 or 8 neighbouring lanes that share a block, in all of them.
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {
  const uint32_t other = dpp_or_zero<CTRL, 0xF>(v);
  return v > other ? v : other;
}
template <int LANES>
__device__ __forceinline__ uint32_t max_of_block(uint32_t v) {
  v = max_with<0xB1>(v);                        // quad_perm [1, 0, 3, 2]
  v = max_with<0x4E>(v);                        // quad_perm [2, 3, 0, 1]
  return LANES == 8 ? max_with<0x141>(v) : v;   // row_half_mirror: the other four of eight
}

template <typename T, int ACT>
__global__ __launch_bounds__(THREADS) void k_compress(RowsOf<const T> x, RowsOf<T> y, int8_t* __restrict__ codes,
                                                      uint8_t* __restrict__ scales, int64_t first, uint32_t chunks,
                                                      Divisor cpr, Width width) {
  constexpr int N = Chunk<T>::N, LANES = GINEX_CODE_BLOCK / N, U = UNROLL;
  uint32_t at[U];
  int64_t r[U];
  float v[U][N];
  // (a chunk behind the last one repeats it and is not written: all lanes of a block do the same, as chunks is a multiple of
  // LANES)
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t t = (blockIdx.x * U + u) * THREADS + threadIdx.x;
    t = t < chunks ? t : chunks - LANES + t % LANES;
    const uint32_t row = cpr.of(t);
    at[u] = t - row * cpr.d;
    r[u] = first + row;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) load_chunk(x.at(r[u]), (int32_t)at[u] * N, width, v[u]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if ((blockIdx.x * U + u) * THREADS + threadIdx.x >= chunks) return;
    const int32_t c = (int32_t)at[u] * N;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t magnitude = __float_as_uint(v[u][i]) & 0x7FFFFFFFu;
      top = top > magnitude ? top : magnitude;
    }
    const uint32_t scale = scale_byte(max_of_block<LANES>(top));
    const float by = to_codes(scale);
    // v by + 1.5 2^23 is rounded to a whole number, halves to even, and has it in its lowest bits
    constexpr float whole = 12582912.f;
    float q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = __builtin_amdgcn_fmed3f(fmaf(v[u][i], by, whole), whole - 127.f, whole + 127.f);
    typename Word<N>::type word = low_bytes(q[0], q[1], q[2], q[3]);
    if constexpr (N == 8) word |= (uint64_t)low_bytes(q[4], q[5], q[6], q[7]) << 32;
    word = scale == NO_NUMBER ? 0 : word;
    const int64_t chunk = r[u] * cpr.d + at[u];
    __builtin_nontemporal_store(word, reinterpret_cast<typename Word<N>::type*>(codes) + chunk);
    if (at[u] % LANES == 0) scales[chunk / LANES] = (uint8_t)scale;
    if (ACT != GINEX_ACT_NONE && c < width.width) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[u][i] = activated<ACT, sizeof(T) == 4>(v[u][i]);
      store_chunk(y.at(r[u]), c, width, v[u]);
    }
  }
}

template <int N>
__device__ __forceinline__ void restored(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                         int64_t chunk, float (&v)[N]) {
  const typename Word<N>::type word = reinterpret_cast<const typename Word<N>::type*>(codes)[chunk];
  const float step = code_step(scales[chunk / (GINEX_CODE_BLOCK / N)]);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (float)(int8_t)(word >> (8 * i)) * step;
}

// ACT < 0: out = the restored values; else out = dy f'(restored).
template <typename T, int ACT>
__global__ __launch_bounds__(THREADS) void k_restore(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                     RowsOf<const T> dy, RowsOf<T> out, int64_t first, uint32_t chunks,
                                                     Divisor cpr, Width width) {
  constexpr int N = Chunk<T>::N, U = UNROLL;
  int32_t c[U];
  int64_t r[U];
  float v[U][N], g[U][N];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t t = (blockIdx.x * U + u) * THREADS + threadIdx.x;
    t = t < chunks ? t : chunks - 1;
    const uint32_t row = cpr.of(t);
    c[u] = (int32_t)(t - row * cpr.d) * N;
    r[u] = first + row;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    restored<N>(codes, scales, r[u] * cpr.d + c[u] / N, v[u]);
    if (ACT >= 0) load_chunk(dy.at(r[u]), c[u], width, g[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if ((blockIdx.x * U + u) * THREADS + threadIdx.x >= chunks) return;
    if (c[u] >= width.width) continue;
    if (ACT >= 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[u][i] = sloped<ACT, sizeof(T) == 4>(v[u][i], g[u][i]);
    }
    store_chunk(out.at(r[u]), c[u], width, v[u]);
  }
}

// Calls go(first row, chunks, chunks of a row) for the launches that cover `rows` rows, chunks numbered in 31 bits.
template <typename T, typename Go>
int32_t by_launches(int64_t rows, int64_t width, Go go) {
  const int64_t cpr = code_blocks(width) * (GINEX_CODE_BLOCK / Chunk<T>::N);
  const int64_t step = (((int64_t)1 << 31) - THREADS * UNROLL) / cpr;
  for (int64_t r = 0; r < rows; r += step) {
    go(r, (uint32_t)((rows - r < step ? rows - r : step) * cpr), Divisor((uint32_t)cpr));
    GINEX_LAUNCH_CHECK();
  }
  return GINEX_OK;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

extern "C" int32_t ginex_compress(const ginex_rows_t* x, int32_t activation, const ginex_rows_t* y,
                                  const ginex_codes_t* kept, void* stream) {
  if (int32_t rc = check_rows("x", x, false)) return rc;
  if (int32_t rc = check_codes(kept)) return rc;
  if (int32_t rc = check_kept("x", x, kept)) return rc;
  if (int32_t rc = check_activation(activation, GINEX_ACT_NONE)) return rc;
  if ((activation != GINEX_ACT_NONE) != (y != nullptr)) return fail(GINEX_ERR_ARG, "y goes with an activation, and only with one");
  if (y) {
    if (int32_t rc = check_rows("y", y, true)) return rc;
    if (int32_t rc = check_same("x", x, "y", y)) return rc;
    if (int32_t rc = check_kept("y", y, kept)) return rc;
  }
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const RowsOf<T> to = y ? rows_of<T>(y) : RowsOf<T>{nullptr, 0};
    const auto kernel = activation == GINEX_ACT_NONE   ? k_compress<T, GINEX_ACT_NONE>
                        : activation == GINEX_ACT_RELU ? k_compress<T, GINEX_ACT_RELU>
                        : activation == GINEX_ACT_SILU ? k_compress<T, GINEX_ACT_SILU>
                                                       : k_compress<T, GINEX_ACT_GELU>;
    return by_launches<T>(x->rows, x->width, [&](int64_t r, uint32_t chunks, Divisor cpr) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(chunks, THREADS * UNROLL)), dim3(THREADS), 0, st, read_rows<T>(x), to,
                         kept->codes, kept->scales, r, chunks, cpr, Width::of<T>(x->width));
    });
  });
}

extern "C" int32_t ginex_restore(const ginex_codes_t* kept, const ginex_rows_t* out, void* stream) {
  if (int32_t rc = check_codes(kept)) return rc;
  if (int32_t rc = check_rows("out", out, true)) return rc;
  if (int32_t rc = check_kept("out", out, kept)) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(out->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    return by_launches<T>(out->rows, out->width, [&](int64_t r, uint32_t chunks, Divisor cpr) {
      hipLaunchKernelGGL((k_restore<T, -1>), dim3((unsigned)ceil_div(chunks, THREADS * UNROLL)), dim3(THREADS), 0, st, kept->codes,
                         kept->scales, RowsOf<const T>{nullptr, 0}, rows_of<T>(out), r, chunks, cpr, Width::of<T>(out->width));
    });
  });
}

extern "C" int32_t ginex_activate_backward(const ginex_codes_t* kept, int32_t activation, const ginex_rows_t* dy,
                                           const ginex_rows_t* dx, void* stream) {
  if (int32_t rc = check_codes(kept)) return rc;
  if (int32_t rc = check_activation(activation, GINEX_ACT_RELU)) return rc;
  if (int32_t rc = check_rows("dy", dy, false)) return rc;
  if (int32_t rc = check_rows("dx", dx, true)) return rc;
  if (int32_t rc = check_same("dy", dy, "dx", dx)) return rc;
  if (int32_t rc = check_kept("dy", dy, kept)) return rc;
  if (int32_t rc = check_kept("dx", dx, kept)) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(dy->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const auto kernel = activation == GINEX_ACT_RELU   ? k_restore<T, GINEX_ACT_RELU>
                        : activation == GINEX_ACT_SILU ? k_restore<T, GINEX_ACT_SILU>
                                                       : k_restore<T, GINEX_ACT_GELU>;
    return by_launches<T>(dy->rows, dy->width, [&](int64_t r, uint32_t chunks, Divisor cpr) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(chunks, THREADS * UNROLL)), dim3(THREADS), 0, st, kept->codes, kept->scales,
                         read_rows<T>(dy), rows_of<T>(dx), r, chunks, cpr, Width::of<T>(dx->width));
    });
  });
}
