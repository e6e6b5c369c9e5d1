// Few rows: a linear layer, or a whole layer of experts in two launches.
//
//   scores(r, e) = <x[r], router[e]>, the experts of the `top` largest, p(r, :) their softmax          (first launch)
//   y[r] = sum over j of p(r, j) f(x[r] W_e(r,j) + bias_e(r,j))                                      (second launch)
//
// What counts is how fast the weights arrive, and before that the latency of a handful of dependent steps.  A workgroup has 64
// columns of one expert and all rows that are sent to it; its waves share the width, and each streams its part of the weights
// from HBM straight into the registers of the matrix instructions (columns are the first operand, rows the second, 16 at a
// time; weights with dense columns are turned over in registers).  The waves' sums meet in LDS.  In a layer of experts each
// leaves f(..) of its pairs in the workspace, and of the workgroups of the same columns the one that comes last adds them up,
// in the order of j.
//
// One row, 1024 -> 1024 f16, 7.2 us as a linear layer, 12.7 through two of 64 experts: latency.  48 rows through four of 32
// experts, 500 -> 777 f16, 26.4 us for both, of which the weights' 25 MB would take 5; rows of 777 elements begin at any 2 bytes (768
// columns: 20.9).
#include "activations.hpp"
#include "codes.hpp"
#include "layers.hpp"

namespace ginex {
namespace {

constexpr int ROUTE_THREADS = 1024, ROUTE_WAVES = ROUTE_THREADS / WAVE;
constexpr int PITCH = WAVE_COLUMNS + 4;                   // of a row of sums in LDS: 16 rows of 4 words use every bank once

// The sum over a wave, in its last lane: lane by lane inside rows of 16 (DPP), then across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ double plus_lane(double v) {
  return v + __longlong_as_double((long long)dpp_or_zero<CTRL, ROWS>((uint64_t)__double_as_longlong(v)));
}
__device__ __forceinline__ double sum_to_last(double v) {
  v = plus_lane<0x111, 0xF>(v);     // row_shr:1
  v = plus_lane<0x112, 0xF>(v);
  v = plus_lane<0x114, 0xF>(v);
  v = plus_lane<0x118, 0xF>(v);
  v = plus_lane<0x142, 0xA>(v);     // row_bcast:15
  return plus_lane<0x143, 0xC>(v);  // row_bcast:31
}

// The largest number of a wave, in all lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t or_lane(uint32_t v) {
  const uint32_t other = dpp_or_zero<CTRL, ROWS>(v);
  return v > other ? v : other;
}
__device__ __forceinline__ uint32_t most_of_wave(uint32_t v) {
  v = or_lane<0x111, 0xF>(v);
  v = or_lane<0x112, 0xF>(v);
  v = or_lane<0x114, 0xF>(v);
  v = or_lane<0x118, 0xF>(v);
  v = or_lane<0x142, 0xA>(v);
  v = or_lane<0x143, 0xC>(v);
  return of_lane(v, WAVE - 1);
}

// A score as a number that is larger where the score is; NaN is the largest, 0 is smaller than all.
__device__ __forceinline__ uint64_t rank_of(double v) {
  if (v != v) return ~(uint64_t)0;
  const uint64_t bits = (uint64_t)__double_as_longlong(v + 0.0);      // (-0 is 0)
  return bits >> 63 ? ~bits : bits | (uint64_t)1 << 63;
}

// What the two launches share.
struct Plan {
  int32_t* chosen;      // [rows x top]
  float* share;         // [rows x top]
  uint32_t* done;       // pairs of which 64 columns are through
  float* part;          // [rows x top x out]
};

// The scores of one row.  Products in f64 are exact for all types, so what is chosen does not depend on how a sum is rounded
// (but for scores that are equal to 2^-50 or so).  Called by ROUTE_THREADS.
template <typename T>
__device__ __forceinline__ void few_scores(const T* row, RowsOf<const T> router, int32_t experts, Width width, double* scores) {
  constexpr int N = Chunk<T>::N, U = 4;
  const int lane = lane_id(), wave = threadIdx.x / WAVE;
  for (int32_t e0 = wave; e0 < experts; e0 += U * ROUTE_WAVES) {
    double sum[U] = {};
    // two chunks of U experts in flight
    for (int32_t c0 = lane * N; c0 < width.width; c0 += 2 * WAVE * N) {
      ChunkWords<T> a[2], b[2][U];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int32_t c = c0 + k * WAVE * N;
        a[k] = load_words(row, c, width);
#pragma unroll
        for (int u = 0; u < U; ++u)
          b[k][u] = load_words(router.at(e0 + u * ROUTE_WAVES < experts ? e0 + u * ROUTE_WAVES : e0), c, width);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int n = 0; n < N; ++n) sum[u] = fma((double)(float)a[k].wide[n], (double)(float)b[k][u].wide[n], sum[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) sum[u] = sum_to_last(sum[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (lane == WAVE - 1 && e0 + u * ROUTE_WAVES < experts) scores[e0 + u * ROUTE_WAVES] = sum[u];
  }
}

// A wave's choice by the scores, EACH a lane at most: lane j gets choice j and its share.  (A wave that comes by once waits for its
// instructions more than for anything else, so that what a call does not need is not there: 48 rows, four of 32 experts each, take
// 35.4 us with EACH 1 and 37.7 with 16.)
template <int EACH>
__device__ __forceinline__ void few_choices(const double* scores, int32_t experts, int32_t top, int32_t& mine, float& share) {
  const int lane = lane_id();
  uint64_t rank[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) rank[i] = lane + i * WAVE < experts ? rank_of(scores[lane + i * WAVE]) : 0;
  mine = 0;
  for (int32_t j = 0; j < top; ++j) {
    uint64_t best = rank[0];
    uint32_t at = lane;
#pragma unroll
    for (int i = 1; i < EACH; ++i)
      if (i * WAVE < experts && rank[i] > best) {
        best = rank[i];
        at = lane + i * WAVE;
      }
    // the largest rank, its upper half first, and of those that have it the first expert; mostly the upper half tells
    const uint32_t hi = most_of_wave((uint32_t)(best >> 32));
    uint64_t who = __ballot(best >> 32 == hi);
    if (who & (who - 1)) {
      const uint32_t lo = most_of_wave(best >> 32 == hi ? (uint32_t)best : 0);
      who = __ballot(best == ((uint64_t)hi << 32 | lo));
      if (who & (who - 1)) who = __ballot(at == ~most_of_wave(who >> lane & 1 ? ~at : 0));
    }
    at = of_lane(at, __ffsll((unsigned long long)who) - 1);
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (i * WAVE < experts && at == (uint32_t)(lane + i * WAVE)) rank[i] = 0;
    if (lane == j) mine = (int32_t)at;
  }
  // 2^t by the f32 instruction, of t's fraction: good to 2^-22
  const double score = scores[mine], far = (score - __shfl(score, 0, WAVE)) * 1.4426950408889634;
  const double t = far < -1000.0 ? -1000.0 : far, whole = rint(t);
  const double weight = lane < top ? ldexp((double)__builtin_amdgcn_exp2f((float)(t - whole)), (int)whole) : 0.0, total = __shfl(sum_to_last(weight), WAVE - 1, WAVE);
  share = (float)(weight / total);
}

// A workgroup a row.
template <typename T, int EACH>
__global__ __launch_bounds__(ROUTE_THREADS) void k_few_route(RowsOf<const T> x, RowsOf<const T> router, int32_t experts,
                                                             int32_t top, Width width, Plan plan, int32_t tiles) {
  __shared__ double scores[GINEX_MAX_EXPERTS];
  if (blockIdx.x == 0)
    for (int32_t i = threadIdx.x; i < tiles; i += ROUTE_THREADS) plan.done[i] = 0;
  few_scores(x.at(blockIdx.x), router, experts, width, scores);
  __syncthreads();
  if (threadIdx.x >= WAVE) return;
  int32_t mine;
  float share;
  few_choices<EACH>(scores, experts, top, mine, share);
  if (lane_id() < top) {
    plan.chosen[(int64_t)blockIdx.x * top + lane_id()] = mine;
    plan.share[(int64_t)blockIdx.x * top + lane_id()] = share;
  }
}

// Rows of one expert and their sums: x[row(i)] W for i < count <= 16; of column 4 (lane % 16) + j of the workgroup's in operand j.
// `row_of(i)` is the row of x, negative for a row of zeros.  `wave` of the `waves` that share the width.
template <typename T, bool TURNED, typename RowOf>
__device__ __forceinline__ void few_sums(int wave, int waves, RowsOf<const T> x, const T* __restrict__ w,
                                         int64_t stride, int32_t width, Width out, int32_t n0, int32_t count, RowOf row_of,
                                         float4v (&sum)[4]) {
  constexpr int N = Chunk<T>::N, STEP = 4 * N, UNIT = 2 * STEP;       // a unit is 128 bytes of a row
  const int lane = lane_id(), group = lane / 16;
  const Width along = {width, (int32_t)((width + N - 1) / N * N - width)};
  const int64_t r = row_of(lane % 16 < count ? lane % 16 : 0);
  const T* const row = x.at(r >= 0 ? r : 0);
  const int32_t n = n0 + lane % 16 * 4;
  for (int32_t k0 = wave * UNIT; k0 < width; k0 += waves * UNIT) {
    ChunkWords<T> fa[2], fb[2][4];
    typename Four<T>::Wide raw[2][N];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int32_t k1 = k0 + s * STEP + group * N;
      if (TURNED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) fb[s][j] = load_words(w + (n + j < out.width ? n + j : out.width - 1) * stride, k1, along);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int32_t k = k1 + i;
          raw[s][i] = four_of(w + (int64_t)(k < width ? k : width - 1) * stride, n < out.width ? n : out.width - 1, out.width);
          if (k >= width) raw[s][i] = (typename Four<T>::Wide)(T)0.f;
        }
      }
      fa[s] = load_words(row, k1, along);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (!TURNED) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < N; ++i) fb[s][j].wide[i] = raw[s][i][j];
      }
      if (r < 0) fa[s].words = words4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] = product(fb[s][j], fa[s], sum[j]);
    }
  }
}

// The waves' sums of 16 rows, added up: wave w gets rows w, w + WAVES, .. of the column that is its lane's.
template <int WAVES>
__device__ __forceinline__ void join_waves(const float4v (&sum)[4], float (*room)[16][PITCH], float (&v)[16 / WAVES]) {
  const int lane = lane_id(), wave = threadIdx.x / WAVE;
  __syncthreads();
  // lane's row is lane % 16; component i of operand j's sums is column 16 (lane / 16) + 4 i + j
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<float4v*>(&room[wave][lane % 16][lane / 16 * 16 + 4 * i]) = float4v{sum[0][i], sum[1][i], sum[2][i], sum[3][i]};
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 16 / WAVES; ++h) {
    v[h] = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v[h] += room[w][wave + h * WAVES][lane];
  }
}

// A workgroup has 64 columns (x) of an expert's 16 pairs (z).  Which expert (y): each has its own workgroups, or, where there are
// fewer pairs than experts, each pair has, and those of an expert's first pair do the work.
template <typename T, bool TURNED, int WAVES>
__global__ __launch_bounds__(WAVES* WAVE) void k_few_experts(RowsOf<const T> x, int32_t pairs, int32_t top, int32_t rows,
                                                             WeightsOf<T> weights, int32_t by_pair,
                                                             const T* __restrict__ bias, int32_t width, Width out,
                                                             int32_t activation, Plan plan, RowsOf<T> y) {
  __shared__ int32_t lists[WAVES][16];
  __shared__ int32_t is_last;
  __shared__ float room[WAVES][16][PITCH];
  const int lane = lane_id(), wave = threadIdx.x / WAVE;
  const int32_t expert = by_pair ? plan.chosen[blockIdx.y] : (int32_t)blockIdx.y;
  // every wave finds its pairs in their order
  int32_t* const list = lists[wave];
  int32_t have = -(int32_t)blockIdx.z * 16;
  for (int32_t p0 = 0; p0 < pairs; p0 += 4 * WAVE) {
    int32_t of_pair[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int32_t p = p0 + k * WAVE + lane;
      of_pair[k] = plan.chosen[p < pairs ? p : pairs - 1];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int32_t p = p0 + k * WAVE + lane;
      const bool is = p < pairs && of_pair[k] == expert;
      const uint64_t who = __ballot(is);
      if (who == 0) continue;
      if (by_pair && p0 + k * WAVE + __ffsll((unsigned long long)who) - 1 < (int32_t)blockIdx.y) return;
      const int32_t place = have + __popcll(who & (((uint64_t)1 << lane) - 1));
      if (is && place >= 0 && place < 16) list[place] = p;
      have += __popcll(who);
    }
  }
  if (have <= 0) return;                    // (the same for all waves)
  const int32_t count = have < 16 ? have : 16;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();          // lanes read what others of their wave have written
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const int32_t n0 = blockIdx.x * WAVE_COLUMNS, c = n0 + lane;
  float4v sum[4] = {};
  few_sums<T, TURNED>(__builtin_amdgcn_readfirstlane(wave), WAVES, x, weights.of(expert), weights.stride, width, out, n0,
                      count, [&](int32_t i) { return (int64_t)(list[i] / top); }, sum);
  const float b = bias && c < out.width ? (float)bias[(int64_t)expert * out.width + c] : 0.f;
  float v[16 / WAVES];
  join_waves<WAVES>(sum, room, v);
#pragma unroll
  for (int h = 0; h < 16 / WAVES; ++h) {
    const int32_t i = wave + h * WAVES;
    if (i < count && c < out.width)
      __hip_atomic_store(plan.part + (int64_t)list[i] * out.width + c, activated_by<sizeof(T) == 4>(activation, v[h] + b),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  // The last workgroup of these columns to come here finds what the others have left, whichever die they were on: stores and
  // loads of that go past the dies' caches, and every wave waits for its stores before one thread counts its pairs.  So the
  // count itself has nothing to write back or to invalidate, which would cost 3 to 8 us.  This rests on the instructions, not on the
  // language, whose relaxed accesses order nothing between them: on gfx950 a relaxed access of agent scope is one with sc1 set,
  // and a store of that kind is counted by vmcnt until it is where all dies see it.  A test reads the listing for both.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    is_last = (int32_t)__hip_atomic_fetch_add(plan.done + blockIdx.x, (uint32_t)count, __ATOMIC_RELAXED,
                                              __HIP_MEMORY_SCOPE_AGENT) + count == pairs;
  __syncthreads();
  if (!is_last || c >= out.width) return;
  // a wave has some rows, whose pairs are neighbours: U of them in flight
  constexpr int U = 16;
  const float* const part = plan.part + c;
  const int32_t each = (rows + WAVES - 1) / WAVES;
  const int32_t first = wave * each * top, end = (wave + 1) * each < rows ? (wave + 1) * each * top : pairs;
  int32_t r = wave * each, j = 0;
  float total = 0.f;
  for (int32_t p0 = first; p0 < end; p0 += U) {
    float v[U], share[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t p = p0 + u < end ? p0 + u : end - 1;
      share[u] = plan.share[p];
      v[u] = __hip_atomic_load(part + (int64_t)p * out.width, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool there = p0 + u < end;
      total = there ? fmaf(share[u], v[u], total) : total;
      j += there ? 1 : 0;
      if (j == top) {
        y.at(r)[c] = (T)total;
        total = 0.f;
        j = 0;
        ++r;
      }
    }
  }
}

// One row, in one launch: every workgroup finds the row's experts by itself and has 64 columns of all of them, a part of its waves
// for each.  It costs the router's bytes once a workgroup, and spares a launch and the meeting of the workgroups.
constexpr int MOST_OF_ONE = 2;
template <typename T, bool TURNED, int EACH>
__global__ __launch_bounds__(ROUTE_THREADS) void k_few_one(RowsOf<const T> x, RowsOf<const T> router, int32_t experts, int32_t top,
                                                           Width along, WeightsOf<T> weights,
                                                           const T* __restrict__ bias, Width out, int32_t activation, T* y) {
  __shared__ double scores[GINEX_MAX_EXPERTS];
  __shared__ int32_t chosen[MOST_OF_ONE];
  __shared__ float shares[MOST_OF_ONE], room[ROUTE_WAVES][WAVE_COLUMNS];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int32_t n0 = blockIdx.x * WAVE_COLUMNS, c = n0 + lane;
  few_scores(x.at(0), router, experts, along, scores);
  __syncthreads();
  if (wave == 0) {
    int32_t mine;
    float share;
    few_choices<EACH>(scores, experts, top, mine, share);
    if (lane < top) {
      chosen[lane] = mine;
      shares[lane] = share;
    }
  }
  __syncthreads();
  const int32_t each = ROUTE_WAVES / top, j = wave / each;      // `each` waves an expert
  float4v sum[4] = {};
  few_sums<T, TURNED>(wave % each, each, x, weights.of(__builtin_amdgcn_readfirstlane(chosen[j])), weights.stride, along.width, out,
                      n0, 1, [](int32_t) { return (int64_t)0; }, sum);
  if (lane % 16 == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4v*>(&room[wave][lane / 16 * 16 + 4 * i]) = float4v{sum[0][i], sum[1][i], sum[2][i], sum[3][i]};
  }
  __syncthreads();
  if (wave > 0 || c >= out.width) return;
  float total = 0.f;
  for (int32_t k = 0; k < top; ++k) {
    float z = bias ? (float)bias[(int64_t)chosen[k] * out.width + c] : 0.f;
    for (int32_t w = 0; w < each; ++w) z += room[k * each + w][lane];
    total = fmaf(shares[k], activated_by<sizeof(T) == 4>(activation, z), total);
  }
  y[c] = (T)total;
}

// 16 slots of one expert, or without one, or 16 rows a workgroup.
template <typename T, bool TURNED, int WAVES>
__global__ __launch_bounds__(WAVES* WAVE) void k_few_linear(RowsOf<const T> x, int64_t rows, WeightsOf<T> weights,
                                                                   const int32_t* __restrict__ source,
                                                                   const int64_t* __restrict__ offsets, int32_t experts,
                                                                   int64_t slots, int32_t width, Width out, Epilogue e) {
  __shared__ float room[WAVES][16][PITCH];
  const int lane = lane_id(), wave = threadIdx.x / WAVE;
  TileRows tile = {0, (int64_t)blockIdx.y * 16, slots};
  if (offsets) {
    if (!find_tile(offsets, experts, slots, blockIdx.y, 16, tile)) return;
  }
  const int32_t expert = tile.expert;
  const int64_t begin = tile.first, end = tile.end;
  const int32_t count = (int32_t)(end - begin < 16 ? end - begin : 16), n0 = blockIdx.x * WAVE_COLUMNS, c = n0 + lane;
  const bool none = expert == experts;        // slots without an expert are cleared
  float4v sum[4] = {};
  if (!none)
    few_sums<T, TURNED>(__builtin_amdgcn_readfirstlane(wave), WAVES, x, weights.of(expert), weights.stride, width, out, n0,
                        count,
                        [&](int32_t i) -> int64_t {
                          const int64_t r = source ? (int64_t)source[begin + i] : begin + i;
                          return r < rows ? r : -1;
                        },
                        sum);
  const float b = !none && e.bias && c < out.width
                      ? (float)static_cast<const T*>(e.bias)[(int64_t)expert * out.width + c] : 0.f;
  float v[16 / WAVES];
  join_waves<WAVES>(sum, room, v);
#pragma unroll
  for (int h = 0; h < 16 / WAVES; ++h) {
    const int32_t i = wave + h * WAVES;
    if (i >= count) continue;               // (the same for the wave)
    const int64_t r = begin + i;
    v[h] = c < out.width ? v[h] + b : 0.f;
    if (e.codes) {
      // a block is half of the wave
      uint32_t most = __float_as_uint(v[h]) & 0x7FFFFFFFu;
#pragma unroll
      for (int d = 1; d < GINEX_CODE_BLOCK; d *= 2) {
        const uint32_t other = (uint32_t)__shfl_xor((int)most, d, WAVE);
        most = most > other ? most : other;
      }
      const uint32_t scale = scale_byte(most);
      constexpr float whole = 12582912.f;
      const float q = __builtin_amdgcn_fmed3f(fmaf(v[h], to_codes(scale), whole), whole - 127.f, whole + 127.f);
      if (c < e.blocks * GINEX_CODE_BLOCK) {
        e.codes[r * ((int64_t)e.blocks * GINEX_CODE_BLOCK) + c] = scale == NO_NUMBER ? 0 : (int8_t)__float_as_uint(q);
        if (c % GINEX_CODE_BLOCK == 0) e.scales[r * e.blocks + c / GINEX_CODE_BLOCK] = (uint8_t)scale;
      }
    }
    if (c >= out.width) continue;
    float to = none ? 0.f : activated_by<sizeof(T) == 4>(e.activation, v[h]);
    if (e.residual && !none) to += (float)static_cast<const T*>(e.residual)[r * e.residual_stride + c];
    static_cast<T*>(e.y)[r * e.y_stride + c] = (T)to;
  }
}

struct FewSpace {
  Plan plan;
  size_t bytes;
};
FewSpace few_space(void* ws, int64_t rows, int32_t top, int64_t out) {
  Arena arena(ws);
  FewSpace s;
  s.plan.chosen = arena.take<int32_t>(rows * top);
  s.plan.share = arena.take<float>(rows * top);
  s.plan.done = arena.take<uint32_t>(ceil_div(out, WAVE_COLUMNS));
  s.plan.part = arena.take<float>(rows * top * out);
  s.bytes = arena.used + 256;
  return s;
}

int32_t check_few(int64_t rows, int32_t top, int32_t experts, int64_t width, int64_t out) {
  if (rows < 0 || rows > GINEX_MAX_FEW_ROWS) return fail(GINEX_ERR_ARG, "rows=%lld (0..%d)", (long long)rows, GINEX_MAX_FEW_ROWS);
  if (experts < 1 || experts > GINEX_MAX_EXPERTS) return fail(GINEX_ERR_ARG, "experts=%d (1..%d)", experts, GINEX_MAX_EXPERTS);
  if (top < 1 || top > GINEX_MAX_FEW_TOP || top > experts)
    return fail(GINEX_ERR_ARG, "top=%d of %d experts (1..%d)", top, experts, GINEX_MAX_FEW_TOP);
  if (width < 1 || width > GINEX_MAX_WIDTH || out < 1 || out > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "width %lld or out %lld (1..%d)", (long long)width, (long long)out, GINEX_MAX_WIDTH);
  return GINEX_OK;
}

// Calls `go` with how many experts a lane has.
template <typename Go>
int32_t with_each(int32_t experts, Go go) {
  if (experts <= WAVE) return go(std::integral_constant<int, 1>{});
  if (experts <= 4 * WAVE) return go(std::integral_constant<int, 4>{});
  return go(std::integral_constant<int, GINEX_MAX_EXPERTS / WAVE>{});
}

// Calls `go` with the waves of a workgroup: as many as the width has units of 128 bytes, 4, 8, or 16 where there are few
// workgroups.
template <typename Go>
int32_t with_waves(int64_t width, int32_t bytes, int64_t groups, Go go) {
  const int64_t units = ceil_div(width * bytes, 128);
  if (units <= 4) return go(std::integral_constant<int, 4>{});
  if (units <= 8 || groups > 256) return go(std::integral_constant<int, 8>{});
  return go(std::integral_constant<int, 16>{});
}

}  // namespace

int64_t few_groups(const ginex_weights_t* w, const ginex_routing_t* route, int64_t slots) {
  const int64_t tiles = route ? most_tiles(slots, route->experts, 16) : ceil_div(slots, 16);
  return ceil_div(w->out, WAVE_COLUMNS) * tiles;
}

int32_t linear_few(const ginex_rows_t* x, const ginex_weights_t* w, const ginex_routing_t* route, bool by_slot, int64_t slots,
                   const Epilogue& epilogue, hipStream_t st) {
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const int64_t groups = few_groups(w, route, slots), tiles = groups / ceil_div(w->out, WAVE_COLUMNS);
    return with_waves(w->width, sizeof(T), groups, [&](auto waves) -> int32_t {
      constexpr int WAVES = decltype(waves)::value;
      const auto kernel = w->turned ? k_few_linear<T, true, WAVES> : k_few_linear<T, false, WAVES>;
      const dim3 grid((unsigned)ceil_div(w->out, WAVE_COLUMNS), (unsigned)tiles);
      hipLaunchKernelGGL(kernel, grid, dim3(WAVES * WAVE), 0, st, read_rows<T>(x), x->rows, weights_of<T>(w),
                         route && !by_slot ? route->source : nullptr, route ? route->offsets : nullptr, w->experts, slots,
                         (int32_t)w->width, Width::of<T>(w->out), epilogue);
      GINEX_LAUNCH_CHECK();
      return GINEX_OK;
    });
  });
}

}  // namespace ginex

using namespace ginex;

extern "C" size_t ginex_expert_layer_workspace_bytes(int64_t rows, int32_t top, int32_t experts, int64_t width, int64_t out) {
  if (check_few(rows, top, experts, width, out)) return 0;
  return few_space(nullptr, rows, top, out).bytes;
}

extern "C" int32_t ginex_expert_layer(const ginex_rows_t* x, const ginex_rows_t* router, const ginex_weights_t* weights,
                                      const void* bias, int32_t top, int32_t activation, const ginex_rows_t* y, void* ws,
                                      size_t ws_bytes, void* stream) {
  if (int32_t rc = check_rows("x", x, false)) return rc;
  if (int32_t rc = check_rows("router", router, false)) return rc;
  if (int32_t rc = check_weights(weights)) return rc;
  if (int32_t rc = check_rows("y", y, true)) return rc;
  if (int32_t rc = check_activation(activation, GINEX_ACT_NONE)) return rc;
  if (int32_t rc = check_same("x", x, "router", router)) return rc;
  if (x->type != weights->type || x->type != y->type) return fail(GINEX_ERR_ARG, "x, weights and y differ in type");
  if (int32_t rc = check_few(x->rows, top, weights->experts, weights->width, weights->out)) return rc;
  if (x->width != weights->width)
    return fail(GINEX_ERR_ARG, "x is %lld wide, the weights take %lld", (long long)x->width, (long long)weights->width);
  if (y->width != weights->out)
    return fail(GINEX_ERR_ARG, "y is %lld wide, the weights give %lld", (long long)y->width, (long long)weights->out);
  if (y->rows != x->rows) return fail(GINEX_ERR_ARG, "x has %lld rows, y %lld", (long long)x->rows, (long long)y->rows);
  if (router->rows != weights->experts)
    return fail(GINEX_ERR_ARG, "router has %lld rows for %d experts", (long long)router->rows, weights->experts);
  if (int32_t rc = check_vector("bias", bias, x->type)) return rc;
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(GINEX_ERR_ARG, "workspace: null or misaligned");
  const FewSpace space = few_space(ws, x->rows, top, weights->out);
  if (ws_bytes < space.bytes) return fail(GINEX_ERR_WORKSPACE, "workspace: need %zu bytes, got %zu", space.bytes, ws_bytes);
  if (x->rows == 0) return GINEX_OK;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(x->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const int32_t rows = (int32_t)x->rows, pairs = rows * top;
    const int32_t tiles = (int32_t)ceil_div(weights->out, WAVE_COLUMNS);
    // One row that has one or two experts in one launch, where what a workgroup reads of router and weights is little: 1024 ->
    // 1024 of 64 experts, one a row, f16 9.8 us instead of 14.1, two 12.7 (14.3), 256 -> 256 of 8, two a row, 7.5 (11.2); but
    // 2048 -> 2048 of 32, two a row, 23.4 (22.3), and eight a row of 256 -> 256 18.0 (15.7).
    const int64_t bytes = sizeof(T), of_one = (weights->experts + (int64_t)top * WAVE_COLUMNS) * weights->width * bytes;
    if (rows == 1 && top <= MOST_OF_ONE && of_one <= 384 * 1024) {
      return with_each(weights->experts, [&](auto of_lane) -> int32_t {
        constexpr int EACH = decltype(of_lane)::value;
        const auto one = weights->turned ? k_few_one<T, true, EACH> : k_few_one<T, false, EACH>;
        hipLaunchKernelGGL(one, dim3((unsigned)tiles), dim3(ROUTE_THREADS), 0, st, read_rows<T>(x), read_rows<T>(router),
                           weights->experts, top, Width::of<T>(x->width), weights_of<T>(weights),
                           static_cast<const T*>(bias), Width::of<T>(weights->out), activation, static_cast<T*>(y->data));
        GINEX_LAUNCH_CHECK();
        return GINEX_OK;
      });
    }
    const int32_t routed = with_each(weights->experts, [&](auto of_lane) -> int32_t {
      hipLaunchKernelGGL((k_few_route<T, decltype(of_lane)::value>), dim3((unsigned)rows), dim3(ROUTE_THREADS), 0, st,
                         read_rows<T>(x), read_rows<T>(router), weights->experts, top, Width::of<T>(x->width), space.plan, tiles);
      GINEX_LAUNCH_CHECK();
      return GINEX_OK;
    });
    if (routed) return routed;
    const int32_t most = pairs < weights->experts ? pairs : weights->experts;
    return with_waves(weights->width, sizeof(T), (int64_t)tiles * most, [&](auto waves) -> int32_t {
      constexpr int WAVES = decltype(waves)::value;
      const auto kernel = weights->turned ? k_few_experts<T, true, WAVES> : k_few_experts<T, false, WAVES>;
      const dim3 grid((unsigned)tiles, (unsigned)most, (unsigned)ceil_div(rows, 16));
      hipLaunchKernelGGL(kernel, grid, dim3(WAVES * WAVE), 0, st, read_rows<T>(x), pairs, top, rows, weights_of<T>(weights),
                         (int32_t)(most < weights->experts), static_cast<const T*>(bias), (int32_t)weights->width, Width::of<T>(weights->out), activation,
                         space.plan, rows_of<T>(y));
      GINEX_LAUNCH_CHECK();
      return GINEX_OK;
    });
  });
}
