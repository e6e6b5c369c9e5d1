// Pairs (row, choice) sorted by expert: a stable counting sort with at most 1025 keys.
//
//   slot(p) = offset(e(p)) + #{q < p : e(q) = e(p)},  offset(e) = sum over e' < e of min(count(e'), capacity)
//
// A wave owns a run of consecutive pairs, 64 at a time.  Lanes of the same expert find each other by
// ballots over the bits of the expert's number, so a pair's rank among them is a popcount, and the run's
// count of the expert so far (in LDS, a row of counters per wave) gives the rest: no atomic decides a
// place, and equal inputs give equal slots.
#include "primitives.hpp"
#include "train.hpp"

namespace ginex {
namespace {

constexpr int TILE_THREADS = 256;
constexpr int TILE_WAVES = TILE_THREADS / WAVE;
constexpr int RUN = 1024;                       // pairs of a wave
constexpr int TILE = TILE_WAVES * RUN;
constexpr int ONE_THREADS = 512;
constexpr int ONE_WAVES = ONE_THREADS / WAVE;
// Up to here one workgroup does it all in one launch.
constexpr int64_t ONE_PAIRS = 8192;

// The expert of pair p, or `experts` for none.
template <typename Key>
__device__ __forceinline__ uint32_t expert_of(const Key* __restrict__ chosen, int64_t p, int64_t end, uint32_t experts) {
  if (p >= end) return experts;
  const Key e = chosen[p];
  return e >= 0 && e < (Key)experts ? (uint32_t)e : experts;
}

// The lanes whose value is this lane's.
__device__ __forceinline__ uint64_t same_lanes(uint32_t value, int bits) {
  uint64_t same = ~(uint64_t)0;
  for (int b = 0; b < bits; ++b) {
    const bool set = (value >> b) & 1;
    const uint64_t lanes = __ballot(set);
    same &= set ? lanes : ~lanes;
  }
  return same;
}

template <typename Key>
__device__ __forceinline__ void count_run(const Key* __restrict__ chosen, int64_t first, int64_t last, int64_t end,
                                          uint32_t experts, uint32_t* counts) {
  for (int64_t p = first + lane_id(); p < last; p += WAVE) atomicAdd(&counts[expert_of(chosen, p, end, experts)], 1u);
}

// Places the pairs of a run.  ranks[e]: pairs of expert e in front of the run; starts[e]: its first slot.
template <typename Key>
__device__ __forceinline__ void place_run(const Key* __restrict__ chosen, int64_t first, int64_t last, int64_t end,
                                          uint32_t experts, int bits, uint32_t capacity, Divisor top,
                                          uint32_t* ranks, const uint32_t* starts, int32_t* __restrict__ slot,
                                          int32_t* __restrict__ source) {
  const uint64_t below = ((uint64_t)1 << lane_id()) - 1;
  for (int64_t at = first; at < last; at += WAVE) {
    const int64_t p = at + lane_id();
    const uint32_t e = expert_of(chosen, p, end, experts);
    const uint64_t same = same_lanes(e, bits);
    const uint32_t before = ranks[e];
    __builtin_amdgcn_wave_barrier();
    if ((same & below) == 0) ranks[e] = before + (uint32_t)__popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (p < end) {
      const uint32_t rank = before + (uint32_t)__popcll(same & below);
      const bool kept = e < experts && rank < capacity;
      const int32_t s = kept ? (int32_t)(starts[e] + rank) : -1;
      slot[p] = s;
      if (kept) source[s] = (int32_t)top.of((uint32_t)p);
    }
  }
}

// From counts[w][e] of W runs: counts[w][e] becomes the pairs of e in front of run w, starts[e] its first slot;
// returns the number of slots.
template <int THREADS, int W>
__device__ __forceinline__ uint32_t runs_to_ranks(uint32_t* counts, uint32_t* starts, uint32_t experts,
                                                  uint32_t capacity, uint32_t* smem) {
  uint32_t done = 0;
  for (uint32_t e0 = 0; e0 < experts; e0 += THREADS) {
    const uint32_t e = e0 + threadIdx.x;
    uint32_t sum = 0;
    if (e < experts) {
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const uint32_t n = counts[w * (experts + 1) + e];
        counts[w * (experts + 1) + e] = sum;
        sum += n;
      }
    }
    uint32_t total;
    const uint32_t first = block_exclusive_scan<uint32_t, THREADS>(sum < capacity ? sum : capacity, smem, total);
    if (e < experts) starts[e] = done + first;
    done += total;
  }
  return done;
}

template <typename Key>
__global__ __launch_bounds__(ONE_THREADS) void k_route_one(const Key* __restrict__ chosen, int64_t pairs, uint32_t experts,
                                                           int bits, uint32_t capacity, Divisor top,
                                                           int64_t* __restrict__ offsets, int32_t* __restrict__ slot,
                                                           int32_t* __restrict__ source) {
  extern __shared__ uint32_t dynamic[];
  __shared__ uint32_t smem[ONE_WAVES + 1];
  uint32_t* const counts = dynamic;                                  // [ONE_WAVES][experts + 1]
  uint32_t* const starts = dynamic + ONE_WAVES * (experts + 1);      // [experts]
  for (uint32_t i = threadIdx.x; i < ONE_WAVES * (experts + 1); i += ONE_THREADS) counts[i] = 0;
  __syncthreads();
  const int w = threadIdx.x / WAVE;
  const int64_t run = (pairs + ONE_THREADS - 1) / ONE_THREADS * WAVE;
  const int64_t first = w * run, last = first + run < pairs ? first + run : pairs;
  uint32_t* const mine = counts + w * (experts + 1);
  count_run(chosen, first, last, pairs, experts, mine);
  __syncthreads();
  const uint32_t kept = runs_to_ranks<ONE_THREADS, ONE_WAVES>(counts, starts, experts, capacity, smem);
  __syncthreads();
  place_run(chosen, first, last, pairs, experts, bits, capacity, top, mine, starts, slot, source);
  for (uint32_t e = threadIdx.x; e < experts; e += ONE_THREADS) offsets[e] = starts[e];
  if (threadIdx.x == 0) offsets[experts] = kept;
  for (int64_t s = kept + threadIdx.x; s < pairs; s += ONE_THREADS) source[s] = -1;
}

template <typename Key>
__global__ __launch_bounds__(TILE_THREADS) void k_route_count(const Key* __restrict__ chosen, int64_t pairs,
                                                              uint32_t experts, uint32_t* __restrict__ hist) {
  extern __shared__ uint32_t counts[];     // [experts + 1]
  for (uint32_t e = threadIdx.x; e <= experts; e += TILE_THREADS) counts[e] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * TILE;
  const int64_t last = first + TILE < pairs ? first + TILE : pairs;
  for (int64_t p = first + threadIdx.x; p < last; p += TILE_THREADS)
    atomicAdd(&counts[expert_of(chosen, p, pairs, experts)], 1u);
  __syncthreads();
  for (uint32_t e = threadIdx.x; e <= experts; e += TILE_THREADS) hist[(int64_t)e * gridDim.x + blockIdx.x] = counts[e];
}

// hist: scanned, expert after expert, tile after tile.
template <typename Key>
__global__ __launch_bounds__(TILE_THREADS) void k_route_place(const Key* __restrict__ chosen, int64_t pairs,
                                                              uint32_t experts, int bits, uint32_t capacity, Divisor top,
                                                              const uint32_t* __restrict__ hist,
                                                              int64_t* __restrict__ offsets, int32_t* __restrict__ slot,
                                                              int32_t* __restrict__ source) {
  extern __shared__ uint32_t dynamic[];
  __shared__ uint32_t smem[TILE_WAVES + 1];
  uint32_t* const counts = dynamic;                                   // [TILE_WAVES][experts + 1]
  uint32_t* const starts = dynamic + TILE_WAVES * (experts + 1);      // [experts]
  for (uint32_t i = threadIdx.x; i < TILE_WAVES * (experts + 1); i += TILE_THREADS) counts[i] = 0;
  __syncthreads();
  const int w = threadIdx.x / WAVE;
  const int64_t tiles = gridDim.x;
  const int64_t first = (int64_t)blockIdx.x * TILE + w * RUN;
  const int64_t last = first + RUN < pairs ? first + RUN : pairs;
  uint32_t* const mine = counts + w * (experts + 1);
  count_run(chosen, first, last, pairs, experts, mine);
  __syncthreads();
  uint32_t kept = 0;
  for (uint32_t e0 = 0; e0 < experts; e0 += TILE_THREADS) {
    const uint32_t e = e0 + threadIdx.x;
    uint32_t all = 0;
    if (e < experts) {
      const uint32_t begin = hist[e * tiles];
      all = hist[(e + 1) * tiles] - begin;
      uint32_t rank = hist[e * tiles + blockIdx.x] - begin;
#pragma unroll
      for (int v = 0; v < TILE_WAVES; ++v) {
        const uint32_t n = counts[v * (experts + 1) + e];
        counts[v * (experts + 1) + e] = rank;
        rank += n;
      }
    }
    uint32_t total;
    const uint32_t start = block_exclusive_scan<uint32_t, TILE_THREADS>(all < capacity ? all : capacity, smem, total);
    if (e < experts) {
      starts[e] = kept + start;
      if (blockIdx.x == 0) offsets[e] = kept + start;
    }
    kept += total;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) offsets[experts] = kept;
  __syncthreads();
  place_run(chosen, first, last, pairs, experts, bits, capacity, top, mine, starts, slot, source);
  for (int64_t s = (int64_t)kept + (int64_t)blockIdx.x * TILE_THREADS + threadIdx.x; s < pairs; s += tiles * TILE_THREADS)
    source[s] = -1;
}

struct RouteSpace {
  uint32_t* hist;
  uint32_t* scratch;
};

RouteSpace route_space(Arena& a, int64_t pairs, int32_t experts) {
  const int64_t counters = pairs > ONE_PAIRS ? ((int64_t)experts + 1) * ceil_div(pairs, TILE) : 0;
  RouteSpace s;
  s.hist = a.take<uint32_t>(counters);
  s.scratch = a.take<uint32_t>(scan_scratch_elems(counters));
  a.take<char>(256);       // (a query never answers 0: that is an error)
  return s;
}

template <typename Key>
int32_t route_pairs(const Key* chosen, int64_t capacity, const ginex_routing_t* out, void* ws, hipStream_t st) {
  const int64_t pairs = out->rows * out->top;
  const uint32_t experts = (uint32_t)out->experts;
  const uint32_t most = capacity < 0 || capacity > INT32_MAX ? (uint32_t)INT32_MAX : (uint32_t)capacity;
  const Divisor top((uint32_t)out->top);
  int bits = 0;
  while ((experts >> bits) != 0) ++bits;       // the numbers 0 .. experts
  if (pairs <= ONE_PAIRS) {
    const size_t lds = (ONE_WAVES * ((size_t)experts + 1) + experts) * sizeof(uint32_t);
    hipLaunchKernelGGL(k_route_one<Key>, dim3(1), dim3(ONE_THREADS), lds, st, chosen, pairs, experts, bits, most, top,
                       out->offsets, out->slot, out->source);
    GINEX_LAUNCH_CHECK();
    return GINEX_OK;
  }
  Arena a(ws);
  const RouteSpace s = route_space(a, pairs, out->experts);
  const int64_t tiles = ceil_div(pairs, TILE);
  hipLaunchKernelGGL(k_route_count<Key>, dim3((unsigned)tiles), dim3(TILE_THREADS), ((size_t)experts + 1) * sizeof(uint32_t),
                     st, chosen, pairs, experts, s.hist);
  GINEX_LAUNCH_CHECK();
  GINEX_HIP(exclusive_scan_inplace(s.hist, (experts + 1) * tiles, s.scratch, st));
  const size_t lds = (TILE_WAVES * ((size_t)experts + 1) + experts) * sizeof(uint32_t);
  hipLaunchKernelGGL(k_route_place<Key>, dim3((unsigned)tiles), dim3(TILE_THREADS), lds, st, chosen, pairs, experts, bits,
                     most, top, s.hist, out->offsets, out->slot, out->source);
  GINEX_LAUNCH_CHECK();
  return GINEX_OK;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

extern "C" size_t ginex_route_workspace_bytes(int64_t rows, int32_t top, int32_t experts) {
  if (check_pairs(rows, top, experts) != GINEX_OK) return 0;
  Arena a(nullptr);
  route_space(a, rows * top, experts);
  return a.used;
}

extern "C" int32_t ginex_route(const void* chosen, int32_t chosen_64, int64_t capacity, const ginex_routing_t* out,
                               void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_routing(out)) return rc;
  if (out->rows > 0 && !chosen) return fail(GINEX_ERR_ARG, "route: null experts");
  if (reinterpret_cast<uintptr_t>(chosen) % (chosen_64 ? 8 : 4)) return fail(GINEX_ERR_ARG, "route: misaligned experts");
  const size_t need = ginex_route_workspace_bytes(out->rows, out->top, out->experts);
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(GINEX_ERR_ARG, "route: null or misaligned workspace (256 bytes)");
  if (ws_bytes < need) return fail(GINEX_ERR_WORKSPACE, "route: workspace %zu bytes, need %zu", ws_bytes, need);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return chosen_64 ? route_pairs(static_cast<const int64_t*>(chosen), capacity, out, ws, st)
                   : route_pairs(static_cast<const int32_t*>(chosen), capacity, out, ws, st);
}
