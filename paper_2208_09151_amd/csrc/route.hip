// Pairs (row, choice) sorted by expert: a stable counting sort with at most 1025 keys.
//
//   slot(p) = offset(e(p)) + #{q < p : e(q) = e(p)},  offset(e) = sum over e' < e of min(count(e'), capacity)
//
// A wave owns a run of consecutive pairs, 64 at a time, all of them in registers.  Lanes of the same expert
// find each other by ballots over the bits of the expert's number, so a pair's rank among them is a
// popcount, and the run's count of the expert so far (in LDS, a row of counters per wave) gives the rest:
// no atomic decides a place, and equal inputs give equal slots.
//
// Bound by launches and their latencies: up to 8192 pairs one workgroup in one launch (up to 512 pairs 2.3 us,
// 7000 7.8), else the tiles' counts and the places, in which every workgroup adds up the counts of the tiles
// itself (354 000 pairs 4.8 + 7.3 us, 1.64 M 5.8 + 18 in 32 experts: 401 workgroups that read 51 KB of counts each, where
// the pairs' bytes would take 4); with a scan between them, five launches, 1.64 M pairs took 35 us in all and 152 000 20
// instead of 15.
#include "primitives.hpp"
#include "train.hpp"

namespace ginex {
namespace {

constexpr int WAVES = 8;
constexpr int THREADS = WAVES * WAVE;
constexpr int TILE_KEYS = 8;                    // pairs of a lane
constexpr int ONE = THREADS * 16;               // up to here one workgroup does it all in one launch
constexpr int TILE = THREADS * TILE_KEYS;
// Up to here the tiles' counts are added up by every workgroup, which reads tiles x experts of them, beyond it they are
// scanned, three launches more.  Adding and scanning, us of a call, by tiles and experts: 2048 x 8 50 and 45, 512 x 32
// 24 and 27, 1024 x 32 42 and 36, 128 x 128 21 and 23, 256 x 128 31 and 26, 16 x 1024 21 and 25, 64 x 1024 45 and 26,
// 1024 x 1024 1063 and 82.
constexpr int64_t MOST_COUNTS = 1 << 14;
constexpr int64_t MOST_TILES = 1024;

// A lane's pair: its expert (`experts` for none), its rank among the lanes with the same one, and how many they are.
struct Place {
  uint32_t packed;
  __device__ __forceinline__ Place(uint32_t expert, uint64_t same) {
    const uint64_t below = ((uint64_t)1 << lane_id()) - 1;
    packed = expert | (uint32_t)__popcll(same & below) << 16 | (uint32_t)__popcll(same) << 24;
  }
  Place() = default;
  __device__ __forceinline__ uint32_t expert() const { return packed & 0xFFFF; }
  __device__ __forceinline__ uint32_t rank() const { return packed >> 16 & 0xFF; }
  __device__ __forceinline__ uint32_t lanes() const { return packed >> 24; }
};

// Reads a wave's run and counts it: counts [experts + 1] of this wave, zero before.  The rounds of 64 go through the bits
// together, and nothing waits for LDS: one round after the other took three times as long.
template <typename Key, int KEYS>
__device__ __forceinline__ void count_run(const Key* __restrict__ chosen, int64_t first, int64_t pairs, uint32_t experts,
                                          int bits, uint32_t* counts, Place (&places)[KEYS]) {
  Key e[KEYS];
  uint64_t same[KEYS];
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    const int64_t p = first + i * WAVE + lane_id();
    e[i] = p < pairs ? chosen[p] : (Key)-1;
  }
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    e[i] = e[i] >= 0 && e[i] < (Key)experts ? e[i] : (Key)experts;
    same[i] = ~(uint64_t)0;
  }
  for (int b = 0; b < bits; ++b) {
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
      const bool set = ((uint32_t)e[i] >> b) & 1;
      const uint64_t lanes = __ballot(set);
      same[i] &= set ? lanes : ~lanes;
    }
  }
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    places[i] = Place((uint32_t)e[i], same[i]);
    if (places[i].rank() == 0) atomicAdd(&counts[(uint32_t)e[i]], places[i].lanes());
  }
}

// ranks[e]: pairs of expert e in front of the run; starts[e]: its first slot.  A wave's LDS accesses are carried out in
// their order, so a round reads what the rounds before it have added without waiting for them.
template <int KEYS>
__device__ __forceinline__ void place_run(const Place (&places)[KEYS], int64_t first, int64_t pairs, uint32_t experts,
                                          uint32_t capacity, Divisor top, uint32_t* ranks, const uint32_t* starts,
                                          int32_t* __restrict__ slot, int32_t* __restrict__ source) {
  uint32_t before[KEYS], start[KEYS];
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    before[i] = ranks[places[i].expert()];
    __builtin_amdgcn_wave_barrier();
    if (places[i].rank() == 0) atomicAdd(&ranks[places[i].expert()], places[i].lanes());
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int i = 0; i < KEYS; ++i) start[i] = starts[places[i].expert() < experts ? places[i].expert() : 0];
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    const int64_t p = first + i * WAVE + lane_id();
    if (p >= pairs) break;
    const uint32_t rank = before[i] + places[i].rank();
    const bool kept = places[i].expert() < experts && rank < capacity;
    const int32_t s = kept ? (int32_t)(start[i] + rank) : -1;
    slot[p] = s;
    if (kept) source[s] = (int32_t)top.of((uint32_t)p);
  }
}

// From counts[w][e] of the waves' runs, the pairs of e in front of them and those of e in all: counts[w][e] becomes the
// pairs of e in front of run w, starts[e] its first slot; returns the number of slots.
template <typename InFront, typename All>
__device__ __forceinline__ uint32_t runs_to_ranks(uint32_t* counts, uint32_t* starts, uint32_t experts, uint32_t capacity,
                                                  uint32_t* smem, InFront in_front, All all) {
  uint32_t done = 0;
  for (uint32_t e0 = 0; e0 < experts; e0 += THREADS) {
    const uint32_t e = e0 + threadIdx.x;
    uint32_t sum = 0;
    if (e < experts) {
      uint32_t rank = in_front(e);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const uint32_t n = counts[w * (experts + 1) + e];
        counts[w * (experts + 1) + e] = rank;
        rank += n;
      }
      sum = all(e, rank);
    }
    uint32_t total;
    const uint32_t first = block_exclusive_scan<uint32_t, THREADS>(sum < capacity ? sum : capacity, smem, total);
    if (e < experts) starts[e] = done + first;
    done += total;
  }
  return done;
}

template <typename Key, int KEYS>
__global__ __launch_bounds__(THREADS) void k_route_one(const Key* __restrict__ chosen, int64_t pairs, uint32_t experts,
                                                       int bits, uint32_t capacity, Divisor top,
                                                       int64_t* __restrict__ offsets, int32_t* __restrict__ slot,
                                                       int32_t* __restrict__ source) {
  extern __shared__ uint32_t dynamic[];
  __shared__ uint32_t smem[WAVES + 1];
  uint32_t* const counts = dynamic;                              // [WAVES][experts + 1]
  uint32_t* const starts = dynamic + WAVES * (experts + 1);      // [experts]
  for (uint32_t i = threadIdx.x; i < WAVES * (experts + 1); i += THREADS) counts[i] = 0;
  __syncthreads();
  const int w = threadIdx.x / WAVE;
  // (as even runs as whole rounds of 64 allow)
  const int64_t run = (pairs + THREADS - 1) / THREADS * WAVE;
  const int64_t first = w * run, last = first + run < pairs ? first + run : pairs;
  uint32_t* const mine = counts + w * (experts + 1);
  Place places[KEYS];
  count_run(chosen, first, last, experts, bits, mine, places);
  __syncthreads();
  const uint32_t kept = runs_to_ranks(counts, starts, experts, capacity, smem, [](uint32_t) { return 0u; },
                                      [](uint32_t, uint32_t sum) { return sum; });
  __syncthreads();
  place_run(places, first, last, experts, capacity, top, mine, starts, slot, source);
  for (uint32_t e = threadIdx.x; e < experts; e += THREADS) offsets[e] = starts[e];
  if (threadIdx.x == 0) offsets[experts] = kept;
  for (int64_t s = kept + threadIdx.x; s < pairs; s += THREADS) source[s] = -1;
}

// hist: [tiles][experts + 1], or (SCANNED) [experts + 1][tiles].
template <typename Key, bool SCANNED>
__global__ __launch_bounds__(THREADS) void k_route_count(const Key* __restrict__ chosen, int64_t pairs, uint32_t experts,
                                                         uint32_t* __restrict__ hist) {
  extern __shared__ uint32_t counts[];     // [experts + 1]
  for (uint32_t e = threadIdx.x; e <= experts; e += THREADS) counts[e] = 0;
  __syncthreads();
  Key e[TILE_KEYS];
#pragma unroll
  for (int i = 0; i < TILE_KEYS; ++i) {
    const int64_t p = (int64_t)blockIdx.x * TILE + i * THREADS + threadIdx.x;
    e[i] = p < pairs ? chosen[p] : (Key)-1;
  }
#pragma unroll
  for (int i = 0; i < TILE_KEYS; ++i) atomicAdd(&counts[e[i] >= 0 && e[i] < (Key)experts ? (uint32_t)e[i] : experts], 1u);
  __syncthreads();
  for (uint32_t e = threadIdx.x; e <= experts; e += THREADS)
    hist[SCANNED ? (int64_t)e * gridDim.x + blockIdx.x : (int64_t)blockIdx.x * (experts + 1) + e] = counts[e];
}

template <typename Key, bool SCANNED>
__global__ __launch_bounds__(THREADS) void k_route_place(const Key* __restrict__ chosen, int64_t pairs, uint32_t experts,
                                                         int bits, uint32_t capacity, Divisor top,
                                                         const uint32_t* __restrict__ hist, int64_t* __restrict__ offsets,
                                                         int32_t* __restrict__ slot, int32_t* __restrict__ source) {
  extern __shared__ uint32_t dynamic[];
  __shared__ uint32_t smem[WAVES + 1];
  uint32_t* const counts = dynamic;                              // [WAVES][experts + 1]
  uint32_t* const starts = counts + WAVES * (experts + 1);       // [experts]
  uint32_t* const in_front = starts + experts;                   // [experts], of the tiles in front of this one
  uint32_t* const all = in_front + experts;                      // [experts]
  for (uint32_t i = threadIdx.x; i < (WAVES + 3) * (experts + 1) - 3; i += THREADS) counts[i] = 0;
  __syncthreads();
  const int w = threadIdx.x / WAVE;
  const int64_t tiles = gridDim.x, first = (int64_t)blockIdx.x * TILE + w * (TILE / WAVES);
  uint32_t* const mine = counts + w * (experts + 1);
  Place places[TILE_KEYS];
  count_run(chosen, first, pairs, experts, bits, mine, places);
  if (!SCANNED) {
    // `lanes` threads beside each other have an expert each, the groups of them every so many tiles
    uint32_t lanes = 1;
    while (lanes < experts && lanes < THREADS) lanes *= 2;
    const uint32_t groups = THREADS / lanes;
    for (uint32_t e = threadIdx.x % lanes; e < experts; e += lanes) {
      uint32_t mine_in_front = 0, mine_all = 0;
#pragma unroll 8
      for (uint32_t q = threadIdx.x / lanes; q < tiles; q += groups) {
        const uint32_t n = hist[q * (experts + 1) + e];
        mine_all += n;
        mine_in_front += q < blockIdx.x ? n : 0;
      }
      atomicAdd(&in_front[e], mine_in_front);
      atomicAdd(&all[e], mine_all);
    }
  } else {
    for (uint32_t e = threadIdx.x; e < experts; e += THREADS) {
      const uint32_t begin = hist[e * tiles];
      in_front[e] = hist[e * tiles + blockIdx.x] - begin;
      all[e] = hist[(e + 1) * tiles] - begin;
    }
  }
  __syncthreads();
  const uint32_t kept = runs_to_ranks(counts, starts, experts, capacity, smem, [&](uint32_t e) { return in_front[e]; },
                                      [&](uint32_t e, uint32_t) { return all[e]; });
  __syncthreads();
  place_run(places, first, pairs, experts, capacity, top, mine, starts, slot, source);
  if (blockIdx.x == 0) {
    for (uint32_t e = threadIdx.x; e < experts; e += THREADS) offsets[e] = starts[e];
    if (threadIdx.x == 0) offsets[experts] = kept;
  }
  for (int64_t s = (int64_t)kept + (int64_t)blockIdx.x * THREADS + threadIdx.x; s < pairs; s += tiles * THREADS) source[s] = -1;
}

struct RouteSpace {
  uint32_t* hist;
  uint32_t* scratch;
};

RouteSpace route_space(Arena& a, int64_t pairs, int32_t experts) {
  const int64_t counters = pairs > ONE ? ((int64_t)experts + 1) * ceil_div(pairs, TILE) : 0;
  RouteSpace s;
  s.hist = a.take<uint32_t>(counters);
  s.scratch = a.take<uint32_t>(scan_scratch_elems(counters));
  a.take<char>(256);       // (a query never answers 0: that is an error)
  return s;
}

template <typename Key, bool SCANNED>
int32_t route_tiles(const Key* chosen, uint32_t experts, int bits, uint32_t most, const ginex_routing_t* out,
                    const RouteSpace& s, hipStream_t st) {
  const int64_t pairs = out->rows * out->top, tiles = ceil_div(pairs, TILE);
  const size_t counters = ((size_t)experts + 1) * sizeof(uint32_t);
  hipLaunchKernelGGL((k_route_count<Key, SCANNED>), dim3((unsigned)tiles), dim3(THREADS), counters, st, chosen, pairs, experts,
                     s.hist);
  GINEX_LAUNCH_CHECK();
  if (SCANNED) GINEX_HIP(exclusive_scan_inplace(s.hist, (experts + 1) * tiles, s.scratch, st));
  hipLaunchKernelGGL((k_route_place<Key, SCANNED>), dim3((unsigned)tiles), dim3(THREADS), (WAVES + 3) * counters, st, chosen,
                     pairs, experts, bits, most, Divisor((uint32_t)out->top), s.hist, out->offsets, out->slot, out->source);
  GINEX_LAUNCH_CHECK();
  return GINEX_OK;
}

template <typename Key>
int32_t route_pairs(const Key* chosen, int64_t capacity, const ginex_routing_t* out, void* ws, hipStream_t st) {
  const int64_t pairs = out->rows * out->top;
  const uint32_t experts = (uint32_t)out->experts;
  const uint32_t most = capacity < 0 || capacity > INT32_MAX ? (uint32_t)INT32_MAX : (uint32_t)capacity;
  int bits = 0;
  while ((experts >> bits) != 0) ++bits;       // the numbers 0 .. experts
  if (pairs <= ONE) {
    const size_t lds = (WAVES * ((size_t)experts + 1) + experts) * sizeof(uint32_t);
    // (lanes go through all the rounds they have registers for: 2.6 us for up to 512 pairs, 5.6 with 16 rounds)
    const auto kernel = pairs <= THREADS ? k_route_one<Key, 1> : pairs <= 4 * THREADS ? k_route_one<Key, 4> : k_route_one<Key, 16>;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(THREADS), lds, st, chosen, pairs, experts, bits, most,
                       Divisor((uint32_t)out->top), out->offsets, out->slot, out->source);
    GINEX_LAUNCH_CHECK();
    return GINEX_OK;
  }
  Arena a(ws);
  const RouteSpace s = route_space(a, pairs, out->experts);
  const int64_t tiles = ceil_div(pairs, TILE);
  return tiles <= MOST_TILES && tiles * experts <= MOST_COUNTS
             ? route_tiles<Key, false>(chosen, experts, bits, most, out, s, st)
             : route_tiles<Key, true>(chosen, experts, bits, most, out, s, st);
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
