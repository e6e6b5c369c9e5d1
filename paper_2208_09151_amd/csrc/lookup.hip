// Lookup of rows of a table, and the table's gradient:
//
//   out[i] = scale table[ids[i]],   dtable[v] = scale * sum over the i with ids[i] = v of dy[i]
//
// Both are bound by HBM.  The gradient adds nothing up by atomics, whose order would be another in every run: (id, position)
// pairs are sorted by id, stable, and the sorted positions are cut into runs.  A group of lanes, one for every chunk of 16
// bytes of a row, goes through a run; what runs beside each other share is joined in LDS.  Ids that begin and end in a
// workgroup's runs are written to the table's gradient; of others it leaves parts in the workspace, at most two.  A second launch
// adds the parts of an id up in their order, and clears the rows that no id names.
//
// 1 000 000 ids of 177 000 rows x 128 f32: 153 us (4.0 TB/s: rows read here and there, in part from the caches), and 126 us for the
// runs, 25 for the second launch and 75 for the sort.
#include "layers.hpp"
#include "primitives.hpp"

namespace ginex {
namespace {

constexpr int THREADS = 256;
constexpr int LONG = 16;          // parts of an id that one group adds up; of more the workgroup does

// ids as sorted by: what is no row of the table comes last.
template <typename Id>
struct IdsWithPositions {
  const Id* ids;
  uint32_t rows;
  __device__ __forceinline__ uint64_t operator()(int64_t j) const {
    const uint64_t id = (uint64_t)(int64_t)ids[j];
    return (id < rows ? id : rows) << 32 | (uint64_t)j;
  }
};

// Few ids: the place of one is the number of those in front of it, which a workgroup counts for 64 of them, a lane each, its waves
// for a part of all ids each.  It is one launch, where sorting by digits takes three or more for every one (us of a whole gradient, with
// it and by digits: 64 ids of 1000 rows x 64 12.4 and 27.0, 4000 of 100 000 x 128 34 and 59, 8000 x 64 38 and 58, but 16 000 of 100 rows
// 46 and 30).
constexpr int PLACE_THREADS = 1024, PLACE_WAVES = PLACE_THREADS / WAVE, PLACE_STEP = 4096;
constexpr int64_t MOST_PLACED = 8192;

template <typename Id>
__global__ __launch_bounds__(PLACE_THREADS) void k_lookup_places(IdsWithPositions<Id> in, int32_t n, uint64_t* __restrict__ sorted,
                                                                 uint32_t* __restrict__ named, int64_t named_words) {
  __shared__ __align__(16) uint32_t all[PLACE_STEP];
  __shared__ uint32_t room[PLACE_WAVES][WAVE];
  const int lane = lane_id(), wave = threadIdx.x / WAVE;
  for (int64_t i = (int64_t)blockIdx.x * PLACE_THREADS + threadIdx.x; i < named_words; i += (int64_t)gridDim.x * PLACE_THREADS)
    named[i] = 0;
  if ((int64_t)blockIdx.x * WAVE >= n) return;          // (one that only clears)
  const int32_t mine = blockIdx.x * WAVE + lane;
  const uint64_t key = in(mine < n ? mine : n - 1);
  uint32_t count = 0;
  for (int32_t first = 0; first < n; first += PLACE_STEP) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PLACE_STEP / PLACE_THREADS; ++i) {
      const int32_t j = first + i * PLACE_THREADS + threadIdx.x;
      all[i * PLACE_THREADS + threadIdx.x] = j < n ? (uint32_t)(in(j) >> 32) : ~0u;         // (behind all)
    }
    __syncthreads();
    const int32_t left = n - first < PLACE_STEP ? n - first : PLACE_STEP;
    const int32_t each = ((left + 4 * PLACE_WAVES - 1) / (4 * PLACE_WAVES)) * 4;
    const int32_t from = wave * each, to = from + each < PLACE_STEP ? from + each : PLACE_STEP;
#pragma unroll 4
    for (int32_t j = from; j < to; j += 4) {
      const words4 id = *reinterpret_cast<const words4*>(&all[j]);
#pragma unroll
      for (int k = 0; k < 4; ++k) count += ((uint64_t)id[k] << 32 | (uint32_t)(first + j + k)) < key ? 1 : 0;
    }
  }
  room[wave][lane] = count;
  __syncthreads();
  if (wave > 0 || mine >= n) return;
  uint32_t place = 0;
  for (int w = 0; w < PLACE_WAVES; ++w) place += room[w][lane];
  sorted[place] = key;
}

// U chunks a thread, THREADS apart; ids first, then rows, then stores.
template <typename T, typename Id>
__global__ __launch_bounds__(THREADS) void k_lookup(RowsOf<const T> table, int64_t rows, const Id* __restrict__ ids,
                                                    RowsOf<T> out, int64_t first, uint32_t chunks, Divisor cpr,
                                                    Width width, float scale) {
  constexpr int N = Chunk<T>::N, U = 4;
  int32_t c[U];
  int64_t i[U], id[U];
  const uint32_t t0 = blockIdx.x * (U * THREADS) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t t = t0 + u * THREADS;
    t = t < chunks ? t : chunks - 1;
    const uint32_t row = cpr.of(t);
    c[u] = (int32_t)(t - row * cpr.d) * N;
    i[u] = first + row;
    id[u] = ids[i[u]];
  }
  ChunkWords<T> v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // (a table of no rows may have no memory)
    if (rows > 0) v[u] = load_words(table.at((uint64_t)id[u] < (uint64_t)rows ? id[u] : 0), c[u], width);
    else v[u].words = words4{0, 0, 0, 0};
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (t0 + u * THREADS >= chunks) break;
    float f[N];
#pragma unroll
    for (int n = 0; n < N; ++n) f[n] = (uint64_t)id[u] < (uint64_t)rows ? scale * (float)v[u].wide[n] : 0.f;
    store_chunk(out.at(i[u]), c[u], width, f);
  }
}

__device__ __forceinline__ uint32_t id_of(uint64_t word) { return (uint32_t)(word >> 32); }

// N f32 sums in the workspace, from column c on.
template <int N>
__device__ __forceinline__ void store_part(float* to, int32_t c, Width width, const float (&v)[N]) {
#pragma unroll
  for (int n = 0; n < N; n += 4) {
    ChunkWords<float> u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.wide[i] = v[n + i];
    if (c + n < width.width) store_words<true>(to, c + n, width, u);
  }
}
template <int N>
__device__ __forceinline__ void load_part(const float* from, int32_t c, Width width, ChunkWords<float> (&v)[N / 4]) {
#pragma unroll
  for (int n = 0; n < N; n += 4) v[n / 4] = load_words(from, c + n, width);
}

template <typename T>
__device__ __forceinline__ void store_scaled(T* row, int32_t c, Width width, float scale, float (&v)[Chunk<T>::N]) {
#pragma unroll
  for (int n = 0; n < Chunk<T>::N; ++n) v[n] *= scale;
  store_chunk(row, c, width, v);
}

// A group goes through RUN sorted positions, a workgroup through as many runs beside each other as it has groups.  Ids that begin
// and end in the workgroup's are written; of others it leaves parts [workgroups x 2 x width]: of the id that began in front, and
// of the one that goes on.  named[v]: id v is there.  The launch's first workgroup is number `first`.
template <typename T, int RUN>
__global__ __launch_bounds__(THREADS) void k_lookup_sums(const uint64_t* __restrict__ sorted, int64_t n, uint32_t rows,
                                                         RowsOf<const T> dy, RowsOf<T> dtable, int32_t shift, Width width,
                                                         float scale, float* __restrict__ part, uint8_t* __restrict__ named,
                                                         int64_t first) {
  constexpr int N = Chunk<T>::N, U = 4;
  __shared__ float heads[THREADS][N + 1];       // of every run, the sums of the id that began in front of it
  __shared__ uint8_t head_ends[THREADS];        // and whether that ends in the run
  const int32_t groups = THREADS >> shift, own = threadIdx.x >> shift, lane = threadIdx.x & ((1 << shift) - 1);
  const int32_t c = ((int32_t)(blockIdx.y << shift) + lane) * N;
  const int64_t block = first + blockIdx.x;
  const int64_t begin = (block * groups + own) * RUN;
  const int64_t end = begin + RUN < n ? begin + RUN : n;
  const bool there = begin < n;
  const uint32_t in_front = there && begin > 0 ? id_of(sorted[begin - 1]) : 0xFFFFFFFFu;
  const uint32_t behind = end < n ? id_of(sorted[end]) : 0xFFFFFFFFu;
  uint32_t id = there ? id_of(sorted[begin]) : 0xFFFFFFFFu;
  const bool headed = id == in_front && id < rows;
  bool began = !headed;                         // whether the id that is summed began in this run
  float sum[N] = {};
  const auto put_head = [&](bool ends) {
#pragma unroll
    for (int i = 0; i < N; ++i) heads[threadIdx.x][i] = sum[i];
    if (lane == 0) head_ends[own] = ends;
  };
  const auto write = [&]() {
    if (c < width.width) store_scaled(dtable.at(id), c, width, scale, sum);
  };
  if (there && id < rows) {                     // (ids without a row are the last)
    for (int64_t p = begin; p < end; p += U) {
      uint64_t word[U];
      ChunkWords<T> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) word[u] = sorted[p + u < end ? p + u : end - 1];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = load_words(dy.at((uint32_t)word[u]), c, width);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t next = id_of(word[u]);
        if (p + u < end && next != id && id < rows) {
          if (began) {
            write();
            if (c == 0) named[id] = 1;
          } else {
            put_head(true);
          }
          id = next;
          began = true;
#pragma unroll
          for (int i = 0; i < N; ++i) sum[i] = 0.f;
        }
        if (p + u < end) {
#pragma unroll
          for (int i = 0; i < N; ++i) sum[i] += (float)v[u].wide[i];
        }
      }
      if (id >= rows) break;
    }
  }
  const bool goes_on = id < rows && id == behind;
  if (id < rows && began) {
    if (!goes_on) write();
    if (c == 0) named[id] = 1;
  }
  if (id < rows && !began) put_head(!goes_on);
  __syncthreads();
  // The id that goes on behind this run, up to where it ends; the first run's head, too.
  const Width of_parts = {width.width, (4 - width.width % 4) % 4};
  const auto follow = [&](int32_t h) {
    for (; h < groups; ++h) {
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += heads[(h << shift) + lane][i];
      if (head_ends[h]) return true;
    }
    return false;
  };
  if (goes_on && began) {
    if (follow(own + 1)) write();
    else store_part<N>(part + (2 * block + 1) * width.width, c, of_parts, sum);
  }
  if (own == 0 && headed) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = heads[threadIdx.x][i];
    if (!head_ends[0]) follow(1);
    store_part<N>(part + 2 * block * width.width, c, of_parts, sum);
  }
}

// The run in which an id ends that is at the end of run `from`.
__device__ __forceinline__ int64_t last_run_of(const uint64_t* __restrict__ sorted, int64_t n, uint32_t id, int64_t from,
                                               int32_t run_length) {
  int64_t lo = (from + 1) * run_length - 1, hi = n;          // sorted[lo] has the id, from hi on none does
  for (int64_t step = 4 * run_length; hi - lo > step; step *= 4) {
    if (id_of(sorted[lo + step]) == id) {
      lo += step;
    } else {
      hi = lo + step;
      break;
    }
  }
  while (hi - lo > 1) {
    const int64_t mid = lo + (hi - lo) / 2;
    if (id_of(sorted[mid]) == id) lo = mid;
    else hi = mid;
  }
  return lo / run_length;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void k_lookup_join(const uint64_t* __restrict__ sorted, int64_t n, int32_t run_length, uint32_t rows,
                                                         RowsOf<T> dtable, int32_t shift, Width width, float scale,
                                                         const float* __restrict__ part, const uint8_t* __restrict__ named) {
  constexpr int N = Chunk<T>::N, U = 8;
  __shared__ int64_t long_last[THREADS];
  __shared__ float sums[THREADS][N + 1];
  const int32_t groups = THREADS >> shift, lane = threadIdx.x & ((1 << shift) - 1), own = threadIdx.x >> shift;
  const int32_t c = ((int32_t)(blockIdx.y << shift) + lane) * N;
  const int64_t runs = (n + run_length - 1) / run_length, run = (int64_t)blockIdx.x * groups + own;

  const Width of_parts = {width.width, (4 - width.width % 4) % 4};
  const auto add_parts = [&](float (&sum)[N], int64_t from, int64_t upto, int64_t step) {
    for (int64_t h = from; h <= upto; h += U * step) {
      ChunkWords<float> v[U][N / 4];
#pragma unroll
      for (int u = 0; u < U; ++u) load_part<N>(part + (h + u * step <= upto ? h + u * step : h) * 2 * width.width, c, of_parts, v[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += h + u * step <= upto ? v[u][i / 4].wide[i % 4] : 0.f;
    }
  };
  const auto first_part = [&](float (&sum)[N], int64_t of) {
    ChunkWords<float> v[N / 4];
    load_part<N>(part + (of * 2 + 1) * width.width, c, of_parts, v);
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = v[i / 4].wide[i % 4];
  };

  // an id that begins in this run and goes on behind it
  bool opens = false;
  uint32_t id = 0;
  int64_t last = -1;
  if (run < runs && (run + 1) * run_length < n) {
    const int64_t next_end = (run + 2) * run_length;
    id = id_of(sorted[(run + 1) * run_length]);
    const uint32_t at_end = id_of(sorted[(run + 1) * run_length - 1]), further = id_of(sorted[next_end < n ? next_end : n - 1]);
    const uint32_t in_front = id_of(sorted[run > 0 ? run * run_length - 1 : 0]);
    opens = id < rows && at_end == id && (run == 0 || in_front != id);
    if (opens) last = next_end < n && further == id ? last_run_of(sorted, n, id, run + 1, run_length) : run + 1;
  }
  const bool is_long = opens && last - run > LONG;
  if (opens && !is_long) {
    float sum[N];
    first_part(sum, run);
    add_parts(sum, run + 1, last, 1);
    if (c < width.width) store_scaled(dtable.at(id), c, width, scale, sum);
  }
  if (lane == 0) long_last[own] = is_long ? last : -1;
  __syncthreads();
  for (int32_t g = 0; g < groups; ++g) {
    const int64_t upto = long_last[g];
    if (upto < 0) continue;                 // (the same for all threads)
    const int64_t from = (int64_t)blockIdx.x * groups + g;
    float sum[N] = {};
    add_parts(sum, from + 1 + own, upto, groups);
#pragma unroll
    for (int i = 0; i < N; ++i) sums[threadIdx.x][i] = sum[i];
    __syncthreads();
    if (own == 0) {
      first_part(sum, from);
      for (int32_t k = 0; k < groups; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += sums[(k << shift) + lane][i];
      if (c < width.width) store_scaled(dtable.at(id_of(sorted[(from + 1) * run_length])), c, width, scale, sum);
    }
    __syncthreads();
  }

  // rows that no id names
  for (int64_t v = run; v < rows; v += (int64_t)gridDim.x * groups) {
    if (named[v] || c >= width.width) continue;
    const float zero[N] = {};
    store_chunk(dtable.at(v), c, width, zero);
  }
}

// Sorted positions of a group: few where there are few groups.
constexpr int SHORT_RUN = 8, LONG_RUN = 16;
int64_t run_of(int64_t n) { return n < (1 << 17) ? SHORT_RUN : LONG_RUN; }

struct LookupSpace {
  uint64_t *a, *b;
  uint32_t* hist;
  float* part;
  uint8_t* named;
  size_t bytes;
};
LookupSpace lookup_space(void* ws, int64_t n, int64_t rows, int64_t width) {
  Arena arena(ws);
  LookupSpace s;
  s.a = arena.take<uint64_t>(n);
  s.b = arena.take<uint64_t>(n);
  s.hist = arena.take<uint32_t>(radix_plan(n).hist_elems);
  s.part = arena.take<float>(ceil_div(n, 4 * run_of(n)) * 2 * width);         // (a workgroup has 4 runs at least)
  s.named = arena.take<uint8_t>(ceil_div(rows, 4) * 4);
  s.bytes = arena.used + 256;
  return s;
}

int32_t check_lookup_sizes(int64_t ids, int64_t rows, int64_t width) {
  if (ids < 0 || ids > ((int64_t)1 << 30)) return fail(GINEX_ERR_ARG, "ids=%lld (0..2^30)", (long long)ids);
  if (rows < 0 || rows >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "rows=%lld", (long long)rows);
  if (width < 1 || width > GINEX_MAX_WIDTH) return fail(GINEX_ERR_ARG, "width=%lld (1..%d)", (long long)width, GINEX_MAX_WIDTH);
  return GINEX_OK;
}

int32_t check_ids(const void* ids, int32_t ids_64, int64_t n) {
  if (ids_64 != 0 && ids_64 != 1) return fail(GINEX_ERR_ARG, "ids_64=%d", ids_64);
  if ((n > 0 && !ids) || reinterpret_cast<uintptr_t>(ids) % (ids_64 ? 8 : 4))
    return fail(GINEX_ERR_ARG, "ids: null or misaligned");
  return GINEX_OK;
}

template <typename Id>
hipError_t sort_ids(const void* ids, int64_t n, int64_t rows, const LookupSpace& s, hipStream_t st, uint64_t** sorted) {
  const int64_t words = ceil_div(rows, 4);
  if (n > 0 && n <= MOST_PLACED) {
    int64_t groups = ceil_div(words, 4 * PLACE_THREADS);        // enough to clear a large table's marks
    groups = groups < 2048 ? groups : 2048;
    groups = groups > ceil_div(n, WAVE) ? groups : ceil_div(n, WAVE);
    hipLaunchKernelGGL(k_lookup_places<Id>, dim3((unsigned)groups), dim3(PLACE_THREADS), 0, st,
                       IdsWithPositions<Id>{static_cast<const Id*>(ids), (uint32_t)rows}, (int32_t)n, s.a,
                       reinterpret_cast<uint32_t*>(s.named), words);
    *sorted = s.a;
    return hipGetLastError();
  }
  if (hipError_t e = fill_async(reinterpret_cast<uint32_t*>(s.named), words, 0u, st)) return e;
  if (n == 0) return hipSuccess;
  int bits = 1;
  while (bits < 32 && rows >> bits) ++bits;         // (of the value `rows`, too)
  const int passes = radix_passes(bits, n);
  uint64_t *from = nullptr, *to = s.a;
  int shift = 32;
  for (int k = 0; k < passes; ++k) {
    const int width = radix_pass_width(bits, passes, k);
    const IdsWithPositions<Id> first = {static_cast<const Id*>(ids), (uint32_t)rows};
    const hipError_t e = k == 0 ? radix_pass(first, to, n, shift, width, s.hist, st)
                                : radix_pass(RadixWords{from}, to, n, shift, width, s.hist, st);
    if (e != hipSuccess) return e;
    from = to;
    to = from == s.a ? s.b : s.a;
    shift += width;
  }
  *sorted = from;
  return hipSuccess;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

extern "C" int32_t ginex_lookup(const ginex_rows_t* table, const void* ids, int32_t ids_64, float scale,
                                const ginex_rows_t* out, void* stream) {
  if (int32_t rc = check_rows("table", table, false)) return rc;
  if (int32_t rc = check_rows("out", out, true)) return rc;
  if (int32_t rc = check_same("table", table, "out", out)) return rc;
  if (int32_t rc = check_ids(ids, ids_64, out->rows)) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(out->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    constexpr int EACH = 4 * THREADS;
    const int64_t cpr = ceil_div(out->width, Chunk<T>::N), step = (((int64_t)1 << 31) - EACH) / cpr;
    for (int64_t r = 0; r < out->rows; r += step) {
      const int64_t chunks = (out->rows - r < step ? out->rows - r : step) * cpr;
      const dim3 grid((unsigned)ceil_div(chunks, EACH));
      if (ids_64)
        hipLaunchKernelGGL((k_lookup<T, int64_t>), grid, dim3(THREADS), 0, st, read_rows<T>(table), table->rows,
                           static_cast<const int64_t*>(ids), rows_of<T>(out), r, (uint32_t)chunks, Divisor((uint32_t)cpr),
                           Width::of<T>(out->width), scale);
      else
        hipLaunchKernelGGL((k_lookup<T, int32_t>), grid, dim3(THREADS), 0, st, read_rows<T>(table), table->rows,
                           static_cast<const int32_t*>(ids), rows_of<T>(out), r, (uint32_t)chunks, Divisor((uint32_t)cpr),
                           Width::of<T>(out->width), scale);
      GINEX_LAUNCH_CHECK();
    }
    return GINEX_OK;
  });
}

extern "C" size_t ginex_lookup_backward_workspace_bytes(int64_t ids, int64_t rows, int64_t width) {
  if (check_lookup_sizes(ids, rows, width)) return 0;
  return lookup_space(nullptr, ids, rows, width).bytes;
}

extern "C" int32_t ginex_lookup_backward(const ginex_rows_t* dy, const void* ids, int32_t ids_64, float scale,
                                         const ginex_rows_t* dtable, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_rows("dy", dy, false)) return rc;
  if (int32_t rc = check_rows("dtable", dtable, true)) return rc;
  if (int32_t rc = check_same("dy", dy, "dtable", dtable)) return rc;
  if (int32_t rc = check_ids(ids, ids_64, dy->rows)) return rc;
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(GINEX_ERR_ARG, "workspace: null or misaligned");
  const int64_t n = dy->rows, rows = dtable->rows;
  if (int32_t rc = check_lookup_sizes(n, rows, dy->width)) return rc;
  const LookupSpace s = lookup_space(ws, n, rows, dy->width);
  if (ws_bytes < s.bytes) return fail(GINEX_ERR_WORKSPACE, "workspace: need %zu bytes, got %zu", s.bytes, ws_bytes);
  if (rows == 0) return GINEX_OK;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  uint64_t* sorted = nullptr;
  GINEX_HIP(ids_64 ? sort_ids<int64_t>(ids, n, rows, s, st, &sorted)
                   : sort_ids<int32_t>(ids, n, rows, s, st, &sorted));
  return with_type(dy->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const int64_t cpr = ceil_div(dy->width, Chunk<T>::N);
    int32_t shift = 0;
    while (shift < 6 && 1 << shift < cpr) ++shift;
    const unsigned across = (unsigned)ceil_div(cpr, 1 << shift);
    const Width width = Width::of<T>(dy->width);
    const int32_t run_length = (int32_t)run_of(n) * (THREADS >> shift);
    const int64_t runs = ceil_div(n, run_length);
    const auto kernel = run_of(n) == SHORT_RUN ? k_lookup_sums<T, SHORT_RUN> : k_lookup_sums<T, LONG_RUN>;
    const int64_t step = (int64_t)1 << 23;        // (a launch has fewer than 2^32 threads)
    for (int64_t first = 0; first < runs; first += step) {
      const int64_t count = runs - first < step ? runs - first : step;
      hipLaunchKernelGGL(kernel, dim3((unsigned)count, across), dim3(THREADS), 0, st, sorted, n, (uint32_t)rows, read_rows<T>(dy),
                         rows_of<T>(dtable), shift, width, scale, s.part, s.named, first);
      GINEX_LAUNCH_CHECK();
    }
    // a group for every run, and enough of them for the rows that are cleared
    int64_t groups = rows < 65536 ? rows : 65536;
    groups = groups > runs ? groups : runs;
    hipLaunchKernelGGL(k_lookup_join<T>, dim3((unsigned)ceil_div(groups, THREADS >> shift), across), dim3(THREADS), 0, st, sorted, n,
                       run_length, (uint32_t)rows, rows_of<T>(dtable), shift, width, scale, s.part, s.named);
    GINEX_LAUNCH_CHECK();
    return GINEX_OK;
  });
}
