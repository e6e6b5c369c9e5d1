// Weight gradients of one linear layer per expert, from rows kept in 8 bits:
//
//   dw[e][c][d] = sum over the slots s of expert e of  x(source[s], c) * dy(s, d)
//
// A product of two matrices whose long axis, the slots, is cut into pieces of equal length within the
// experts, so that few experts or uneven ones still fill the GPU.  An expert of one piece is written where
// it belongs; the pieces of a longer one go to the workspace and are added up in their order by a second
// launch, so that equal inputs give equal bits.
#include "codes.hpp"

namespace ginex {
namespace {

constexpr int JOIN_THREADS = 256;
constexpr int WAVE_TILE = 64;     // channels and outputs of a wave: 2 x 2 tiles of a matrix instruction
constexpr int DEPTH = 32;         // slots in LDS at a time
constexpr int PAD = 32;           // elements behind a row in LDS, see product()

typedef short half_words __attribute__((ext_vector_type(4)));
typedef bf16 fragment __attribute__((ext_vector_type(8)));
typedef float tile __attribute__((ext_vector_type(16)));
typedef uint32_t words4 __attribute__((ext_vector_type(4)));

// A gradient as a sum of bf16 numbers, exactly: the significand's bits eight at a time (bf16 has 8, f16 11, f32 24).
template <typename T>
constexpr int TERMS = 1;
template <>
constexpr int TERMS<f16> = 2;
template <>
constexpr int TERMS<float> = 3;

// The pieces of all experts: ceil(slots of the expert / length) each, numbered in order.
struct Piece {
  int32_t expert;      // -1: no such piece
  int64_t begin, end;  // its slots
  int32_t part;        // its place in the workspace; -1: the expert's only piece
};

struct Shares {
  int64_t length;      // slots of a piece
  int64_t pieces;      // at most, of all experts
  int64_t parts;       // at most, of experts with more than one
};

// An expert's slots; a routing that was not made by ginex_route cannot name slots that are not there.
__device__ __forceinline__ void slots_of(const int64_t* __restrict__ offsets, int32_t e, int64_t slots, int64_t& begin,
                                         int64_t& end) {
  begin = offsets ? offsets[e] : 0;
  end = offsets ? offsets[e + 1] : slots;
  begin = begin < 0 ? 0 : (begin < slots ? begin : slots);
  end = end < begin ? begin : (end < slots ? end : slots);
}

template <int THREADS>
__device__ __forceinline__ Piece find_piece(const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                            int64_t length, int64_t wanted, int64_t most_parts, Piece* found,
                                            uint32_t* smem) {
  if (threadIdx.x == 0) *found = {-1, 0, 0, -1};
  __syncthreads();
  uint32_t pieces_before = 0, parts_before = 0;
  for (int32_t e0 = 0; e0 < experts; e0 += THREADS) {
    const int32_t e = e0 + (int32_t)threadIdx.x;
    int64_t begin = 0, end = 0;
    if (e < experts) slots_of(offsets, e, slots, begin, end);
    const uint32_t pieces = (uint32_t)((end - begin + length - 1) / length);
    const uint32_t parts = pieces > 1 ? pieces : 0;
    uint32_t all_pieces, all_parts;
    const uint32_t piece = pieces_before + block_exclusive_scan<uint32_t, THREADS>(pieces, smem, all_pieces);
    const uint32_t part = parts_before + block_exclusive_scan<uint32_t, THREADS>(parts, smem, all_parts);
    // (parts beyond the workspace: offsets that do not ascend, which ginex_route does not make)
    if (wanted >= piece && wanted < piece + pieces && (parts == 0 || part + (wanted - piece) < most_parts)) {
      const int64_t at = begin + (wanted - piece) * length;
      *found = {e, at, at + length < end ? at + length : end, parts ? (int32_t)(part + (wanted - piece)) : -1};
    }
    pieces_before += all_pieces;
    parts_before += all_parts;
  }
  __syncthreads();
  return *found;
}

// Waits for this wave's LDS accesses and for the other waves, not for loads from HBM that are under way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The upper halves of two f32: two bf16 in a word.
__device__ __forceinline__ uint32_t upper_halves(float first, float second) {
  return __builtin_amdgcn_perm(__float_as_uint(second), __float_as_uint(first), 0x07060302u);
}

// Eight elements of a gradient on their way from HBM to LDS: as they came, until they are cut into terms.
template <typename T>
struct Eight {
  static constexpr int N = Chunk<T>::N;
  typename Chunk<T>::Wide v[8 / N];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) v[i] = *reinterpret_cast<const typename Chunk<T>::At*>(p + i * N);
  }
  __device__ __forceinline__ void load(const T* p, int left) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i / N][i % N] = i < left ? p[i] : (T)0.f;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i / N][i % N] = (T)0.f;
  }
};

// Term t is the upper half (sign, exponent, 8 bits of significand) of what the terms before it have left.  An infinity
// is its first term alone: taken from itself it would leave a NaN.  One is looked for in all eight numbers at once.
template <typename T>
struct Terms {
  float v[8];
  bool infinite;
  __device__ __forceinline__ explicit Terms(const Eight<T>& from) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = (float)from.v[i / Eight<T>::N][i % Eight<T>::N];
      top = fmaxf(top, fabsf(v[i]));
    }
    infinite = __any(top == INFINITY);
  }
  __device__ __forceinline__ words4 next() {
    words4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = upper_halves(v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float left = v[i] - __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u);
      v[i] = infinite && fabsf(v[i]) == INFINITY ? 0.f : left;
    }
    return out;
  }
};
template <>
struct Terms<bf16> {
  words4 v;
  __device__ __forceinline__ explicit Terms(const Eight<bf16>& from) : v(__builtin_bit_cast(words4, from.v[0])) {}
  __device__ __forceinline__ words4 next() { return v; }
};

// Eight numbers along the slots for a lane's row of a matrix operand, from an LDS array that has slots as its rows:
// the 16 lanes of a group bring 4 rows of 16 numbers and get a column each.
__device__ __forceinline__ fragment column_of(const bf16* at, int pitch) {
  typedef __attribute__((address_space(3))) half_words* Local;
  union {
    half_words half[2];
    fragment whole;
  } u;
  u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Local)at);
  u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Local)(at + 4 * pitch));
  return u.whole;
}

// A workgroup of WM x WN waves has 64 WM channels and 64 WN outputs of one piece.
template <typename T, int WM, int WN>
__global__ __launch_bounds__(WM* WN* WAVE, WM == 4 ? 4 : 3) void k_weights(
    const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int32_t blocks,
    const int32_t* __restrict__ source, const int64_t* __restrict__ offsets, int32_t experts, int64_t slots, int64_t length,
    int64_t most_parts, RowsOf<const T> dy, int32_t width, int32_t out_width, int64_t whole_slots, int32_t tiles_m, int32_t tiles,
    float* __restrict__ dw, float* __restrict__ partial) {
  constexpr int THREADS = WM * WN * WAVE, TM = WM * WAVE_TILE, TN = WN * WAVE_TILE, TERM = TERMS<T>;
  constexpr int XS = DEPTH * TM / 16, YS = DEPTH * TN / 8;             // chunks of 16 codes and of 8 gradients
  constexpr int XN = (XS + THREADS - 1) / THREADS, YN = YS / THREADS;
  static_assert(YS % THREADS == 0, "every thread has as many chunks");
  constexpr int XP = TM + PAD, YP = TN + PAD;
  __shared__ bf16 xs[DEPTH * XP];
  __shared__ bf16 ys[TERM][DEPTH * YP];
  __shared__ uint32_t smem[THREADS / WAVE + 1];
  __shared__ Piece found;

  // Workgroups go to the 8 dies in turn: the tiles of a piece, which read the same rows, to one of them.
  const uint32_t die = blockIdx.x % 8, local = blockIdx.x / 8;
  const int32_t tile_of = (int32_t)(local % tiles);
  const Piece piece = find_piece<THREADS>(offsets, experts, slots, length, (int64_t)(local / tiles) * 8 + die, most_parts,
                                          &found, smem);
  if (piece.expert < 0) return;
  const int32_t c0 = tile_of % tiles_m * TM, d0 = tile_of / tiles_m * TN;

  // Loads are issued a step ahead and not looked at before put(): no branch and no use stands between them.  What
  // lies behind the piece's last slot is read from that slot and cleared in put(); what lies behind the last channel or
  // output goes to sums that are not written.
  words4 x[XN];
  uint32_t scale[XN];
  Eight<T> y[YN];
  int32_t row[XN], row_of[XN];       // rows of the slots of the next step, and of the one in x
  const int64_t last = piece.end - 1;
  // Steps that end here or before read whole chunks: a row of dy that ends inside a chunk is read beyond its end, which
  // is inside dy except for the rows at its end.
  const int64_t whole_end = piece.end < whole_slots ? piece.end : whole_slots;
  const uint32_t pitch = (uint32_t)blocks * GINEX_CODE_BLOCK;
  const int8_t* x_at[XN];
  const uint8_t* scale_at[XN];
  const T* y_at[YN];
#pragma unroll
  for (int i = 0; i < XN; ++i) {
    const int q = threadIdx.x + i * THREADS, b = c0 / GINEX_CODE_BLOCK + q % (TM / 16) / 2;
    const int block = b < blocks ? b : blocks - 1;
    x_at[i] = codes + block * GINEX_CODE_BLOCK + q % 2 * 16;
    scale_at[i] = scales + block;
  }
#pragma unroll
  for (int i = 0; i < YN; ++i) {
    const int q = threadIdx.x + i * THREADS, d = d0 + q % (TN / 8) * 8;
    y_at[i] = dy.at(piece.begin + q / (TN / 8), d < out_width ? d : 0);
  }
  auto find_rows = [&](int64_t s0) {
#pragma unroll
    for (int i = 0; i < XN; ++i) {
      const int k = (threadIdx.x + i * THREADS) / (TM / 16);
      const int64_t s = s0 + k < last ? s0 + k : last;
      row[i] = (int32_t)s;
      if (source) row[i] = source[s];
    }
  };
  auto fetch = [&](int64_t s0) {
#pragma unroll
    for (int i = 0; i < XN; ++i) {
      row_of[i] = row[i];
      // (a row that is not there, of a routing made elsewhere, is cleared in put() as well)
      const uint32_t r = (uint32_t)row[i] < (uint32_t)rows ? (uint32_t)row[i] : 0;
      typedef words4 At __attribute__((aligned(8)));
      x[i] = *reinterpret_cast<const At*>(x_at[i] + (uint64_t)r * pitch);
      scale[i] = scale_at[i][(uint64_t)r * (uint32_t)blocks];
    }
    if (s0 + DEPTH <= whole_end) {
#pragma unroll
      for (int i = 0; i < YN; ++i) {
        y[i].load(y_at[i]);
        y_at[i] += DEPTH * dy.stride;
      }
    } else {
#pragma unroll
      for (int i = 0; i < YN; ++i) {
        const int q = threadIdx.x + i * THREADS, k = q / (TN / 8), d = d0 + q % (TN / 8) * 8;
        const int64_t s = s0 + k < last ? s0 + k : last;
        y[i].load(dy.at(s, d < out_width ? d : 0), out_width - (d < out_width ? d : 0));
      }
    }
  };
  auto put = [&](int64_t s0) {
    const bool ends = s0 + DEPTH > piece.end;
#pragma unroll
    for (int i = 0; i < XN; ++i) {
      const int q = threadIdx.x + i * THREADS;
      if (XS % THREADS && q >= XS) break;
      const float step = code_step(scale[i]), below = -128.f * step;
      words4 out[2];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        // q step = (q + 128) step - 128 step, exactly: a byte becomes a float in one instruction if it has no sign
        const uint32_t word = x[i][w] ^ 0x80808080u;
        const float f0 = fmaf((float)(word & 255), step, below), f1 = fmaf((float)(word >> 8 & 255), step, below);
        const float f2 = fmaf((float)(word >> 16 & 255), step, below), f3 = fmaf((float)(word >> 24), step, below);
        out[w / 2][w % 2 * 2] = upper_halves(f0, f1);
        out[w / 2][w % 2 * 2 + 1] = upper_halves(f2, f3);
      }
      if ((ends && s0 + q / (TM / 16) > last) || (uint32_t)row_of[i] >= (uint32_t)rows) out[0] = out[1] = words4{0, 0, 0, 0};
      words4* const to = reinterpret_cast<words4*>(xs + q / (TM / 16) * XP + q % (TM / 16) * 16);
      to[0] = out[0];
      to[1] = out[1];
    }
#pragma unroll
    for (int i = 0; i < YN; ++i) {
      const int q = threadIdx.x + i * THREADS;
      if (ends && s0 + q / (TN / 8) > last) y[i].clear();
      Terms<T> terms(y[i]);
#pragma unroll
      for (int t = 0; t < TERM; ++t)
        *reinterpret_cast<words4*>(ys[t] + q / (TN / 8) * YP + q % (TN / 8) * 8) = terms.next();
    }
  };

  // A lane's place in the operands: the group of 16 lanes reads rows k .. k+3 of 16 columns; lanes 32 to 63
  // have slots 8 to 15.  Rows lie 64 bytes (of 256: all banks) apart, so that a half-wave's 4 rows of 64 bytes
  // use every bank once.
  const int lane = lane_id(), wave = threadIdx.x / WAVE;
  const int wm = wave % WM, wn = wave / WM;
  const int k_of = 8 * (lane / 32) + lane % 16 / 4, col_of = lane % 32 / 16 * 16 + lane % 4 * 4;
  const bf16* const xa = xs + k_of * XP + wm * WAVE_TILE + col_of;
  const int yb = k_of * YP + wn * WAVE_TILE + col_of;
  tile sum[2][2] = {};
  auto product = [&]() {
#pragma unroll
    for (int k = 0; k < DEPTH; k += 16) {
      fragment a[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) a[m] = column_of(xa + k * XP + m * 32, XP);
#pragma unroll
      for (int t = 0; t < TERM; ++t) {
        fragment b[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) b[n] = column_of(ys[t] + yb + k * YP + n * 32, YP);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int n = 0; n < 2; ++n) sum[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[m], b[n], sum[m][n], 0, 0, 0);
      }
    }
  };

  find_rows(piece.begin);
  fetch(piece.begin);
  find_rows(piece.begin + DEPTH);
  for (int64_t s0 = piece.begin; s0 < piece.end; s0 += DEPTH) {
    lds_barrier();
    put(s0);
    fetch(s0 + DEPTH);
    find_rows(s0 + 2 * DEPTH);
    lds_barrier();
    product();
  }

  const int64_t size = (int64_t)width * out_width;
  float* const to = piece.part < 0 ? dw + piece.expert * size : partial + piece.part * size;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int32_t c = c0 + wm * WAVE_TILE + m * 32 + i % 4 + i / 4 * 8 + lane / 32 * 4;
        const int32_t d = d0 + wn * WAVE_TILE + n * 32 + lane % 32;
        if (c < width && d < out_width) to[(int64_t)c * out_width + d] = sum[m][n][i];
      }
}

// Experts of several pieces: added up in order.  Experts without slots: cleared.
__global__ __launch_bounds__(JOIN_THREADS) void k_weights_join(const int64_t* __restrict__ offsets, int32_t experts,
                                                          int64_t slots, int64_t length, int64_t most_parts, int64_t size,
                                                          const float* __restrict__ partial, float* __restrict__ dw) {
  __shared__ uint32_t smem[JOIN_THREADS / WAVE + 1];
  const int32_t mine = blockIdx.y;
  uint32_t before = 0;
  for (int32_t e0 = 0; e0 < mine; e0 += JOIN_THREADS) {
    const int32_t e = e0 + (int32_t)threadIdx.x;
    int64_t begin = 0, end = 0;
    if (e < mine) slots_of(offsets, e, slots, begin, end);
    const uint32_t pieces = (uint32_t)((end - begin + length - 1) / length);
    uint32_t total;
    block_exclusive_scan<uint32_t, JOIN_THREADS>(pieces > 1 ? pieces : 0, smem, total);
    before += total;
  }
  int64_t begin, end;
  slots_of(offsets, mine, slots, begin, end);
  const int64_t pieces = (end - begin + length - 1) / length;
  if (pieces == 1) return;
  for (int64_t i = (int64_t)blockIdx.x * JOIN_THREADS + threadIdx.x; i < size; i += (int64_t)gridDim.x * JOIN_THREADS) {
    float sum = 0.f;
    for (int64_t p = 0; p < pieces && before + p < most_parts; ++p) sum += partial[(before + p) * size + i];
    dw[mine * size + i] = sum;
  }
}

// Waves of a workgroup along the channels and the outputs.
struct Tiling {
  int32_t wm, wn;
  int64_t tiles_m, tiles_n;
  int64_t tiles() const { return tiles_m * tiles_n; }
};

Tiling tiling_of(int64_t width, int64_t out_width) {
  Tiling t;
  t.wm = width > 2 * WAVE_TILE ? 4 : width > WAVE_TILE ? 2 : 1;
  t.wn = t.wm == 1 ? 4 : 2;
  t.tiles_m = ceil_div(width, t.wm * WAVE_TILE);
  t.tiles_n = ceil_div(out_width, t.wn * WAVE_TILE);
  return t;
}

Shares shares_of(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  const Tiling t = tiling_of(width, out_width);
  // Two workgroups to a CU.  Every expert's last piece may be a short one, so there are up to `experts` more pieces than
  // cuts: they are to fit in as well, unless there are so many that the GPU goes through its pieces several times anyway.
  int64_t cuts = 512 / t.tiles() - experts;
  if (cuts < 256 / t.tiles()) cuts = ceil_div(1024, t.tiles());
  const int64_t most = ceil_div(slots, 512);
  cuts = cuts < most ? cuts : most;
  cuts = cuts < 1 ? 1 : cuts;
  Shares s;
  s.length = ceil_div(ceil_div(slots, cuts), DEPTH) * DEPTH;
  if (s.length < DEPTH) s.length = DEPTH;
  // sum over the experts of ceil(n / length), for those of more than one piece: fewer than cuts of them
  s.pieces = cuts + experts;
  s.parts = cuts + (experts < cuts ? experts : cuts);
  return s;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

static int32_t check_sizes(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  if (slots < 0 || slots >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "slots=%lld", (long long)slots);
  if (experts < 1 || experts > GINEX_MAX_EXPERTS) return fail(GINEX_ERR_ARG, "experts=%d (1..%d)", experts, GINEX_MAX_EXPERTS);
  if (width < 1 || width > GINEX_MAX_WIDTH || out_width < 1 || out_width > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "%lld x %lld weights (1..%d each)", (long long)width, (long long)out_width, GINEX_MAX_WIDTH);
  return GINEX_OK;
}

extern "C" size_t ginex_weight_gradient_workspace_bytes(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  if (check_sizes(slots, experts, width, out_width) != GINEX_OK) return 0;
  Arena a(nullptr);
  a.take<float>(shares_of(slots, experts, width, out_width).parts * width * out_width);
  a.take<char>(256);
  return a.used;
}

extern "C" int32_t ginex_weight_gradient(const ginex_codes_t* kept, const ginex_routing_t* route, const ginex_rows_t* dy,
                                         float* dw, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_codes(kept)) return rc;
  if (route)
    if (int32_t rc = check_routing(route)) return rc;
  if (int32_t rc = check_rows("dy", dy, false)) return rc;
  if (route && route->rows != kept->rows)
    return fail(GINEX_ERR_ARG, "the routing has %lld rows, the codes %lld", (long long)route->rows, (long long)kept->rows);
  const int64_t slots = route ? route->rows * route->top : kept->rows;
  const int32_t experts = route ? route->experts : 1;
  if (dy->rows != slots) return fail(GINEX_ERR_ARG, "dy has %lld rows for %lld slots", (long long)dy->rows, (long long)slots);
  if (!dw || reinterpret_cast<uintptr_t>(dw) % 4) return fail(GINEX_ERR_ARG, "dw: null or misaligned");
  const size_t need = ginex_weight_gradient_workspace_bytes(slots, experts, kept->width, dy->width);
  if (need == 0) return GINEX_ERR_ARG;
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256)
    return fail(GINEX_ERR_ARG, "weight gradient: null or misaligned workspace (256 bytes)");
  if (ws_bytes < need) return fail(GINEX_ERR_WORKSPACE, "weight gradient: workspace %zu bytes, need %zu", ws_bytes, need);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const Shares share = shares_of(slots, experts, kept->width, dy->width);
  const int32_t* const source = route ? route->source : nullptr;
  const int64_t* const offsets = route ? route->offsets : nullptr;
  float* const partial = static_cast<float*>(ws);
  const int64_t size = kept->width * dy->width;
  return with_type(dy->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    // rows at the end of dy from which no 8 elements can be read at the last chunk
    const int64_t over = (8 - dy->width % 8) % 8;
    const int64_t cut_off = over == 0 ? 0 : dy->stride == 0 ? slots : ceil_div(over, dy->stride);
    const Tiling by = tiling_of(kept->width, dy->width);
    const auto kernel = by.wm == 4 ? k_weights<T, 4, 2> : by.wm == 2 ? k_weights<T, 2, 2> : k_weights<T, 1, 4>;
    const int64_t groups = ceil_div(share.pieces, 8) * 8 * by.tiles();
    if (groups >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "weight gradient: %d x %lld x %lld weights are too many",
                                                  experts, (long long)kept->width, (long long)dy->width);
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups),
                       dim3((unsigned)(by.wm * by.wn * WAVE)), 0, st, kept->codes, kept->scales, kept->rows,
                       (int32_t)code_blocks(kept->width), source, offsets, experts, slots, share.length, share.parts,
                       RowsOf<const T>{static_cast<const T*>(dy->data), dy->stride}, (int32_t)kept->width,
                       (int32_t)dy->width, slots - cut_off, (int32_t)by.tiles_m, (int32_t)by.tiles(), dw, partial);
    GINEX_LAUNCH_CHECK();
    const int64_t blocks = ceil_div(size, JOIN_THREADS);
    hipLaunchKernelGGL(k_weights_join, dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)experts), dim3(JOIN_THREADS), 0,
                       st, offsets, experts, slots, share.length, share.parts, size, partial, dw);
    GINEX_LAUNCH_CHECK();
    return GINEX_OK;
  });
}
