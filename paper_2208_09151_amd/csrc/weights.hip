// Weight gradients of one linear layer per expert, from rows kept in 8 bits:
//
//   dw[e][c][d] = sum over the slots s of expert e of  x(source[s], c) * dy(s, d)
//
// A product of two matrices whose long axis, the slots, is cut into ranges of equal length whatever the
// experts, so that few experts or uneven ones do not leave most of the GPU idle.  A workgroup goes through its
// range expert by expert.  An expert that lies in one range is written where it belongs; one that several
// ranges share leaves its parts in the workspace, and a second launch adds them up in their order, so that
// equal inputs give equal bits.
//
// Codes are exact in bf16, and so are the terms that a gradient is cut into: all products are exact (an f32 gradient
// below 2^-110 loses what it has below 2^-133, bf16's least bit), and the sums are the matrix cores' f32.  Codes and gradients come from HBM into registers two steps ahead, are
// taken apart on the vector unit and put into LDS with the slots as rows, where transposing reads turn them
// into operands.
//
// Measured, kernel + join, 820 000 x 2 slots in 32 experts, 256 x 256 (medians of calls in a row; the counters are of calls
// with pauses between them, in which the clock falls less): f32 593 + 15 us, 1087 TFLOP/s of bf16 products, the matrix cores
// busy in 60 % of the cycles at 1.95 GHz instead of 2.4; f16 396 + 15, 55 % at 2.1 GHz; bf16 264 + 15, 34 % at 2.4 GHz and 1.37 GB
// from HBM, 5.2 TB/s (codes are read once per expert of a row).  So f32 and f16 are bound by power and by the vector unit,
// which cuts the terms, bf16 by HBM.  76 000 x 2 in 8 experts, 128 x 256, bf16: 31 + 5 us where 89 MB come from HBM (14 us
// at its rate); the parts of 512 workgroups are 17 MB.
#include "codes.hpp"
#include "tiling.hpp"

namespace ginex {
namespace {

constexpr int JOIN_THREADS = 256;
// Elements from a row in LDS to the next: an odd multiple of 64 bytes, see k_weights.
constexpr int pitch_of(int columns) { return columns == 32 ? 32 : columns + 32; }

typedef short half_words __attribute__((ext_vector_type(4)));
typedef bf16 fragment __attribute__((ext_vector_type(8)));
typedef float tile __attribute__((ext_vector_type(16)));

// A gradient as a sum of bf16 numbers: the significand's bits eight at a time (bf16 has 8, f16 11, f32 24).  That is exact
// where the last bit is worth 2^-133 or more, which is all of bf16 and f16, and f32 from 2^-110 on.
template <typename T>
constexpr int TERMS = 1;
template <>
constexpr int TERMS<f16> = 2;
template <>
constexpr int TERMS<float> = 3;

// An expert's slots; a routing that was not made by ginex_route cannot name slots that are not there.
__device__ __forceinline__ void slots_of(const int64_t* __restrict__ offsets, int32_t e, int64_t slots, int64_t& begin,
                                         int64_t& end) {
  begin = offsets ? offsets[e] : 0;
  end = offsets ? offsets[e + 1] : slots;
  bound_slots(slots, begin, end);
}

// A number that all lanes have, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v);
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uint64_t)v >> 32)) << 32 | lo);
}

// The slots of 64 experts, one to a lane: what a wave knows of the experts, read in one trip to memory.
struct Experts {
  int32_t first;
  int64_t begin, end;
  __device__ __forceinline__ void read(const int64_t* __restrict__ offsets, int32_t experts, int64_t slots, int32_t from) {
    first = from;
    begin = end = 0;
    if (from + lane_id() < experts) slots_of(offsets, from + lane_id(), slots, begin, end);
  }
  __device__ __forceinline__ int64_t begin_of(int lane) const { return (int64_t)of_lane((uint64_t)begin, lane); }
  __device__ __forceinline__ int64_t end_of(int lane) const { return (int64_t)of_lane((uint64_t)end, lane); }
};

// The ends of a range and the expert that its first slot is of (`experts` for a range behind all slots), which is among those
// in `some` afterwards, as some[0] is before.  Every wave finds them by itself, without a barrier.
__device__ __forceinline__ int32_t find_range(const int64_t* __restrict__ offsets, int32_t experts, int64_t slots,
                                              int64_t range, int64_t length, Experts& some, int64_t& range_begin,
                                              int64_t& range_end) {
  int32_t first = experts;
  Experts now = some;
  for (int32_t e0 = 0; e0 < experts; e0 += WAVE) {
    if (e0 > 0) now.read(offsets, experts, slots, e0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t at = (range + i) * length;
      const uint64_t has = __ballot(now.begin <= at && at < now.end);
      if (has == 0) continue;
      const int lane = __ffsll((unsigned long long)has) - 1;
      const int64_t snapped = range_begin_of(at, length, now.begin_of(lane), now.end_of(lane));
      if (i == 0) {
        range_begin = snapped;
        first = e0 + lane;
        some = now;
      } else {
        range_end = snapped;
      }
    }
  }
  return first;
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

// Term t is the upper half (sign, exponent, 8 bits of significand) of what the terms before it have left: of a normal number it
// leaves 16 bits, of one below 2^-126 what is worth less than 2^-133.  What an
// infinity or a NaN leaves is that of the largest number: finite, so that its first term alone decides.
template <typename T>
struct Terms {
  float v[8];
  __device__ __forceinline__ explicit Terms(const Eight<T>& from) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = (float)from.v[i / Eight<T>::N][i % Eight<T>::N];
      // (a signalling NaN may have its bits in the lower half alone, a quiet one has not)
      if (sizeof(T) == 4) v[i] = __builtin_canonicalizef(v[i]);
    }
  }
  template <bool FIRST>
  __device__ __forceinline__ words4 next() {
    words4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = upper_halves(v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (FIRST) v[i] = __builtin_amdgcn_fmed3f(v[i], -3.402823466e38f, 3.402823466e38f);
      v[i] -= __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u);
    }
    return out;
  }
};
template <>
struct Terms<bf16> {
  words4 v;
  __device__ __forceinline__ explicit Terms(const Eight<bf16>& from) : v(__builtin_bit_cast(words4, from.v[0])) {}
  template <bool FIRST>
  __device__ __forceinline__ words4 next() {
    return v;
  }
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

// A workgroup of WM x WN waves of 32 MT x 32 NT has 32 MT WM channels and 32 NT WN outputs of a range.
template <typename T, int WM, int MT, int WN, int NT>
struct Shape {
  static constexpr int THREADS = WM * WN * WAVE, TM = WM * MT * 32, TN = WN * NT * 32, TERM = TERMS<T>;
  static constexpr int BUFFERS = WM * WN == 8 ? 2 : 1;
  static constexpr int DEPTH = TERM == 1 || TN == 32 ? 64 : 32;       // slots in LDS at a time
  static constexpr int XP = pitch_of(TM), YP = pitch_of(TN);
  static constexpr int XSIZE = DEPTH * XP, YSIZE = DEPTH * YP;            // of an array in LDS
  static constexpr int SIZE = XSIZE + TERM * YSIZE;
};

// NARROW: dy has fewer than 8 columns.
template <typename T, int WM, int MT, int WN, int NT, bool NARROW>
__global__ __launch_bounds__(WM* WN* WAVE, 2) void k_weights(
    const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int32_t blocks,
    const int32_t* __restrict__ source, const int64_t* __restrict__ offsets, int32_t experts, int64_t slots, int32_t ranges,
    RowsOf<const T> dy, int32_t width, int32_t out_width, int32_t tiles_m, int32_t tiles, float* __restrict__ dw,
    float* __restrict__ partial) {
  using S = Shape<T, WM, MT, WN, NT>;
  constexpr int THREADS = S::THREADS, TM = S::TM, TN = S::TN, TERM = S::TERM, DEPTH = S::DEPTH, XP = S::XP, YP = S::YP;
  constexpr int XS = DEPTH * TM / 16, YS = DEPTH * TN / 8;             // chunks of 16 codes and of 8 gradients
  constexpr int XN = (XS + THREADS - 1) / THREADS, YN = YS / THREADS;
  static_assert(YS % THREADS == 0 && (XS % THREADS == 0 || XS < THREADS), "chunks of a thread");
  __shared__ __attribute__((aligned(16))) bf16 lds[S::BUFFERS * S::SIZE];

  // Workgroups go to the 8 dies in turn: each die has an eighth of all, and the tiles of a range, which read the same rows,
  // stay together.  Neighbouring ranges go to different dies where all dies have as many (20 000 x 2 slots in 128 experts,
  // 256 x 256: 51 -> 47 us); with fewer than 8 ranges the dies share their tiles (16 slots, 4096 x 4096: 104 us by whole
  // ranges, 33).
  const uint32_t unit = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
  const int32_t tile_of = (int32_t)(unit % (uint32_t)tiles);
  int64_t range = unit / (uint32_t)tiles;
  if (ranges % 8 == 0) range = (blockIdx.x / 8 / (uint32_t)tiles) * 8 + blockIdx.x % 8;
  if (range >= ranges) return;
  Experts some;
  some.read(offsets, experts, slots, 0);
  const int64_t length = uniform(range_length(offsets ? offsets[experts] : slots, slots, ranges));
  const int32_t c0 = tile_of % tiles_m * TM, d0 = tile_of / tiles_m * TN;

  // its ends, and the first expert that has slots in it
  int64_t range_begin = slots, range_end = slots;
  const int32_t first_expert = find_range(offsets, experts, slots, range, length, some, range_begin, range_end);

  // Where a thread's chunks are in a row of codes and of dy.  Chunks behind the end repeat one that is there, and their
  // sums are not written; the last chunk of dy ends with the row, so it may share columns with the one in front of it.
  const uint32_t pitch = (uint32_t)blocks * GINEX_CODE_BLOCK, stride = (uint32_t)dy.stride;
  uint32_t x_at[XN], scale_at[XN], y_at[YN];
#pragma unroll
  for (int i = 0; i < XN; ++i) {
    const int q = threadIdx.x + i * THREADS, b = c0 / GINEX_CODE_BLOCK + q % (TM / 16) / 2;
    scale_at[i] = b < blocks ? b : blocks - 1;
    x_at[i] = scale_at[i] * GINEX_CODE_BLOCK + q % 2 * 16;
  }
#pragma unroll
  for (int i = 0; i < YN; ++i) {
    const int d = d0 + (threadIdx.x + i * THREADS) % (TN / 8) * 8;
    y_at[i] = NARROW ? 0 : (d <= out_width - 8 ? d : out_width - 8);
  }
  // (without a source the rows are the slots: something that is there is read in its place)
  const int32_t* const source_or_any = source ? source : reinterpret_cast<const int32_t*>(codes);

  // A lane's place in the operands: the group of 16 lanes reads rows k .. k+3 of 16 columns; lanes 32 to 63
  // have slots 8 to 15.  Rows lie 64 bytes (of 256: all banks) apart, so that a half-wave's 4 rows of 64 bytes
  // use every bank once.
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int wm = wave % WM, wn = wave / WM;
  const int k_of = 8 * (lane / 32) + lane % 16 / 4, col_of = lane % 32 / 16 * 16 + lane % 4 * 4;
  const int xb = k_of * XP + wm * MT * 32 + col_of, yb = S::XSIZE + k_of * YP + wn * NT * 32 + col_of;

  for (int32_t expert = first_expert; expert < experts; ++expert) {
    if (expert >= some.first + WAVE) some.read(offsets, experts, slots, expert);
    const int64_t expert_begin = some.begin_of(expert - some.first), expert_end = some.end_of(expert - some.first);
    if (expert_begin >= range_end) break;
    const int64_t begin = expert_begin > range_begin ? expert_begin : range_begin;
    const int64_t end = expert_end < range_end ? expert_end : range_end;
    if (begin >= end) continue;

    // Loads are issued two steps ahead and not looked at before put(): no branch and no use stands between them.  With
    // one step ahead the requests of all workgroups come at once, and then HBM waits for the next ones.  What lies
    // behind the last slot is read from that slot and cleared in put().
    words4 x[2][XN];
    uint32_t scale[2][XN];
    Eight<T> y[2][YN];
    bool there[2][XN];                 // whether the row in x exists: it may not, in a routing made elsewhere
    int32_t row[XN];                   // of the slots of the step that is fetched next
    const int64_t last = end - 1;
    auto find_rows = [&](int32_t (&row)[XN], int64_t s0) {
      const int64_t from = s0 < last ? s0 : last;
      const uint32_t left = (uint32_t)(last - from < DEPTH ? last - from : DEPTH);
      const int32_t* const at = source_or_any + (source ? from : 0);
#pragma unroll
      for (int i = 0; i < XN; ++i) {
        const uint32_t k = (threadIdx.x + i * THREADS) / (TM / 16);
        row[i] = at[source ? (k < left ? k : left) : 0];
      }
    };
    auto fetch = [&](auto set, const int32_t (&row)[XN], int64_t s0) {
      constexpr int P = decltype(set)::value;
      const int64_t from = s0 < last ? s0 : last;
      const uint32_t left = (uint32_t)(last - from < DEPTH ? last - from : DEPTH);
      // (the gradients first: they need not wait for the rows)
      const T* const at = dy.data + from * dy.stride;
#pragma unroll
      for (int i = 0; i < YN; ++i) {
        const uint32_t k = (threadIdx.x + i * THREADS) / (TN / 8);
        const T* const p = at + ((uint64_t)(k < left ? k : left) * stride + y_at[i]);
        if (NARROW) y[P][i].load(p, out_width);
        else y[P][i].load(p);
      }
#pragma unroll
      for (int i = 0; i < XN; ++i) {
        const uint32_t k = (threadIdx.x + i * THREADS) / (TM / 16);
        uint32_t r = source ? (uint32_t)row[i] : (uint32_t)from + (k < left ? k : left);
        there[P][i] = r < (uint32_t)rows;
        r = there[P][i] ? r : 0;
        typedef words4 At __attribute__((aligned(8)));
        x[P][i] = *reinterpret_cast<const At*>(codes + ((uint64_t)r * pitch + x_at[i]));
        scale[P][i] = scales[(uint64_t)r * (uint32_t)blocks + scale_at[i]];
      }
    };
    auto put = [&](auto set, bf16* to, int64_t s0) {
      constexpr int P = decltype(set)::value;
      const int left = (int)(last - s0 < DEPTH ? last - s0 : DEPTH);      // the last row that is a slot's
#pragma unroll
      for (int i = 0; i < XN; ++i) {
        const int q = threadIdx.x + i * THREADS;
        if (XS < THREADS && q >= XS) break;
        const float step = there[P][i] && q / (TM / 16) <= left ? code_step(scale[P][i]) : 0.f;
        words4 out[2];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t word = x[P][i][w];
          const float f0 = (float)(int8_t)word * step, f1 = (float)(int8_t)(word >> 8) * step;
          const float f2 = (float)(int8_t)(word >> 16) * step, f3 = (float)((int32_t)word >> 24) * step;
          out[w / 2][w % 2 * 2] = upper_halves(f0, f1);
          out[w / 2][w % 2 * 2 + 1] = upper_halves(f2, f3);
        }
        words4* const at = reinterpret_cast<words4*>(to + q / (TM / 16) * XP + q % (TM / 16) * 16);
        at[0] = out[0];
        at[1] = out[1];
      }
      if (__builtin_expect(left < DEPTH - 1, false)) {
#pragma unroll
        for (int i = 0; i < YN; ++i)
          if ((int)(threadIdx.x + i * THREADS) / (TN / 8) > left) y[P][i].clear();
      }
#pragma unroll
      for (int i = 0; i < YN; ++i) {
        const int q = threadIdx.x + i * THREADS;
        words4* const at = reinterpret_cast<words4*>(to + S::XSIZE + q / (TN / 8) * YP + q % (TN / 8) * 8);
        Terms<T> terms(y[P][i]);
        at[0] = terms.template next<true>();
#pragma unroll
        for (int t = 1; t < TERM; ++t) at[t * S::YSIZE / 8] = terms.template next<false>();
      }
    };
    tile sum[MT][NT] = {};
    auto product = [&](const bf16* from) {
      constexpr int FRAGMENTS = TERM * NT, STEPS = DEPTH / 16;
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        fragment a[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) a[m] = column_of(from + xb + k * 16 * XP + m * 32, XP);
#pragma unroll
        for (int j = 0; j < FRAGMENTS; ++j) {
          const int t = j / NT, n = j % NT;
          const fragment b = column_of(from + yb + t * S::YSIZE + k * 16 * YP + n * 32, YP);
#pragma unroll
          for (int m = 0; m < MT; ++m) sum[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[m], b, sum[m][n], 0, 0, 0);
        }
      }
      // The order of issue: a fragment is read AHEAD groups of matrix instructions (32 MT cycles each) before its own.
      constexpr int AHEAD = MT == 2 ? 3 : 2, LDS_READ = 0x100, MATRIX = 0x008;
      __builtin_amdgcn_sched_group_barrier(LDS_READ, 2 * MT + 2 * AHEAD, 0);
#pragma unroll
      for (int j = 0; j < FRAGMENTS * STEPS; ++j) {
        __builtin_amdgcn_sched_group_barrier(MATRIX, MT, 0);
        if (j + AHEAD < FRAGMENTS * STEPS) {
          if ((j + AHEAD) % FRAGMENTS == 0) __builtin_amdgcn_sched_group_barrier(LDS_READ, 2 * MT + 2, 0);
          else __builtin_amdgcn_sched_group_barrier(LDS_READ, 2, 0);
        }
      }
    };

    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    {
      int32_t row0[XN], row1[XN];
      find_rows(row0, begin);
      find_rows(row1, begin + DEPTH);
      find_rows(row, begin + 2 * DEPTH);
      fetch(even, row0, begin);
      fetch(odd, row1, begin + DEPTH);
    }
    if (S::BUFFERS == 1) {
      auto step = [&](auto set, int64_t s0) {
        lds_barrier();
        put(set, lds, s0);
        fetch(set, row, s0 + 2 * DEPTH);
        find_rows(row, s0 + 3 * DEPTH);
        lds_barrier();
        product(lds);
      };
      for (int64_t s0 = begin; s0 < end; s0 += 2 * DEPTH) {
        step(even, s0);
        if (s0 + DEPTH < end) step(odd, s0 + DEPTH);
      }
    } else {
      // The next step is put into one half of LDS while the matrix cores work from the other.  The two waves of a SIMD
      // do the two things in opposite order, so that one has the matrix core while the other has the vector unit: the
      // late one is half a turn of the loop ahead with its product.  What is put behind the last step is not read.
      const bool late = wave >= WM * WN / 2;
      put(even, lds, begin);
      fetch(even, row, begin + 2 * DEPTH);
      find_rows(row, begin + 3 * DEPTH);
      lds_barrier();
      if (late) product(lds);
      auto step = [&](auto set, int64_t s0) {
        constexpr int P = decltype(set)::value;
        put(set, lds + P * S::SIZE, s0 + DEPTH);
        fetch(set, row, s0 + 3 * DEPTH);
        find_rows(row, s0 + 4 * DEPTH);
        if (late) lds_barrier();
        if (s0 + (late ? DEPTH : 0) < end) product(lds + (late ? P : 1 - P) * S::SIZE);
        if (!late) lds_barrier();
      };
      for (int64_t s0 = begin; s0 < end; s0 += 2 * DEPTH) {
        step(odd, s0);
        step(even, s0 + DEPTH);
      }
    }

    const int64_t size = (int64_t)width * out_width;
    const bool whole = expert_begin >= range_begin && expert_end <= range_end;
    float* const to = whole ? dw + expert * size : partial + part_of(range, expert_begin >= range_begin) * size;
    // (the lane's number is made anew: addresses that do not depend on the expert would be kept through the loop above)
    int here = lane;
    asm volatile("" : "+v"(here));
    const int32_t c1 = c0 + wm * MT * 32 + here / 32 * 4, d1 = d0 + wn * NT * 32 + here % 32;
    if (c0 + TM <= width && d0 + TN <= out_width) {
      float* at = to + (int64_t)c1 * out_width + d1;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float* const line = at + (int64_t)(m * 32 + i % 4 + i / 4 * 8) * out_width;
#pragma unroll
          for (int n = 0; n < NT; ++n) line[n * 32] = sum[m][n][i];
        }
    } else {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        int32_t d = d1 + n * 32;
        // (a chunk that ends with the row, see y_at)
        if (!NARROW && d / 8 * 8 > out_width - 8 && d / 8 * 8 < out_width) d = out_width - 8 + d % 8;
        float* const at = to + d;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int32_t c = c1 + m * 32 + i % 4 + i / 4 * 8;
            if (c < width && d < out_width) at[(int64_t)c * out_width] = sum[m][n][i];
          }
      }
    }
  }
}

// Experts that several ranges share: added up in order.  Experts without slots: cleared.  A workgroup's threads are 2^shift
// groups, each of which adds up its share of the parts, four elements a thread; the first group adds up the groups' sums.
__global__ __launch_bounds__(JOIN_THREADS) void k_weights_join(const int64_t* __restrict__ offsets, int32_t experts,
                                                               int64_t slots, int32_t ranges, int64_t size, int32_t shift,
                                                               const float* __restrict__ partial, float* __restrict__ dw) {
  typedef float four __attribute__((ext_vector_type(4)));
  typedef four At __attribute__((aligned(4)));
  __shared__ four sums[JOIN_THREADS];
  const int32_t mine = blockIdx.y;
  int64_t begin, end;
  slots_of(offsets, mine, slots, begin, end);
  const int64_t length = uniform(range_length(offsets ? offsets[experts] : slots, slots, ranges));
  const auto [first, last] = shared_by(begin, end, length, ranges);
  if (end > begin && last < first) return;
  const int32_t lanes = JOIN_THREADS >> shift, lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
  const int64_t i = ((int64_t)blockIdx.x * lanes + lane) * 4;
  four sum = {};
  if (end > begin && i < size) {
    // range first - 1 and those that follow; only what the first of them has is in its second place
    const int32_t share = (last - first + 2 + (1 << shift) - 1) >> shift;
    int64_t r = first - 1 + group * share;
    const int64_t behind = r + share < last + 1 ? r + share : last + 1;
    const float* const at = partial + i;
    if (i + 4 <= size) {
      if (group == 0) sum = *reinterpret_cast<const At*>(at + part_of(r++, true) * size);
#pragma unroll 4
      for (; r < behind; ++r) sum += *reinterpret_cast<const At*>(at + part_of(r, false) * size);
    } else {
      for (int n = 0; i + n < size; ++n) {
        float one = group == 0 ? at[part_of(r, true) * size + n] : 0.f;
        for (int64_t q = group == 0 ? r + 1 : r; q < behind; ++q) one += at[part_of(q, false) * size + n];
        sum[n] = one;
      }
    }
  }
  if (shift > 0) {
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (group > 0) return;
    for (int32_t other = 1; other < 1 << shift; ++other) sum += sums[other * lanes + lane];
  }
  if (i >= size) return;
  float* const to = dw + mine * size + i;
  if (i + 4 <= size) {
    *reinterpret_cast<At*>(to) = sum;
  } else {
    for (int n = 0; n < 3; ++n)
      if (i + n < size) to[n] = sum[n];
  }
}

template <typename T>
auto kernel_of(const Tiling& t, int64_t out_width) {
  if (t.nt == 4) return k_weights<T, 4, 2, 2, 4, false>;
  if (t.wn == 4 && t.nt == 2) return k_weights<T, 2, 2, 4, 2, false>;
  if (t.wn == 4) return k_weights<T, 1, 2, 4, 1, false>;
  if (t.wm == 4) return out_width < 8 ? k_weights<T, 4, 1, 1, 1, true> : k_weights<T, 4, 1, 1, 1, false>;
  if (t.nt == 2) return k_weights<T, 2, 2, 2, 2, false>;
  return t.mt == 2 ? k_weights<T, 2, 2, 2, 1, false> : k_weights<T, 2, 1, 2, 1, false>;
}

}  // namespace
}  // namespace ginex

using namespace ginex;

static int32_t check_sizes(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  if (slots < 0 || slots >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "slots=%lld", (long long)slots);
  if (experts < 1 || experts > GINEX_MAX_EXPERTS) return fail(GINEX_ERR_ARG, "experts=%d (1..%d)", experts, GINEX_MAX_EXPERTS);
  if (width < 1 || width > GINEX_MAX_WIDTH || out_width < 1 || out_width > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "%lld x %lld weights (1..%d each)", (long long)width, (long long)out_width, GINEX_MAX_WIDTH);
  // (the second launch has a thread for four, and fewer than 2^32 threads)
  if (width * out_width >= (int64_t)1 << 33)
    return fail(GINEX_ERR_ARG, "%lld x %lld weights are too many", (long long)width, (long long)out_width);
  return GINEX_OK;
}

extern "C" size_t ginex_weight_gradient_workspace_bytes(int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  if (check_sizes(slots, experts, width, out_width) != GINEX_OK) return 0;
  Arena a(nullptr);
  const int64_t one = tiling_of(1, slots, experts, width, out_width).parts();
  const int64_t more = tiling_of(2, slots, experts, width, out_width).parts();
  a.take<float>((one > more ? one : more) * width * out_width);
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
  const Tiling by = tiling_of(dy->type == GINEX_BF16 ? 1 : 2, slots, experts, kept->width, dy->width);
  const int32_t* const source = route ? route->source : nullptr;
  const int64_t* const offsets = route ? route->offsets : nullptr;
  float* const partial = static_cast<float*>(ws);
  const int64_t size = kept->width * dy->width;
  return with_type(dy->type, [&](auto t) -> int32_t {
    using T = decltype(t);
    const int64_t groups = ceil_div(by.ranges * by.tiles(), 8) * 8;
    hipLaunchKernelGGL(kernel_of<T>(by, dy->width), dim3((unsigned)groups), dim3((unsigned)(by.wm * by.wn * WAVE)), 0, st,
                       kept->codes, kept->scales, kept->rows, (int32_t)code_blocks(kept->width), source, offsets, experts,
                       slots, by.ranges, read_rows<T>(dy), (int32_t)kept->width,
                       (int32_t)dy->width, (int32_t)by.tiles_m, (int32_t)by.tiles(), dw, partial);
    GINEX_LAUNCH_CHECK();
    // few elements: more threads for each (512 parts of 1024 elements: 46 us with one, 7 with 64)
    const auto threads = [&](int32_t shift) { return (ceil_div(size, 4) * experts) << shift; };
    int32_t shift = 0;
    while (shift < 6 && 4 << shift < by.ranges && threads(shift) < 256 * 512) ++shift;
    hipLaunchKernelGGL(k_weights_join, dim3((unsigned)ceil_div(size, 4 * (JOIN_THREADS >> shift)), (unsigned)experts),
                       dim3(JOIN_THREADS), 0, st, offsets, experts, slots, by.ranges, size, shift, partial, dw);
    GINEX_LAUNCH_CHECK();
    return GINEX_OK;
  });
}
