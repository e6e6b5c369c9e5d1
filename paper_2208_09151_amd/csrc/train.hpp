// Shared by the training operators: element types, chunks of 16 bytes at any element's address, division
// of a chunk's number by the chunks of a row, and the host-side checks of the descriptors.
#pragma once

#include "common.hpp"
#include "ginex_train.h"
#include "slots.hpp"

namespace ginex {

using bf16 = __bf16;
using f16 = _Float16;

// Elements of 16 bytes.  The hardware reads and writes such a vector at any address of an element, so rows
// of odd widths and strides take the same path as aligned ones.
template <typename T>
struct Chunk {
  static constexpr int N = 16 / sizeof(T);
  typedef T Wide __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef Wide At __attribute__((aligned(sizeof(T))));
};

typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef words2 words2_at __attribute__((aligned(2)));
typedef uint32_t word_at __attribute__((aligned(2)));

// What a kernel knows about the rows' ends: the width, and how many elements the last chunk of a row has too few.
struct Width {
  int32_t width;
  int32_t missing;
  template <typename T>
  static Width of(int64_t width) {
    constexpr int N = Chunk<T>::N;
    return {(int32_t)width, (int32_t)(ceil_div(width, N) * N - width)};
  }
};

template <typename T>
union ChunkWords {
  typename Chunk<T>::Wide wide;
  words4 words;
};

// The chunk of the row that begins at `row` from column c on, a multiple of N, as it is; columns behind the width are 0.
// The last chunk of a row that N does not divide is read so that it ends with the row, in the same instruction as all
// others, and moved into its place: element by element it was a second trip to memory for nearly every wave.
template <typename T>
__device__ __forceinline__ ChunkWords<T> load_words(const T* row, int32_t c, Width w) {
  constexpr int N = Chunk<T>::N;
  ChunkWords<T> u;
  if (w.width < N) {
#pragma unroll
    for (int i = 0; i < N; ++i) u.wide[i] = c + i < w.width ? row[c + i] : (T)0.f;
    return u;
  }
  const bool ends = c + N > w.width;
  u.wide = *reinterpret_cast<const typename Chunk<T>::At*>(row + (ends ? w.width - N : c));
  if (w.missing) {
    words4 m = u.words;
    const int bytes = w.missing * (int)sizeof(T);
    if (bytes & 8) m = words4{m[2], m[3], 0, 0};
    if (bytes & 4) m = words4{m[1], m[2], m[3], 0};
    if (bytes & 2)
      m = words4{__builtin_amdgcn_alignbit(m[1], m[0], 16), __builtin_amdgcn_alignbit(m[2], m[1], 16),
                 __builtin_amdgcn_alignbit(m[3], m[2], 16), m[3] >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) u.words[i] = ends ? m[i] : u.words[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) u.words[i] = c < w.width ? u.words[i] : 0;
  return u;
}

// The same as f32.
template <typename T>
__device__ __forceinline__ void load_chunk(const T* row, int32_t c, Width w, float (&v)[Chunk<T>::N]) {
  const ChunkWords<T> u = load_words(row, c, w);
#pragma unroll
  for (int i = 0; i < Chunk<T>::N; ++i) v[i] = (float)u.wide[i];
}

// KEEP: through the caches, which put together lines that several rows share; else past them.
template <bool KEEP = false, typename T>
__device__ __forceinline__ void store_words(T* row, int32_t c, Width w, const ChunkWords<T>& u) {
  T* p = row + c;
  if (c + Chunk<T>::N <= w.width) {
    if (KEEP) *reinterpret_cast<typename Chunk<T>::At*>(p) = u.wide;
    else __builtin_nontemporal_store(u.wide, reinterpret_cast<typename Chunk<T>::At*>(p));
    return;
  }
  // 8, 4 and 2 bytes of what is left, the same for all rows
  const int bytes = (w.width - c) * (int)sizeof(T);
  words4 m = u.words;
  if (bytes & 8) {
    *reinterpret_cast<words2_at*>(p) = words2{m[0], m[1]};
    p += 8 / sizeof(T);
    m[0] = m[2];
    m[1] = m[3];
  }
  if (bytes & 4) {
    *reinterpret_cast<word_at*>(p) = m[0];
    p += 4 / sizeof(T);
    m[0] = m[1];
  }
  if (bytes & 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)m[0];
}

// Rounded to nearest, halves to even.
template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int32_t c, Width w, const float (&v)[Chunk<T>::N]) {
  ChunkWords<T> u;
#pragma unroll
  for (int i = 0; i < Chunk<T>::N; ++i) u.wide[i] = (T)v[i];
  store_words(row, c, w, u);
}

// n / d for n below 2^31 by a multiplication (Granlund and Montgomery, "Division by invariant integers
// using multiplication", 1994).
struct Divisor {
  uint32_t d, mul, shift;
  explicit Divisor(uint32_t by) : d(by), shift(0) {
    while (shift < 31 && (1u << shift) < by) ++shift;
    mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - by)) / by + 1);
  }
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(mul, n) + n) >> shift; }
};

template <typename T>
struct RowsOf {
  T* data;
  int64_t stride;
  __device__ __forceinline__ T* at(int64_t r) const { return data + r * stride; }
};

template <typename T>
inline RowsOf<T> rows_of(const ginex_rows_t* r) {
  return {static_cast<T*>(r->data), r->stride};
}

template <typename T>
inline RowsOf<const T> read_rows(const ginex_rows_t* r) {
  return {static_cast<const T*>(r->data), r->stride};
}

inline int element_bytes(int32_t type) { return type == GINEX_F32 ? 4 : 2; }

inline int32_t check_rows(const char* what, const ginex_rows_t* r, bool written) {
  if (!r) return fail(GINEX_ERR_ARG, "%s: null descriptor", what);
  if (r->type != GINEX_F32 && r->type != GINEX_BF16 && r->type != GINEX_F16)
    return fail(GINEX_ERR_ARG, "%s: unknown type %d", what, r->type);
  if (r->rows < 0 || r->rows >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "%s: rows=%lld", what, (long long)r->rows);
  if (r->width < 1 || r->width > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "%s: width=%lld (1..%d)", what, (long long)r->width, GINEX_MAX_WIDTH);
  if ((r->stride < r->width && (written || r->stride != 0)) || r->stride > ((int64_t)1 << 31))
    return fail(GINEX_ERR_ARG, "%s: stride %lld below width %lld, or too large", what, (long long)r->stride, (long long)r->width);
  if (r->rows > 0 && !r->data) return fail(GINEX_ERR_ARG, "%s: null data", what);
  if (reinterpret_cast<uintptr_t>(r->data) % element_bytes(r->type))
    return fail(GINEX_ERR_ARG, "%s: not aligned to its elements", what);
  return GINEX_OK;
}

inline int32_t check_pairs(int64_t rows, int32_t top, int32_t experts) {
  if (top < 1 || top > GINEX_MAX_TOP) return fail(GINEX_ERR_ARG, "top=%d (1..%d)", top, GINEX_MAX_TOP);
  if (experts < 1 || experts > GINEX_MAX_EXPERTS)
    return fail(GINEX_ERR_ARG, "experts=%d (1..%d)", experts, GINEX_MAX_EXPERTS);
  if (rows < 0 || rows >= ((int64_t)1 << 31) || rows * top >= ((int64_t)1 << 31))
    return fail(GINEX_ERR_ARG, "rows=%lld of %d experts each: 2^31 pairs or more", (long long)rows, top);
  return GINEX_OK;
}

inline int32_t check_routing(const ginex_routing_t* r) {
  if (!r) return fail(GINEX_ERR_ARG, "routing: null descriptor");
  if (int32_t rc = check_pairs(r->rows, r->top, r->experts)) return rc;
  if (!r->offsets || (r->rows > 0 && (!r->slot || !r->source))) return fail(GINEX_ERR_ARG, "routing: null array");
  if (reinterpret_cast<uintptr_t>(r->offsets) % 8 || reinterpret_cast<uintptr_t>(r->slot) % 4 ||
      reinterpret_cast<uintptr_t>(r->source) % 4)
    return fail(GINEX_ERR_ARG, "routing: misaligned array");
  return GINEX_OK;
}

inline int64_t code_blocks(int64_t width) { return ceil_div(width, GINEX_CODE_BLOCK); }

inline int32_t check_codes(const ginex_codes_t* k) {
  if (!k) return fail(GINEX_ERR_ARG, "codes: null descriptor");
  if (k->rows < 0 || k->rows >= ((int64_t)1 << 31)) return fail(GINEX_ERR_ARG, "codes: rows=%lld", (long long)k->rows);
  if (k->width < 1 || k->width > GINEX_MAX_WIDTH)
    return fail(GINEX_ERR_ARG, "codes: width=%lld (1..%d)", (long long)k->width, GINEX_MAX_WIDTH);
  if (k->rows > 0 && (!k->codes || !k->scales)) return fail(GINEX_ERR_ARG, "codes: null array");
  if (reinterpret_cast<uintptr_t>(k->codes) % 8) return fail(GINEX_ERR_ARG, "codes: not aligned to 8 bytes");
  return GINEX_OK;
}

inline int32_t check_same(const char* a_is, const ginex_rows_t* a, const char* b_is, const ginex_rows_t* b) {
  if (a->type != b->type) return fail(GINEX_ERR_ARG, "%s and %s differ in type", a_is, b_is);
  if (a->width != b->width)
    return fail(GINEX_ERR_ARG, "%s and %s differ in width: %lld and %lld", a_is, b_is, (long long)a->width, (long long)b->width);
  return GINEX_OK;
}

// Calls `go` with a value of the element type.
template <typename Go>
inline int32_t with_type(int32_t type, Go go) {
  if (type == GINEX_F32) return go(float{});
  if (type == GINEX_BF16) return go(bf16{});
  return go(f16{});
}

}  // namespace ginex
