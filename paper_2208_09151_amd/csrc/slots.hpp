// What the training operators make of slots' numbers alone: plain C++, compiled for the GPU and, in the tests, for the CPU.
#pragma once

#include <cstdint>

#if defined(__HIP__)
#define GINEX_BOTH __host__ __device__ __forceinline__
#else
#define GINEX_BOTH inline
#endif

namespace ginex {

// An offset of a routing that may have been made elsewhere: between 0 and the number of slots, whatever it holds.  Nothing
// is computed from an offset before this.
GINEX_BOTH int64_t inside(int64_t offset, int64_t slots) { return offset < 0 ? 0 : (offset < slots ? offset : slots); }

// The chunks of the rows from `end` on, which no slot takes: the first of them, in numbers below slots * chunks a row.
GINEX_BOTH int64_t first_free_chunk(int64_t end, int64_t slots, uint32_t chunks_a_row) {
  return inside(end, slots) * (int64_t)chunks_a_row;
}

// ---- the ranges that a weight gradient's slots are cut into ----

constexpr int STEP = 16;          // the length of a range is a multiple of it

// The slots of an expert that a routing gives from `begin` to `end`.
GINEX_BOTH void bound_slots(int64_t slots, int64_t& begin, int64_t& end) {
  begin = begin < 0 ? 0 : (begin < slots ? begin : slots);
  end = end < begin ? begin : (end < slots ? end : slots);
}

// Slots of a range: the slots that are taken, over `ranges` ranges, rounded up.  (There are fewer than 2^31 slots: divisions
// are in 32 bits, a quarter of the instructions of 64.)  A single range has all slots, whatever a routing says is taken: no
// expert can go on behind it.
GINEX_BOTH int64_t range_length(int64_t taken, int64_t slots, int32_t ranges) {
  taken = ranges == 1 ? slots : inside(taken, slots);
  const uint32_t length = ((uint32_t)(taken + ranges - 1) / (uint32_t)ranges + STEP - 1) / STEP * STEP;
  return (int64_t)(length > STEP ? length : STEP);
}

// Ranges begin at multiples of their length, but not near to where an expert begins: there they begin with it, which
// spares its part in the workspace and the start of another sum.  Both cost about as much as NEAR slots do.
constexpr int64_t NEAR = 256;

GINEX_BOTH int64_t near_of(int64_t length) { return length / 2 < NEAR ? length / 2 : NEAR; }

// Where a range that would begin at `at`, a slot of the expert that has begin .. end - 1, does begin.
GINEX_BOTH int64_t range_begin_of(int64_t at, int64_t length, int64_t begin, int64_t end) {
  const int64_t near = near_of(length);
  return at - begin <= near ? begin : end - at <= near ? end : at;
}

// Where a range leaves its part of an expert that it shares: only the first of its experts can have begun in front of
// it, and only the last can go on behind it.  One range shares no expert and needs no room for parts.
GINEX_BOTH int64_t part_of(int64_t range, bool first) { return 2 * range + (first ? 1 : 0); }
GINEX_BOTH int64_t parts_of(int64_t ranges) { return ranges > 1 ? 2 * ranges : 0; }

// The ranges first .. last that begin inside the expert that has begin .. end - 1; with last < first it lies in one range,
// else range first - 1 has its first part.  Offsets that do not ascend may put an expert behind all ranges: last is a range
// that there is before it is compared with first, and both are read only where it is not below.
struct Shared {
  int32_t first, last;
};
GINEX_BOTH Shared shared_by(int64_t begin, int64_t end, int64_t length, int32_t ranges) {
  const int64_t near = near_of(length);
  const int32_t first = (int32_t)((uint32_t)(begin + near) / (uint32_t)length) + 1;
  const int32_t last = end > near ? (int32_t)((uint32_t)(end - near - 1) / (uint32_t)length) : 0;
  return {first, last < ranges ? last : ranges - 1};
}

}  // namespace ginex
