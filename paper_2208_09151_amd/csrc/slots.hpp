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

}  // namespace ginex
