// The rules of csrc/slots.hpp behind a C ABI, for tests/test_slot_rules.py (test infrastructure, host code only).
#include "slots.hpp"

using namespace ginex;

extern "C" int64_t rules_first_free_chunk(int64_t end, int64_t slots, uint32_t chunks_a_row) {
  return first_free_chunk(end, slots, chunks_a_row);
}
