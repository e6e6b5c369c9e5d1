// The rules of csrc/slots.hpp and tiling.hpp behind a C ABI, for tests/test_slot_rules.py (test infrastructure, host code only).
#include <cstdio>
#include <map>
#include <set>
#include <utility>
#include <vector>

#include "slots.hpp"
#include "tiling.hpp"

using namespace ginex;

extern "C" int64_t rules_first_free_chunk(int64_t end, int64_t slots, uint32_t chunks_a_row) {
  return first_free_chunk(end, slots, chunks_a_row);
}

// Walks all ranges of a weight gradient, and the second launch's parts, as the kernels do.  made_here: offsets ascend, so
// every slot that is taken has to be in one range and expert, and the second launch has to read the parts that the first
// left, and no others.  0, or a number that says what is wrong.
extern "C" int32_t rules_ranges(const int64_t* offsets, int32_t experts, int64_t slots, int32_t ranges, int32_t made_here) {
  const int64_t taken = inside(offsets[experts], slots), parts = parts_of(ranges);
  const int64_t length = range_length(offsets[experts], slots, ranges);
  if (length % STEP != 0 || length * ranges < taken) return 1;
  std::vector<std::pair<int64_t, int64_t>> of(experts);
  for (int32_t e = 0; e < experts; ++e) {
    int64_t begin = offsets[e], end = offsets[e + 1];
    bound_slots(slots, begin, end);
    of[e] = {begin, end};
  }
  // the first expert of every 64 that has `at`, the last such 64 count
  const auto expert_at = [&](int64_t at) {
    int32_t found = experts;
    for (int32_t e0 = 0; e0 < experts; e0 += 64)
      for (int32_t e = e0; e < experts && e < e0 + 64; ++e)
        if (of[e].first <= at && at < of[e].second) {
          found = e;
          break;
        }
    return found;
  };
  const auto begin_of = [&](int64_t at) {
    const int32_t e = expert_at(at);
    return e == experts ? slots : range_begin_of(at, length, of[e].first, of[e].second);
  };
  std::map<int64_t, int32_t> left;      // part -> its expert
  int64_t covered = 0;
  for (int64_t range = 0; range < ranges; ++range) {
    const int32_t first_expert = expert_at(range * length);
    const int64_t range_begin = begin_of(range * length), range_end = begin_of((range + 1) * length);
    for (int32_t e = first_expert; e < experts; ++e) {
      if (of[e].first >= range_end) break;
      const int64_t begin = of[e].first > range_begin ? of[e].first : range_begin;
      const int64_t end = of[e].second < range_end ? of[e].second : range_end;
      if (begin >= end) continue;
      if (begin < 0 || end > slots) return 2;
      covered += end - begin;
      if (of[e].first >= range_begin && of[e].second <= range_end) continue;
      const int64_t part = part_of(range, of[e].first >= range_begin);
      if (part < 0 || part >= parts) return 3;
      if (!left.emplace(part, e).second && made_here) return 4;
    }
  }
  if (made_here && covered != taken) return 5;
  std::set<int64_t> read;
  for (int32_t e = 0; e < experts; ++e) {
    const auto [begin, end] = of[e];
    const Shared by = shared_by(begin, end, length, ranges);
    if (end <= begin || by.last < by.first) continue;
    for (int64_t r = by.first - 1; r <= by.last; ++r) {
      const int64_t part = part_of(r, r == by.first - 1);
      if (part < 0 || part >= parts) return 6;
      if (!made_here) continue;
      if (!read.insert(part).second) return 7;
      const auto found = left.find(part);
      if (found == left.end() || found->second != e) return 8;
    }
  }
  return made_here && read.size() != left.size() ? 9 : 0;
}

// The workgroup's shape (wm, mt, wn, nt), the tiles and the ranges of a weight gradient.
extern "C" void rules_tiling(int32_t terms, int64_t slots, int32_t experts, int64_t width, int64_t out_width, int32_t* out) {
  const Tiling t = tiling_of(terms, slots, experts, width, out_width);
  const int32_t found[6] = {t.wm, t.mt, t.wn, t.nt, (int32_t)t.tiles(), t.ranges};
  for (int i = 0; i < 6; ++i) out[i] = found[i];
}
