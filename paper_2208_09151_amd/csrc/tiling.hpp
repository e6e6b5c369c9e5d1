// How a weight gradient is cut: the workgroup's shape and the number of ranges.  Plain C++ for the host, which the tests
// compile as well, to know which kernel their sizes reach.
#pragma once

#include "sizes.hpp"
#include "slots.hpp"

namespace ginex {

// The workgroup's shape and the number of ranges by the sizes and the terms that a gradient is cut into.
struct Tiling {
  int32_t wm, mt, wn, nt;
  int64_t tiles_m, tiles_n;
  int32_t ranges;
  int64_t tiles() const { return tiles_m * tiles_n; }
  int64_t parts() const { return parts_of(ranges); }
};

inline Tiling tiling_of(int32_t terms, int64_t slots, int32_t experts, int64_t width, int64_t out_width) {
  Tiling t;
  const auto shape = [&](int wm, int mt, int wn, int nt) {
    t.wm = wm;
    t.mt = mt;
    t.wn = wn;
    t.nt = nt;
    t.tiles_m = ceil_div(width, wm * mt * 32);
    t.tiles_n = ceil_div(out_width, wn * nt * 32);
  };
  // One tile for all of up to 256 outputs where every CU has a thousand slots to go through: gradients and codes are
  // then taken apart once (and not once per tile of 128), but a CU has room for one such workgroup.  256 x 256 weights of
  // 128 experts from 40 000 slots: 60 us in these, 43 in small ones; 512 x 512 of 32 from 200 000: 151 and 190; 100 x 250
  // of 64 from 708 000: 99 and 113.  With 128 outputs and fewer there is nothing in it (54 and 54, 65 and 67 us).
  if (width > 128) shape(4, 2, 2, 4);
  else shape(2, 2, 4, 2);
  const bool large = out_width > 128 && slots * t.tiles() >= 256 * 1024;
  // Else 128 x 128, or as narrow as the layer: what a tile has too many of is read, cut and multiplied for nothing (us of a
  // call, here and below with inputs that are not in the caches, in tiles of 128 x 128 and of the layer's: f32, 1 000 000 slots,
  // 128 x 8: 104 and 52; 500 000 x 2 in 512 experts, 64 x 64: 123 and 86; 820 000, 256 x 47: 171 and 124; 820 000 x 2, 16 x 128:
  // 193 and 160; bf16, 820 000 x 2, 64 x 64: 89 and 70).
  if (!large) {
    if (out_width <= 32) shape(4, 1, 1, 1);
    else if (out_width <= 64 && width <= 64) shape(2, 1, 2, 1);
    else if (out_width <= 64) shape(2, 2, 2, 1);
    else if (width <= 64) shape(1, 2, 4, 1);
    else shape(2, 2, 2, 2);
    // With few slots what costs is the parts that the workgroups leave, and half a tile has half a part (bf16: 76 000 x 2,
    // 128 x 256 37.7 -> 36.7 us, 128 x 128 27.9 -> 25.7; but 500 000 x 2, 128 x 100 72 -> 81, 820 000 x 2, 256 x 100 183 -> 219.
    // f32: 76 000 x 2, 128 x 128 38.2 both, with parts in the caches 37 -> 33; but 128 x 256 55.7 -> 56.6 and 177 000 x 2,
    // 128 x 128 62.8 -> 64.1).  With many tiles there are few parts (bf16, 2000 x 2, 1024 x 1024: 27 -> 30).
    if (t.mt == 2 && t.nt == 2 && t.tiles() <= 16 && slots * t.tiles() < (terms == 1 ? 512 : 200) * 1024) {
      if (terms == 1) shape(1, 2, 4, 1);
      else shape(2, 2, 2, 1);
    }
  }
  // one large workgroup to a CU, or two small ones (of three that it has room for; with three: 65 -> 71 us).  Rounded down:
  // a layer of 129 to 255 large tiles has one range and leaves CUs idle, one of somewhat more takes a second round for few.
  int64_t ranges = (large ? 256 : 512) / t.tiles();
  // 128 slots at least, but a range for every expert of few slots (64 rows of 8 experts: 27 -> 14 us)
  const int64_t each = ceil_div(slots, STEP) < experts ? ceil_div(slots, STEP) : experts;
  const int64_t most = ceil_div(slots, 128) > each ? ceil_div(slots, 128) : each;
  ranges = ranges < most ? ranges : most;
  t.ranges = (int32_t)(ranges < 1 ? 1 : ranges);
  return t;
}

}  // namespace ginex
