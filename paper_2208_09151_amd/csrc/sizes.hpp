// Arithmetic on sizes, for sources with and without device code.
#pragma once

#include <cstdint>

namespace ginex {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace ginex
