// Sizes and limits of launches, in plain C++.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace himuon {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// Whether a launch of this many blocks (of `threads` each, in x) stays below 2^32 threads.
inline bool launchable(int64_t blocks, int threads) { return blocks <= (int64_t)(UINT32_MAX / (uint32_t)threads); }

// True if the product of two non-negative values stays below 2^62.
inline bool small_product(int64_t a, int64_t b) { return a == 0 || b <= (INT64_C(1) << 62) / a; }

}  // namespace himuon
