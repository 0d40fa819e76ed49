// Host-side checks that entry points of several files share.
#pragma once

#include <climits>
#include <cstdint>

// log2 of a page size, or -1
inline int page_shift(int32_t page_size) {
  for (int s = 5; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

// What is wrong with a pool of pages, or null
inline const char* pages_error(int32_t page_size, int32_t n_pages) {
  if (page_shift(page_size) < 0) return "page_size must be 32, 64, 128 or 256";
  if (n_pages < 1 || (long long)n_pages * page_size > INT_MAX) return "n_pages must be positive, n_pages * page_size below 2^31";
  return nullptr;
}

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
