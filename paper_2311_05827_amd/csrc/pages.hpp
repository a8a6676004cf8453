// What a cache's table says, for host and device: no other header is needed.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define ACCEPT_BOTH __host__ __device__ inline
#else
#define ACCEPT_BOTH inline
#endif

namespace accept {

struct Pages {
  int32_t count;        // of pages
  int32_t table_pages;  // of a sequence in the table
  int32_t shift;        // page_size = 1 << shift
  int32_t kv_heads;
};
// Is there a place `j` in a sequence's table; is what the table says there a page; and then, which row of head_size values
// in a cache it is (of key head `head`).
ACCEPT_BOTH bool has_place(const Pages& p, int64_t j) { return j >= 0 && (j >> p.shift) < p.table_pages; }
ACCEPT_BOTH bool is_page(const Pages& p, int32_t page) { return page >= 0 && page < p.count; }
ACCEPT_BOTH int64_t cache_row(const Pages& p, int32_t page, int64_t j, int head) {
  return ((int64_t(page) * p.kv_heads + head) << p.shift) + (j & ((int64_t(1) << p.shift) - 1));
}
// Places are counted in 32 bits, and a table may have all but 16 of 2^31 of them: a sum of one with a tile's or a unit's size does not fit.
// Place key0 + by, or the last one of `keys` where that is none (0 <= key0 < keys).
ACCEPT_BOTH int32_t place_at(int32_t key0, int32_t by, int32_t keys) { return by < keys - key0 ? key0 + by : keys - 1; }
// Where the places of units that end before unit `unit1`, `unit` places each, end among the first `some`.
ACCEPT_BOTH int32_t units_end(int32_t unit1, int32_t unit, int32_t some) {
  const int64_t end = int64_t(unit1) * unit;
  return end < some ? int32_t(end) : some;
}

}  // namespace accept
