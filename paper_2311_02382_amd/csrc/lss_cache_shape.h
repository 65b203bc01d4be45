// Which sizes a paged cache may have.  Plain C++ without a HIP header, so that a host program can go over them (tests/host/cache_shape_check.cpp).
#pragma once
#include <stdint.h>

namespace lss {

// A power of two: positions are split into page and slot by a shift
inline bool cache_page_ok(int64_t page_size) { return page_size >= 16 && page_size <= 65536 && (page_size & (page_size - 1)) == 0; }
// A sequence's table holds 2^30 tokens at most (positions are 32 bits); divided, since any max_pages may be asked for and the product need not fit 64 bits
inline bool cache_table_ok(int64_t max_pages, int64_t page_size) { return max_pages >= 1 && max_pages <= ((int64_t)1 << 30) / page_size; }

} // namespace lss
