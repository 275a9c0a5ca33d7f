// The paged cache as the kernels see it: a row of a request is found through the request's list of pages.  The arithmetic is plain
// C++, so that it can be checked on a host.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define PK_HD __host__ __device__ __forceinline__
#else
#define PK_HD inline
#endif

namespace purekv {

// n / d for 0 <= n < 2^31 and a divisor known on the host: with s = ceil(log2 d) and m = floor(2^(31 + s) / d) + 1,
// m d - 2^(31 + s) <= d <= 2^s, so n m / 2^(31 + s) is above n / d by less than 1 / d.  m < 2^32, as d > 2^(s - 1).
struct FastDiv {
  uint32_t d, mul;
  int32_t shift;
  static FastDiv of(int32_t d) {
    int32_t s = 0;
    while ((int64_t(1) << s) < d) ++s;
    return {(uint32_t)d, (uint32_t)((uint64_t(1) << (31 + s)) / (uint32_t)d + 1), 31 + s};
  }
  PK_HD uint32_t quotient(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};

// Strides in bytes; K and V share them.  `table` [n_req, table_stride] and `seq_lens` [n_req] are device arrays.
struct PagedView {
  const int32_t* table;
  const int32_t* seq_lens;
  int64_t table_stride, page_stride, token_stride, head_stride;
  int32_t n_pages, max_pages;
  FastDiv page_size;

  // rows that a request's list of pages can hold, in 32 bits (a longer list's further rows are out of reach)
  PK_HD int32_t capacity() const {
    const int64_t c = (int64_t)max_pages * page_size.d;
    return c < INT32_MAX ? (int32_t)c : INT32_MAX;
  }
  // byte offset of row `row`'s head 0 in the pool, given its page; -1 if there is no such page
  PK_HD int64_t offset(int32_t page, uint32_t slot) const {
    return page >= 0 && page < n_pages ? (int64_t)page * page_stride + (int64_t)slot * token_stride : -1;
  }
  // the same from the request's list; -1 too for a row outside it
  PK_HD int64_t row_offset(const int32_t* list, int32_t row) const {
    if (row < 0 || row >= capacity()) return -1;
    const uint32_t p = page_size.quotient((uint32_t)row);
    return offset(list[p], (uint32_t)row - p * page_size.d);
  }
};

// Which request a packed row belongs to: the last r of 0 .. n_req - 1 with cu[r] <= t (cu does not decrease).  The caller checks
// cu[r] <= t < cu[r + 1].
PK_HD int32_t request_of(const int32_t* cu, int32_t n_req, int32_t t) {
  int32_t lo = 0, hi = n_req;
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

}  // namespace purekv
