// Rules of the 8-bit cache's host side that choose a launch by sizes alone.  Host code, no HIP.
#pragma once
#include <cstdint>

namespace k8 {

// Rows that a work-group of k8_append looks at: a power of two up to a block's 16, as many as leave 1000 to 2000 work-groups.
// What it costs to be wrong is not alike on the two sides.  Rows of one request, with more rows to a group: fewer work-groups that find no run to begin
// (8192 rows of 8 heads of 128, a layer, by 1 / 4 / 16: 71 / 24 / 10.7 us; 2000 by 1 / 4 / 8: 20 / 8.5 / 5.8).  Single rows of as many requests: a group's
// runs one after the other, which memory hides for the most part (1000 rows by 1 / 4: 14.6 / 16.7; 2000 by 1 / 8: 28.3 / 31.5; 4096 by 1 / 16: 53.5 / 58.0).
// So neither the requests' number nor the handle's capacity for them is asked.  Requests of 8 and of 20 rows are within 10% of their best.
inline int append_group(int64_t n_rows, int n_kv_heads) {
  const int64_t groups = n_rows * ((2 * n_kv_heads + 3) / 4);  // work-groups of one row
  return groups > 16384 ? 16 : groups > 6400 ? 8 : groups > 2666 ? 4 : groups > 1333 ? 2 : 1;
}

}  // namespace k8
