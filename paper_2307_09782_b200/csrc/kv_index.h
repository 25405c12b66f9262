// Index arithmetic of the operators around the 8-bit cache: how a ragged batch is dealt out to blocks of threads.  Plain C++,
// so that it is tested without a GPU.
#pragma once

#include <cstdint>

#include "fp8_index.h"

namespace zq {
namespace kv {

// A batch of B sequences whose rows are cu[b] .. cu[b + 1] - 1 is cut into units of up to `size` rows, aligned to the
// sequences' own pages.  Sequence b owns the units unit_base(cu[b], b, ..) .. unit_base(cu[b + 1], b + 1, ..) - 1, more than it
// needs: `extra` is 1 where a sequence's rows begin at a unit's border, 2 where they may begin inside one.
ZQ_HOST_DEVICE int64_t unit_base(int64_t row, int64_t b, int size, int extra) { return row / size + b * extra; }

// The sequence that owns unit u.  `row_of(b)` gives cu[b]; they ascend.
template <typename F>
ZQ_HOST_DEVICE int unit_sequence(int64_t u, int B, int size, int extra, F row_of) {
  int lo = 0, hi = B - 1;  // the last b with unit_base(cu[b], b) <= u
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (unit_base(row_of(mid), mid, size, extra) <= u)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

}  // namespace kv
}  // namespace zq
