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

// Whether sequence b, with the rows lo .. hi - 1 of `rows`, owns unit u; not where its offsets do not describe rows.
ZQ_HOST_DEVICE bool owns_unit(int64_t u, int64_t lo, int64_t hi, int64_t b, int size, int extra, int64_t rows) {
  return lo >= 0 && hi > lo && hi <= rows && unit_base(lo, b, size, extra) <= u && u < unit_base(hi, b + 1, size, extra);
}

// The first of the sequences `start`, start + step, .. that owns unit u, or -1.  `row_of(b)` gives cu[b].  (Where offsets fall, several may
// own one: the kernels take the first, so that it does not hang on their threads' order.)
template <typename F>
ZQ_HOST_DEVICE int unit_sequence(int64_t u, int B, int size, int extra, F row_of, int64_t rows = INT64_MAX, int start = 0, int step = 1) {
  for (int64_t b = start; b < B; b += step)
    if (owns_unit(u, row_of(static_cast<int>(b)), row_of(static_cast<int>(b + 1)), b, size, extra, rows)) return static_cast<int>(b);
  return -1;
}

}  // namespace kv
}  // namespace zq
