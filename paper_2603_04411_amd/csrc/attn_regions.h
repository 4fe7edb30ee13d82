// Which memory the tensors of an attention call take, and whether two of them share some.  Host code without HIP.
#pragma once

#include <algorithm>
#include <cstdint>
#include <utility>

#include "../../include/dynakv.h"

namespace lmhead {

// From the first to the last of `count` places `by` bytes apart.  (Limits allow 2^70, which no memory holds: 2^61 then.)
inline int64_t spanned(int64_t by, int64_t count) {
  constexpr int64_t kMost = 1ll << 61;
  return count > 1 && by > kMost / (count - 1) ? kMost : by * (count - 1);
}

// Memory of a tensor of a call: pieces of `width` bytes from `p` on, in up to three dimensions with steps of their own (widest step last).
struct Region {
  uintptr_t p = 0;      // 0: there is none
  int64_t width = 0, extent = 0, step[3] = {}, size[3] = {};
  int dims = 0;
  bool nested = true;      // each step spans all of the dimensions within
  Region() = default;
  Region(const void* at, int64_t bytes) : p(reinterpret_cast<uintptr_t>(at)), width(bytes), extent(bytes) {}
  // n sequences, t slots and h heads with strides in units of `unit` bytes, rows of `row` bytes
  Region(const void* at, const attn_layout& x, int64_t n, int64_t t, int64_t h, int64_t row, int unit) : Region(at, row) {
    std::pair<int64_t, int64_t> d[3] = {{x.seq * unit, n}, {x.slot * unit, t}, {x.head * unit, h}};
    std::sort(d, d + 3);
    for (const auto& [by, count] : d) {
      if (count == 1 || by == 0) continue;
      nested = nested && by >= extent;
      extent += spanned(by, count);
      if (dims == 0 && by == width) width *= count;
      else step[dims] = by, size[dims++] = count;
    }
  }
  bool dense() const { return dims == 0; }
};

// Whether [x, y), relative to the region's dimensions below `dim`, meets a piece.
inline bool meets(const Region& r, int dim, int64_t x, int64_t y) {
  if (dim == 0) return x < r.width && y > 0;
  int64_t inner = r.width;
  for (int i = 0; i < dim - 1; ++i) inner += r.step[i] * (r.size[i] - 1);
  const int64_t by = r.step[dim - 1];
  // copies of the dimensions within that lie in part in [x, y): of three the middle one lies in it whole
  const int64_t first = std::max<int64_t>(0, x < inner ? 0 : (x - inner) / by + 1), last = std::min(r.size[dim - 1] - 1, y > 0 ? (y - 1) / by : -1);
  if (last - first >= 2) return true;
  for (int64_t k = first; k <= last; ++k)
    if (meets(r, dim - 1, x - k * by, y - k * by)) return true;
  return false;
}

// Whether two tensors share memory.  Of two with gaps only the same beginning is found out: heads of one buffer side by side are ordinary.
inline bool share(const Region& a, const Region& b) {
  if (!a.p || !b.p) return false;
  if (a.p == b.p) return true;
  if (a.p + a.extent <= b.p || b.p + b.extent <= a.p) return false;
  const Region &flat = a.dense() ? a : b, &other = a.dense() ? b : a;
  if (!flat.dense() || !other.nested) return false;
  const int64_t x = static_cast<int64_t>(flat.p - other.p);
  return meets(other, other.dims, x, x + flat.extent);
}

}  // namespace lmhead
