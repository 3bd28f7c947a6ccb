// Whether arrays of a call share memory that the call writes: the check that entry points which take many arrays begin with, on the host.
#pragma once

#include <algorithm>
#include <stdint.h>

#include "hashgrid.h"

namespace hg {

// Bytes of one array of a call; none where begin == end.
struct Range {
  uintptr_t begin, end;
  bool written;
};
// Whether an array shares memory with *stats, which the calls on lists write.
inline bool in_stats(const void* array, uint64_t bytes, const hashgrid_grad_stats* stats) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(array), st = reinterpret_cast<uintptr_t>(stats);
  return stats && bytes && at < st + sizeof(*stats) && st < at + bytes;
}
// Whether something is written that another array of the call shares: range_of(k, i) for k < KINDS kinds of arrays (values, gradients,
// ...) of n <= HG_MAX_TENSORS tensors.  Each kind in the order of its addresses, as the arrays mostly come, and then all kinds
// side by side; 2 KB of stack a kind.
template <int KINDS, typename RangeOf>
bool ranges_clash(const uint32_t n, RangeOf&& range_of) {
  uint16_t order[KINDS][HG_MAX_TENSORS];
  uint32_t count[KINDS] = {}, at[KINDS] = {};
  for (int k = 0; k < KINDS; ++k) {
    for (uint32_t i = 0; i < n; ++i) {
      const Range r = range_of(k, i);
      if (r.begin != r.end) order[k][count[k]++] = (uint16_t)i;
    }
    auto before = [&](uint16_t a, uint16_t b) { return range_of(k, a).begin < range_of(k, b).begin; };
    if (!std::is_sorted(order[k], order[k] + count[k], before)) std::sort(order[k], order[k] + count[k], before);
  }
  uintptr_t any = 0, written = 0;  // ends of the ranges before the next one
  for (;;) {
    int first = -1;
    Range r{};
    for (int k = 0; k < KINDS; ++k) {
      if (at[k] == count[k]) continue;
      const Range head = range_of(k, order[k][at[k]]);
      if (first < 0 || head.begin < r.begin) {
        first = k;
        r = head;
      }
    }
    if (first < 0) return false;
    if (r.begin < (r.written ? any : written)) return true;
    any = std::max(any, r.end);
    if (r.written) written = std::max(written, r.end);
    ++at[first];
  }
}

}  // namespace hg
