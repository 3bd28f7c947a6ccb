// Compiled for the host by tests/test_host_tensor_list.py: the check for arrays that share memory and the places of a list of arrays,
// as csrc/tensor_list.hpp computes them for the kernels.
#include <stdint.h>

#include "tensor_list.hpp"

extern "C" {

// begin, end, written: [kinds][n]
int32_t clash2(uint32_t n, const uint64_t* begin, const uint64_t* end, const uint8_t* written) {
  return hg::ranges_clash<2>(n, [&](int k, uint32_t i) {
    return hg::Range{(uintptr_t)begin[k * n + i], (uintptr_t)end[k * n + i], written[k * n + i] != 0};
  });
}
int32_t clash5(uint32_t n, const uint64_t* begin, const uint64_t* end, const uint8_t* written) {
  return hg::ranges_clash<5>(n, [&](int k, uint32_t i) {
    return hg::Range{(uintptr_t)begin[k * n + i], (uintptr_t)end[k * n + i], written[k * n + i] != 0};
  });
}

// The units of arrays of n_scalars[i] > 0 scalars: first[i] and last[i] of each; returns the units of all.
uint32_t places(uint32_t n, const uint64_t* n_scalars, uint32_t unit, uint32_t* first, uint32_t* last) {
  struct {
    uint32_t units, unit;
  } list{0, unit};
  for (uint32_t i = 0; i < n; ++i) {
    const hg::Place at = hg::next_place(list, n_scalars[i], i % 3, i % 2);
    if (at.dtype != i % 3 || at.copy_dtype != i % 2) return 0;
    first[i] = at.first;
    last[i] = at.last;
  }
  return list.units;
}

uint32_t unit_for(uint64_t scalars) { return hg::unit_for(scalars); }
uint32_t step_unit_for(uint64_t scalars) { return hg::step_unit_for(scalars); }
}
