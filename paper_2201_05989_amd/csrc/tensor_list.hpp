// Lists of arrays as kernel arguments: what the kernels that pass over all of a model's tensors at once share (the
// gradient norm, clipping, the optimiser step).
//
// The arrays' descriptions travel by value in the kernel's arguments, so that a call neither copies nor allocates device
// memory and can be recorded into a graph.  The arrays are cut into units of kUnit scalars, numbered through all arrays of the
// list, and every workgroup takes an equal run of them: arrays of any sizes, one scalar or 2^32 and more, give workgroups the
// same work to within a unit.  Scalars are read and written 16 bytes a lane wherever the array starts: global loads and
// stores of this target need no more than the element's own alignment.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hashgrid.h"

namespace hg {

constexpr int kListThreads = 256;
constexpr uint32_t kUnit = 2048;  // scalars: 8 a thread, one 16-byte access of a 16-bit type, two of fp32

// N descriptions of type Item (with members n and first: scalars, and the first unit)
template <typename Item, int N>
struct TensorList {
  static constexpr int kMost = N;
  uint32_t n_items;
  uint32_t units;          // of all items together
  uint32_t per, longer;    // a workgroup's units: per + 1 for the first `longer` of them, per for the others
  Item item[N];
};

// Calls f(item, begin, end) for every stretch of scalars that is this workgroup's.
template <typename Item, int N, typename Fn>
__device__ __forceinline__ void for_spans(const TensorList<Item, N>& list, Fn&& f) {
  const uint32_t b = blockIdx.x;
  uint32_t u = b * list.per + (b < list.longer ? b : list.longer);
  const uint32_t end = u + list.per + (b < list.longer ? 1u : 0u);
  if (u >= end) return;
  // the item of unit u: as many items as start at or before it, less one; each lane looks at one of 64
  uint32_t i = 0;
#pragma unroll
  for (int at = 0; at < N; at += 64) {
    const uint32_t k = at + (threadIdx.x & 63);
    i += __popcll(__ballot(k < list.n_items && list.item[k < N ? k : N - 1].first <= u));
  }
  i = __builtin_amdgcn_readfirstlane(i) - 1;
  while (u < end) {
    const Item& it = list.item[i];
    const uint32_t next = i + 1 < list.n_items ? list.item[i + 1].first : list.units;
    const uint32_t stop = end < next ? end : next;
    const uint64_t from = (uint64_t)(u - it.first) * kUnit, to = (uint64_t)(stop - it.first) * kUnit;
    f(it, from, to < it.n ? to : it.n);
    u = stop;
    ++i;
  }
}

// Workgroups for a list of `units`: two thousand, eight a compute unit, keep the memory busy; fewer where there is less.
constexpr uint32_t kMaxListGroups = 2048;
template <typename List>
uint32_t deal_out(List& list) {
  const uint32_t groups = list.units < kMaxListGroups ? (list.units ? list.units : 1) : kMaxListGroups;
  list.per = list.units / groups;
  list.longer = list.units % groups;
  return groups;
}

inline uint64_t units_of(uint64_t n) { return n / kUnit + (n % kUnit != 0); }

inline uint32_t dtype_bytes(uint32_t dtype) { return dtype == HG_F32 ? 4 : 2; }

// V scalars of type T at any address that T may have
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
  T v[V];
};
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T* p) {
  return *reinterpret_cast<const Vec<T, V>*>(p);
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, V>& v) {
  *reinterpret_cast<Vec<T, V>*>(p) = v;
}

// Calls f with a null pointer of the C++ type behind an hg_dtype.
template <typename Fn>
__device__ __forceinline__ void with_type(const uint32_t dtype, Fn&& f) {
  if (dtype == HG_F32)
    f(static_cast<float*>(nullptr));
  else if (dtype == HG_F16)
    f(static_cast<_Float16*>(nullptr));
  else
    f(static_cast<__bf16*>(nullptr));
}

// Byte ranges of one call's arrays, to refuse calls in which something is written that another array of the call shares.
struct Range {
  uintptr_t begin, end;
  bool written;
};
// Sorts; true where a written range meets another one.
bool ranges_clash(Range* r, uint32_t n);

}  // namespace hg
