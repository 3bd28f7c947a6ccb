// Lists of arrays as kernel arguments: what the kernels that pass over all of a model's tensors at once share (the
// gradient norm, clipping, the optimiser step).
//
// The arrays' descriptions travel by value in the kernel's arguments, so that a call neither copies nor allocates device
// memory and can be recorded into a graph.  The arrays are cut into units of some thousand scalars, numbered through all arrays of
// the list, and dealt out to the workgroups in turn: arrays of any sizes, one scalar or 2^32 and more, give workgroups the same
// work to within a unit, and what the chip reads at a time lies together (in turn 2.56 ms, a run of its own for each workgroup
// 2.64: norm and optimiser step on 408 M fp32 scalars; on 12 M 73.6 and 76.7 us).  Scalars are read and
// written 16 bytes a lane wherever the array starts: global loads and stores of this target need no more than the
// element's own alignment.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "hashgrid.h"
#include "array_ranges.hpp"

namespace hg {

constexpr int kListThreads = 256;
// Scalars a unit: from 8 a thread, which give the most workgroups something to do, to 32, several loads on their way at a time.
constexpr uint32_t kSmallUnit = 2048, kLargeUnit = 8192;
constexpr uint32_t kWaveUnit = 1024;  // where a team is one wave: 16 a lane
// Workgroups at most, four a compute unit: as many as run at a time in the optimiser step, whose four vectors ahead take the
// registers.  Norm and clipping, of which more fit, read no faster with more (norm of 408 M fp16 scalars 121 us with 1024 and 128
// with 2048, of 12 M fp32 11.7 and 12.9).
constexpr uint32_t kMaxListGroups = 1024;

// What every description of an array begins its place in the list with: its first unit, and the scalars of its last one (the
// others are full), with the types beside them.  Short, because 4 KB of arguments hold the list.
struct Place {
  uint32_t first;
  uint32_t last : 16, dtype : 4, copy_dtype : 4;
};

// N descriptions of type Item, with a Place `at`
template <typename Item, int N>
struct TensorList {
  static constexpr int kMost = N;
  uint32_t n_items;
  uint32_t units;  // of all items together
  uint32_t unit;   // scalars of one
  Item item[N];
};

// A team's way through its stretches of scalars: units first, first + teams, ...; a team is a workgroup, or one of its waves.
//   for (Spans at(list, first, teams); at.within(list); at.advance()) ... list.item[at.i], scalars at.begin .. at.end-1
// (The kernels' loops are written out with it: a function that took their bodies as a lambda made the compiler copy the list
// from the arguments to every thread's private memory as soon as the body kept anything from one stretch to the next.)
struct Spans {
  uint32_t u, teams, i, next;
  uint64_t begin, end;

  template <typename List>
  __device__ __forceinline__ Spans(const List& list, const uint32_t first, const uint32_t n_teams)
      : u(first), teams(n_teams), i(0), next(0) {}
  template <typename List>
  __device__ __forceinline__ bool within(const List& list) {
    if (u >= list.units) return false;
    if (u >= next) {
      // the item of unit u: as many items as start at or before it, less one; each lane looks at one of 64.  (Item by item a step
      // over a hundred small tensors costs 10 us.)
      uint32_t before = 0;
      auto look = [&](const uint32_t k) __attribute__((always_inline)) {
        before += __popcll(__ballot(k < list.n_items && list.item[k < List::kMost ? k : 0].at.first <= u));
      };
      look(threadIdx.x & 63);
      if (list.n_items > 64) {  // (short lists are not to wait for arguments that they do not use)
#pragma unroll
        for (int at = 64; at < List::kMost; at += 64) look(at + (threadIdx.x & 63));
      }
      i = __builtin_amdgcn_readfirstlane(before) - 1;
      next = i + 1 < list.n_items ? list.item[i + 1].at.first : list.units;
    }
    begin = (uint64_t)(u - list.item[i].at.first) * list.unit;
    end = begin + (u + 1 == next ? list.item[i].at.last : list.unit);
    return true;
  }
  __device__ __forceinline__ void advance() { u += teams; }
};

inline uint64_t units_of(uint64_t n, uint32_t unit) { return n / unit + (n % unit != 0); }

// The place of the next array of the list, of n > 0 scalars.
template <typename List>
Place next_place(List& list, uint64_t n, uint32_t dtype, uint32_t copy_dtype = 0) {
  Place at;
  at.first = list.units;
  at.last = (uint32_t)((n - 1) % list.unit) + 1;
  at.dtype = dtype;
  at.copy_dtype = copy_dtype;
  list.units += (uint32_t)units_of(n, list.unit);
  return at;
}

// Scalars a unit for a list of so many.  Norm and clipping: the smallest unit with which a workgroup has two at the most, and the
// large one beyond that (4.5 M fp32 scalars: norm 7.8 us with units of 4096 as with 2048, clipped 12.6 and 12.5; 12 M 11.7 with 8192,
// 12.0 with 4096 and 12.1 with 2048; 408 M fp16 121 with 8192, 120 with 4096 and 187 with 2048).
inline uint32_t unit_for(uint64_t scalars) {
  uint32_t unit = kSmallUnit;
  while (unit < kLargeUnit && scalars > 2ull * unit * kMaxListGroups) unit *= 2;
  return unit;
}
// The optimiser step, with four arrays to a scalar, fills the memory with small units for longer (norm and step on 6 M scalars 40.8
// us with 2048, 40.9 with 4096 and 42.7 with 8192; 12 M 72.8, 74.2 and 73.4; 408 M between 2.53 and 2.56 ms with each).
inline uint32_t step_unit_for(uint64_t scalars) { return scalars > (8u << 20) ? kLargeUnit : kSmallUnit; }

// Whether a list's gradients are too many for the last-level cache to hold from the norm's reading to the next: both then
// pass by the caches.  (Measured on either side: the norm of 408 M fp16 gradients 121 us passing by and 135 through the caches, fp32,
// 1.6 GB, 236 and 266; norm and optimiser step on the latter 2.56 ms and 2.53; on 58 M fp32, 232 MB, 342 us and 308, on 12 M 79 and 73.6.)
constexpr uint64_t kCacheBytes = 256u << 20;

inline uint32_t groups_of(uint32_t units, uint32_t most = kMaxListGroups) { return units < most ? (units ? units : 1) : most; }

inline uint32_t dtype_bytes(uint32_t dtype) { return dtype == HG_F32 ? 4 : 2; }

// V scalars of type T at any address that T may have.  STREAM: nothing will read them again soon (non-temporal).
template <typename T, int V>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <typename T, int V>
struct Scalars {
  T v[V];
};
template <typename T, int V, bool STREAM>
__device__ __forceinline__ Scalars<T, V> load_vec(const T* p) {
  const auto* at = reinterpret_cast<const typename VecOf<T, V>::type*>(p);
  if constexpr (STREAM)
    return __builtin_bit_cast(Scalars<T, V>, __builtin_nontemporal_load(at));
  else
    return __builtin_bit_cast(Scalars<T, V>, *at);
}
// Every store here is of that kind (clipping 58 M fp16 scalars into other arrays 54.8 us, with plain stores 77.3; norm and step on 408 M
// 2.56 ms and 2.71, on 12 M 73.6 us and 79.7).
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const Scalars<T, V>& v) {
  __builtin_nontemporal_store(__builtin_bit_cast(typename VecOf<T, V>::type, v), reinterpret_cast<typename VecOf<T, V>::type*>(p));
}

// Calls f(first, std::integral_constant<int, K>) for vectors first, first + T, ... (K of them), over vectors 0 .. n-1 for the T
// threads of a team: K = kAhead as long as all threads have that many, so that the loads in f stand side by side with no
// branch between them (behind one the compiler waits for each), then what is left.
template <int kAhead, int T, typename Fn>
__device__ __forceinline__ void for_vectors(const uint32_t n, const uint32_t thread, Fn&& f) {
  uint32_t q = 0;
  for (; q + kAhead * T <= n; q += kAhead * T) f(q + thread, std::integral_constant<int, kAhead>{});
  if (q + 2 * T <= n) {
    f(q + thread, std::integral_constant<int, 2>{});
    q += 2 * T;
  }
  for (q += thread; q < n; q += T) f(q, std::integral_constant<int, 1>{});
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

}  // namespace hg
