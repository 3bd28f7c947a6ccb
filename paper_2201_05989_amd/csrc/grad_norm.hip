// The Euclidean norm over the gradients of all of a model's tensors, and clipping by it.
//
//   S = sum of g^2 over all tensors,  norm = grad_scale sqrt(S),  factor = min(1, max_norm / norm), 0 where S is not finite
//
// Memory bound: every scalar is read once for the norm.  The squares are summed in 64 bits from the first addition on: an fp32
// square leaves fp32's range from 2e19 upwards and loses bits below 1e-19, both of which gradients reach (the latter
// where losses are means), and a sum of 2^29 of them would lose some more; 64-bit multiply-adds run at the rate of the 32-bit
// ones here, two instructions a scalar beside 4 bytes of memory traffic.  Every workgroup leaves its sum in an array and the
// last one adds those up in the order of their places: the norm of the same arrays is the same bits every time.
// (408 M scalars: fp16 121 us, 6.7 TB/s; fp32 236 us, 6.9 TB/s, where a large copy reaches 4.9.  12 M fp32 scalars
// 11.7 us, of which 4 are the launch, the first loads and the meeting of the workgroups at the end.)
//
// Clipping reads and writes what it cannot be spared once more (58 M fp16 scalars into other arrays: 54.8 us, 23 for the norm
// and 32, 7.3 TB/s, the second reading from the last-level cache), and nothing where the factor is 1 and it is in place.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "hashgrid.h"
#include "tensor_list.hpp"

namespace hg {

namespace {

struct NormItem {
  const void* data;
  Place at;
};
using NormList = TensorList<NormItem, 240>;

struct ClipItem {
  const void* data;
  void* out;
  Place at;
};
using ClipList = TensorList<ClipItem, 160>;
static_assert(kMaxListGroups <= HG_GRAD_NORM_GROUPS, "a place for every workgroup's sum");
static_assert(sizeof(NormList) <= 4000 && sizeof(ClipList) <= 4000, "with the other arguments at most 4 KB");

// Squares of scalars [begin, end): the share of one of a team's THREADS threads.
template <bool STREAM, int THREADS, typename T>
__device__ __forceinline__ double sum_squares(const T* __restrict__ g, const uint64_t begin, const uint64_t end, const uint32_t thread) {
  constexpr int V = 16 / sizeof(T);
  const uint32_t n = (uint32_t)(end - begin), n_vec = n / V;
  const T* base = g + begin;
  double sum[2] = {0.0, 0.0};
  for_vectors<4, THREADS>(n_vec, thread, [&](const uint32_t q, auto many) __attribute__((always_inline)) {
    constexpr int K = decltype(many)::value;
    Scalars<T, V> x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = load_vec<T, V, STREAM>(base + (q + k * THREADS) * V);
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const double d = (double)(float)x[k].v[j];
        sum[j & 1] = fma(d, d, sum[j & 1]);
      }
    }
  });
  const uint32_t at = n_vec * V + thread;
  if (at < n) {
    const double d = (double)(float)base[at];
    sum[0] = fma(d, d, sum[0]);
  }
  return sum[0] + sum[1];
}

// The workgroup's sum; `part`: one double a wave.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_down(v, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) total += part[w];
  return total;
}

// Returns the factor.
__device__ __forceinline__ float write_norm(hashgrid_grad_stats* st, const double sum, const float grad_scale, const float max_norm) {
  const double norm = (double)grad_scale * sqrt(sum);
  const bool finite = isfinite(sum);
  st->norm = (float)norm;
  const float factor = !finite ? 0.0f : (norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f);
  st->factor = factor;
  st->step = finite ? st->steps + 1u : 0u;
  return factor;
}

// Whether this workgroup is the last of the launch to come here, in thread 0.  Two levels: a counter serves one addition after
// the other, and a thousand on one word would queue up for longer than the sums take.
__device__ __forceinline__ bool last_to_arrive(uint32_t (*arrived)[32]) {
  constexpr uint32_t kGates = HG_GRAD_NORM_GATES - 1;
  auto last_of = [](uint32_t* counter, const uint32_t n) {
    if (__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != n - 1) return false;
    __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next call
    return true;
  };
  if (gridDim.x <= 2 * kGates) return last_of(arrived[kGates], gridDim.x);
  const uint32_t gate = blockIdx.x % kGates;
  const uint32_t through = (gridDim.x - gate + kGates - 1) / kGates;  // workgroups of this gate
  return last_of(arrived[gate], through) && last_of(arrived[kGates], kGates);
}

// Sums of one launch, on top of those that the `prior` workgroups of the list's earlier launches left (more than
// NormList::kMost tensors take several).  The last workgroup of the list's last launch (`groups` > 0: as many have left sums)
// adds them all up, in the order of their places.
template <bool STREAM>
__global__ __launch_bounds__(kListThreads) void norm(const NormList list, hashgrid_grad_stats* __restrict__ st, const uint32_t prior,
                                                     const uint32_t groups, const float grad_scale, const float max_norm) {
  __shared__ double part[kListThreads / 64];
  __shared__ bool last;
  double sum = 0.0;
  for (Spans at(list, blockIdx.x, gridDim.x); at.within(list); at.advance()) {
    const NormItem& it = list.item[at.i];
    with_type(it.at.dtype, [&](auto* t) __attribute__((always_inline)) {
      using T = std::remove_pointer_t<decltype(t)>;
      sum += sum_squares<STREAM, kListThreads>(static_cast<const T*>(it.data), at.begin, at.end, threadIdx.x);
    });
  }
  double total = block_sum<kListThreads>(sum, part);
  if (threadIdx.x == 0) {
    if (blockIdx.x < prior) total += st->partials[blockIdx.x];
    last = groups == 1;
    if (groups != 1) __hip_atomic_store(&st->partials[blockIdx.x], total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (groups > 1) {
      // The sum is performed before this workgroup is counted: it, the counters and the last one's loads are device-scope
      // atomics, which meet behind the caches, so nothing else has to be ordered.  (With release and acquire on the
      // counter, which write this XCD's L2 back, the norm of 12 M scalars takes 35 us for 11.7, 408 M fp16 160 for 121; with a
      // launch of their own for the last sums 13.1 and 123, and 4.5 M scalars 9.1 for 7.9.)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      last = last_to_arrive(st->arrived);
    }
  }
  if (groups == 0) return;
  __syncthreads();
  if (!last) return;
  if (groups > 1) {
    constexpr uint32_t kEach = HG_GRAD_NORM_GROUPS / kListThreads;
    double left[kEach];  // all on their way at once
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
      const uint32_t i = k * kListThreads + threadIdx.x;
      left[k] = __hip_atomic_load(&st->partials[i < groups ? i : 0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    sum = 0.0;
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) sum += k * kListThreads + threadIdx.x < groups ? left[k] : 0.0;
    total = block_sum<kListThreads>(sum, part);
  }
  if (threadIdx.x == 0) write_norm(st, total, grad_scale, max_norm);
}

template <int THREADS, typename T>
__device__ __forceinline__ void scale_span(const T* g, T* out, const float factor, const uint64_t begin, const uint64_t end,
                                           const uint32_t thread) {
  constexpr int V = 16 / sizeof(T);
  const uint32_t n = (uint32_t)(end - begin), n_vec = n / V;
  const T* from = g + begin;
  T* to = out + begin;
  // factor 0 also where the norm is not finite: 0, not 0 * infinity.  An fp16 product is rounded once (the compiler takes the
  // instruction that multiplies fp16 by fp32 into fp16), a bf16 one to fp32 first, 2^-24 beside the 2^-8 of its type.
  auto scaled = [&](const T x) { return factor == 0.0f ? (T)0.0f : (T)((float)x * factor); };
  for_vectors<4, THREADS>(n_vec, thread, [&](const uint32_t q, auto many) __attribute__((always_inline)) {
    constexpr int K = decltype(many)::value;
    Scalars<T, V> x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = load_vec<T, V, true>(from + (q + k * THREADS) * V);
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) x[k].v[j] = scaled(x[k].v[j]);
      store_vec<T, V>(to + (q + k * THREADS) * V, x[k]);
    }
  });
  const uint32_t at = n_vec * V + thread;
  if (at < n) to[at] = scaled(from[at]);
}

__global__ __launch_bounds__(kListThreads) void clip(const ClipList list, const float* __restrict__ factor_at) {
  const float factor = *factor_at;
  for (Spans at(list, blockIdx.x, gridDim.x); at.within(list); at.advance()) {
    const ClipItem& it = list.item[at.i];
    if (factor == 1.0f && it.data == it.out) continue;  // in place, nothing to clip
    with_type(it.at.dtype, [&](auto* t) __attribute__((always_inline)) {
      using T = std::remove_pointer_t<decltype(t)>;
      scale_span<kListThreads>(static_cast<const T*>(it.data), static_cast<T*>(it.out), factor, at.begin, at.end, threadIdx.x);
    });
  }
}

// Norm, and clipping where `clipped`, of a list that one workgroup is enough for: its sixteen waves are the teams, with a unit each at
// the most.  (Norm of 3 K scalars in three tensors 2.7 us, in several workgroups 4.3; clipped 3.8, in two launches 6.7.  With two units
// a wave 32 K scalars would take 4.4 us for the 4.5 of several workgroups, clipped 6.9 for 6.8, and 32 tensors of 100 3.5 for 4.5, clipped
// 5.5 for 7.0, which this rule gives away.  GPU time of calls one after the other, in a graph.)
constexpr int kSmallThreads = 1024;
__global__ __launch_bounds__(kSmallThreads) void small_list(const ClipList list, hashgrid_grad_stats* __restrict__ st, const bool clipped,
                                                            const float grad_scale, const float max_norm) {
  __shared__ double part[kSmallThreads / 64];
  __shared__ float s_factor;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  double sum = 0.0;
  for (Spans at(list, wave, kSmallThreads / 64); at.within(list); at.advance()) {
    const ClipItem& it = list.item[at.i];
    with_type(it.at.dtype, [&](auto* t) __attribute__((always_inline)) {
      using T = std::remove_pointer_t<decltype(t)>;
      sum += sum_squares<false, 64>(static_cast<const T*>(it.data), at.begin, at.end, lane);
    });
  }
  const double total = block_sum<kSmallThreads>(sum, part);
  if (threadIdx.x == 0) s_factor = write_norm(st, total, grad_scale, max_norm);
  if (!clipped) return;
  __syncthreads();  // every scalar has been read, too
  const float factor = s_factor;
  for (Spans at(list, wave, kSmallThreads / 64); at.within(list); at.advance()) {
    const ClipItem& it = list.item[at.i];
    if (factor == 1.0f && it.data == it.out) continue;
    with_type(it.at.dtype, [&](auto* t) __attribute__((always_inline)) {
      using T = std::remove_pointer_t<decltype(t)>;
      scale_span<64>(static_cast<const T*>(it.data), static_cast<T*>(it.out), factor, at.begin, at.end, lane);
    });
  }
}

bool bad_array(const void* p, uint32_t dtype) {
  return p == nullptr || dtype > HG_BF16 || (reinterpret_cast<uintptr_t>(p) & (dtype_bytes(dtype) - 1)) != 0;
}

// The arguments that both calls have; the list's scalars and bytes, all tensors together.
hg_status check_grads(uint32_t n, const hashgrid_grad* grads, float grad_scale, float max_norm, const hashgrid_grad_stats* stats,
                      uint64_t* scalars, uint64_t* bytes) {
  if (n > HG_MAX_TENSORS) return HG_ERR_UNSUPPORTED;
  if ((n && !grads) || stats == nullptr || (reinterpret_cast<uintptr_t>(stats) & 15)) return HG_ERR_INVALID_ARG;
  if (!(grad_scale > 0.0f && grad_scale < INFINITY) || !(max_norm >= 0.0f)) return HG_ERR_INVALID_ARG;
  *scalars = *bytes = 0;
  for (uint32_t i = 0; i < n; ++i) {
    if (grads[i].dtype > HG_BF16 || (grads[i].n_scalars && bad_array(grads[i].data, grads[i].dtype))) return HG_ERR_INVALID_ARG;
    if (grads[i].n_scalars > HG_MAX_TENSOR_SCALARS) return HG_ERR_UNSUPPORTED;
    *scalars += grads[i].n_scalars;
    *bytes += grads[i].n_scalars * dtype_bytes(grads[i].dtype);
  }
  if (*scalars > HG_MAX_TENSOR_SCALARS) return HG_ERR_UNSUPPORTED;
  for (uint32_t i = 0; i < n; ++i)
    if (in_stats(grads[i].data, grads[i].n_scalars * dtype_bytes(grads[i].dtype), stats)) return HG_ERR_INVALID_ARG;
  return HG_OK;
}

// The next descriptions of the list from tensor i on, as many as List holds.
template <typename List, typename Make>
void take(List& list, uint32_t& i, const uint32_t n_tensors, const hashgrid_grad* grads, Make&& make) {
  list.n_items = list.units = 0;
  for (; i < n_tensors && list.n_items < (uint32_t)List::kMost; ++i) {
    if (grads[i].n_scalars == 0) continue;
    list.item[list.n_items++] = make(i, next_place(list, grads[i].n_scalars, grads[i].dtype));
  }
}

// The norm, and clipping (`clipped`) into `out` or in place; arguments checked.
hg_status launch(uint32_t n_tensors, const hashgrid_grad* grads, const bool clipped, void* const* out, const uint64_t scalars,
                 const uint64_t bytes, const float grad_scale, const float max_norm, hashgrid_grad_stats* stats, hipStream_t s) {
  auto clip_item = [&](const uint32_t i, const Place& at) { return ClipItem{grads[i].data, out ? out[i] : grads[i].data, at}; };
  constexpr uint32_t kWaves = kSmallThreads / 64;
  uint64_t small_units = 0;
  for (uint32_t i = 0; i < n_tensors && small_units <= kWaves; ++i) small_units += units_of(grads[i].n_scalars, kWaveUnit);
  if (small_units <= kWaves) {  // (so at most kWaves tensors have any scalars)
    ClipList list;
    list.unit = kWaveUnit;
    uint32_t i = 0;
    take(list, i, n_tensors, grads, clip_item);
    hipLaunchKernelGGL(small_list, dim3(1), dim3(kSmallThreads), 0, s, list, stats, clipped, grad_scale, max_norm);
    return hipGetLastError() == hipSuccess ? HG_OK : HG_ERR_DEVICE;
  }
  NormList norms;
  norms.unit = unit_for(scalars);
  uint32_t i = 0, prior = 0;
  while (i < n_tensors) {
    take(norms, i, n_tensors, grads, [&](const uint32_t k, const Place& at) { return NormItem{grads[k].data, at}; });
    const uint32_t now = groups_of(norms.units), all = now > prior ? now : prior;
    hipLaunchKernelGGL(bytes > kCacheBytes ? norm<true> : norm<false>, dim3(now), dim3(kListThreads), 0, s, norms, stats, prior,
                       i < n_tensors ? 0u : all, grad_scale, max_norm);
    prior = all;
  }
  ClipList list;
  list.unit = norms.unit;
  for (i = 0; clipped && i < n_tensors;) {
    take(list, i, n_tensors, grads, clip_item);
    if (list.n_items) hipLaunchKernelGGL(clip, dim3(groups_of(list.units)), dim3(kListThreads), 0, s, list, &stats->factor);
  }
  return hipGetLastError() == hipSuccess ? HG_OK : HG_ERR_DEVICE;
}

}  // namespace
}  // namespace hg

extern "C" hg_status hashgrid_grad_norm(uint32_t n_tensors, const hashgrid_grad* grads, float grad_scale, float max_norm,
                                        hashgrid_grad_stats* stats, void* stream) {
  uint64_t scalars, bytes;
  const hg_status ok = hg::check_grads(n_tensors, grads, grad_scale, max_norm, stats, &scalars, &bytes);
  if (ok != HG_OK) return ok;
  return hg::launch(n_tensors, grads, false, nullptr, scalars, bytes, grad_scale, max_norm, stats, static_cast<hipStream_t>(stream));
}

extern "C" hg_status hashgrid_clip_grads(uint32_t n_tensors, const hashgrid_grad* grads, void* const* out, float grad_scale,
                                         float max_norm, hashgrid_grad_stats* stats, void* stream) {
  uint64_t scalars, bytes;
  const hg_status ok = hg::check_grads(n_tensors, grads, grad_scale, max_norm, stats, &scalars, &bytes);
  if (ok != HG_OK) return ok;
  for (uint32_t i = 0; out && i < n_tensors; ++i)
    if (grads[i].n_scalars && (hg::bad_array(out[i], grads[i].dtype) ||
                               hg::in_stats(out[i], grads[i].n_scalars * hg::dtype_bytes(grads[i].dtype), stats)))
      return HG_ERR_INVALID_ARG;
  const bool clash = hg::ranges_clash<2>(n_tensors, [&](int kind, uint32_t i) {
    const uintptr_t size = grads[i].n_scalars * hg::dtype_bytes(grads[i].dtype);
    const uintptr_t from = reinterpret_cast<uintptr_t>(grads[i].data), to = out ? reinterpret_cast<uintptr_t>(out[i]) : from;
    if (kind == 0) return hg::Range{to, to + size, true};
    return to == from ? hg::Range{} : hg::Range{from, from + size, false};
  });
  if (clash) return HG_ERR_INVALID_ARG;
  return hg::launch(n_tensors, grads, true, out, scalars, bytes, grad_scale, max_norm, stats, static_cast<hipStream_t>(stream));
}
