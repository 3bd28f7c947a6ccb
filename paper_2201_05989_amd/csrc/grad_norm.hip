// The Euclidean norm over the gradients of all of a model's tensors, and clipping by it.
//
//   S = sum of g^2 over all tensors,  norm = grad_scale sqrt(S),  factor = min(1, max_norm / norm), 0 where S is not finite
//
// Memory bound: every scalar is read once for the norm.  The squares are summed in 64 bits from the first addition on: an fp32
// square leaves fp32's range from 2e19 upwards and loses bits below 1e-19, both of which gradients reach (the latter
// where losses are means), and a sum of 2^29 of them would lose some more; 64-bit multiply-adds run at the rate of the 32-bit
// ones here, two instructions a scalar beside 4 bytes of memory traffic.  Every workgroup leaves its sum in an array and
// one workgroup adds those up in a fixed order: the norm of the same arrays is the same bits every time.
#include <hip/hip_runtime.h>
#include <math.h>
#include <algorithm>
#include <stdint.h>

#include "hashgrid.h"
#include "tensor_list.hpp"

namespace hg {

bool ranges_clash(Range* r, const uint32_t n) {
  std::sort(r, r + n, [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t any = 0, written = 0;  // ends of the ranges before this one
  for (uint32_t i = 0; i < n; ++i) {
    if (r[i].begin < (r[i].written ? any : written)) return true;
    any = std::max(any, r[i].end);
    if (r[i].written) written = std::max(written, r[i].end);
  }
  return false;
}

namespace {

struct NormItem {
  const void* data;
  uint64_t n;
  uint32_t first, dtype;
};
using NormList = TensorList<NormItem, 128>;

struct ClipItem {
  const void* data;
  void* out;
  uint64_t n;
  uint32_t first, dtype;
};
using ClipList = TensorList<ClipItem, 64>;

// Squares of scalars [begin, end), this thread's share: kAhead 16-byte loads on their way at a time.
template <typename T>
__device__ __forceinline__ double sum_squares(const T* __restrict__ g, const uint64_t begin, const uint64_t end) {
  constexpr int V = 16 / sizeof(T), kAhead = 4;
  const uint64_t n_vec = (end - begin) / V;
  const T* base = g + begin;
  double sum[2] = {0.0, 0.0};
  for (uint64_t q = threadIdx.x; q < n_vec; q += kAhead * kListThreads) {
    Vec<T, V> x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint64_t at = q + k * kListThreads;
      x[k] = load_vec<T, V>(base + (at < n_vec ? at : q) * V);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool there = q + k * kListThreads < n_vec;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const double d = there ? (double)(float)x[k].v[j] : 0.0;
        sum[j & 1] = fma(d, d, sum[j & 1]);
      }
    }
  }
  const uint64_t at = n_vec * V + threadIdx.x;
  if (at < end - begin) {
    const double d = (double)(float)base[at];
    sum[0] = fma(d, d, sum[0]);
  }
  return sum[0] + sum[1];
}

// The workgroup's sum, in thread 0; `part`: one double a wave.
__device__ __forceinline__ double block_sum(double v, double* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_down(v, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int w = 0; w < kListThreads / 64; ++w) total += part[w];
  return total;
}

__device__ __forceinline__ void write_norm(hashgrid_grad_stats* st, const double sum, const float grad_scale, const float max_norm) {
  const double norm = (double)grad_scale * sqrt(sum);
  const bool finite = isfinite(sum);
  st->norm = (float)norm;
  st->factor = !finite ? 0.0f : (norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f);
  st->step = finite ? st->steps + 1u : 0u;
}

// Sums of one launch, on top of those that the `prior` workgroups of the list's earlier launches left (more than
// NormList::kMost tensors take several).  A single workgroup that has seen everything ends the job itself: `alone`.
__global__ __launch_bounds__(kListThreads) void norm_partials(const NormList list, hashgrid_grad_stats* __restrict__ st,
                                                              const uint32_t prior, const bool alone, const float grad_scale,
                                                              const float max_norm) {
  __shared__ double part[kListThreads / 64];
  double sum = 0.0;
  for_spans(list, [&](const NormItem& it, const uint64_t begin, const uint64_t end) {
    with_type(it.dtype, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      sum += sum_squares(static_cast<const T*>(it.data), begin, end);
    });
  });
  double total = block_sum(sum, part);
  if (threadIdx.x != 0) return;
  if (blockIdx.x < prior) total += st->partials[blockIdx.x];
  if (alone)
    write_norm(st, total, grad_scale, max_norm);
  else
    st->partials[blockIdx.x] = total;
}

__global__ __launch_bounds__(kListThreads) void norm_finish(hashgrid_grad_stats* __restrict__ st, const uint32_t groups,
                                                            const float grad_scale, const float max_norm) {
  __shared__ double part[kListThreads / 64];
  double sum = 0.0;
  for (uint32_t i = threadIdx.x; i < groups; i += kListThreads) sum += st->partials[i];
  const double total = block_sum(sum, part);
  if (threadIdx.x == 0) write_norm(st, total, grad_scale, max_norm);
}

template <typename T>
__device__ __forceinline__ void scale_span(const T* g, T* out, const float factor, const uint64_t begin, const uint64_t end) {
  constexpr int V = 16 / sizeof(T), kAhead = 4;
  const uint64_t n_vec = (end - begin) / V;
  const T* from = g + begin;
  T* to = out + begin;
  // factor 0 also where the norm is not finite: 0, not 0 * infinity
  auto scaled = [&](const T x) { return factor == 0.0f ? (T)0.0f : (T)((float)x * factor); };
  for (uint64_t q = threadIdx.x; q < n_vec; q += kAhead * kListThreads) {
    Vec<T, V> x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint64_t at = q + k * kListThreads;
      x[k] = load_vec<T, V>(from + (at < n_vec ? at : q) * V);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) x[k].v[j] = scaled(x[k].v[j]);
      if (q + k * kListThreads < n_vec) store_vec<T, V>(to + (q + k * kListThreads) * V, x[k]);
    }
  }
  const uint64_t at = n_vec * V + threadIdx.x;
  if (at < end - begin) to[at] = scaled(from[at]);
}

__global__ __launch_bounds__(kListThreads) void clip(const ClipList list, const float* __restrict__ factor_at) {
  const float factor = *factor_at;
  for_spans(list, [&](const ClipItem& it, const uint64_t begin, const uint64_t end) {
    if (factor == 1.0f && it.data == it.out) return;  // in place, nothing to clip
    with_type(it.dtype, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      scale_span(static_cast<const T*>(it.data), static_cast<T*>(it.out), factor, begin, end);
    });
  });
}

bool bad_array(const void* p, uint32_t dtype) {
  return p == nullptr || dtype > HG_BF16 || (reinterpret_cast<uintptr_t>(p) & (dtype_bytes(dtype) - 1)) != 0;
}

hg_status check_grads(uint32_t n, const hashgrid_grad* grads) {
  if (n > HG_MAX_TENSORS) return HG_ERR_UNSUPPORTED;
  if (n && !grads) return HG_ERR_INVALID_ARG;
  uint64_t units = 0;
  for (uint32_t i = 0; i < n; ++i) {
    if (grads[i].dtype > HG_BF16 || (grads[i].n_scalars && bad_array(grads[i].data, grads[i].dtype))) return HG_ERR_INVALID_ARG;
    if (grads[i].n_scalars > HG_MAX_TENSOR_SCALARS) return HG_ERR_UNSUPPORTED;
    units += units_of(grads[i].n_scalars);
  }
  return units > UINT32_MAX ? HG_ERR_UNSUPPORTED : HG_OK;
}

bool bad_stats(const hashgrid_grad_stats* st) { return st == nullptr || (reinterpret_cast<uintptr_t>(st) & 15) != 0; }

}  // namespace
}  // namespace hg

extern "C" hg_status hashgrid_grad_norm(uint32_t n_tensors, const hashgrid_grad* grads, float grad_scale, float max_norm,
                                        hashgrid_grad_stats* stats, void* stream) {
  const hg_status ok = hg::check_grads(n_tensors, grads);
  if (ok != HG_OK) return ok;
  if (hg::bad_stats(stats) || !(grad_scale > 0.0f && grad_scale < INFINITY) || !(max_norm >= 0.0f)) return HG_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hg::NormList list;
  uint32_t i = 0, prior = 0;
  bool alone = false;
  do {  // once for an empty list too: its norm is 0
    list.n_items = list.units = 0;
    for (; i < n_tensors && list.n_items < (uint32_t)hg::NormList::kMost; ++i) {
      if (grads[i].n_scalars == 0) continue;
      list.item[list.n_items++] = hg::NormItem{grads[i].data, grads[i].n_scalars, list.units, grads[i].dtype};
      list.units += (uint32_t)hg::units_of(grads[i].n_scalars);
    }
    const uint32_t groups = hg::deal_out(list);
    alone = groups == 1 && prior == 0 && i == n_tensors;
    hipLaunchKernelGGL(hg::norm_partials, dim3(groups), dim3(hg::kListThreads), 0, s, list, stats, prior, alone, grad_scale,
                       max_norm);
    if (groups > prior) prior = groups;
  } while (i < n_tensors);
  if (!alone) hipLaunchKernelGGL(hg::norm_finish, dim3(1), dim3(hg::kListThreads), 0, s, stats, prior, grad_scale, max_norm);
  return hipGetLastError() == hipSuccess ? HG_OK : HG_ERR_DEVICE;
}

extern "C" hg_status hashgrid_clip_grads(uint32_t n_tensors, const hashgrid_grad* grads, void* const* out,
                                         const hashgrid_grad_stats* stats, void* stream) {
  const hg_status ok = hg::check_grads(n_tensors, grads);
  if (ok != HG_OK) return ok;
  if (hg::bad_stats(stats)) return HG_ERR_INVALID_ARG;
  hg::Range ranges[2 * HG_MAX_TENSORS];
  uint32_t n_ranges = 0;
  for (uint32_t i = 0; i < n_tensors; ++i) {
    if (grads[i].n_scalars == 0) continue;
    if (out && hg::bad_array(out[i], grads[i].dtype)) return HG_ERR_INVALID_ARG;
    const uintptr_t bytes = grads[i].n_scalars * hg::dtype_bytes(grads[i].dtype);
    const uintptr_t from = reinterpret_cast<uintptr_t>(grads[i].data), to = out ? reinterpret_cast<uintptr_t>(out[i]) : from;
    ranges[n_ranges++] = hg::Range{to, to + bytes, true};
    if (to != from) ranges[n_ranges++] = hg::Range{from, from + bytes, false};
  }
  if (n_ranges == 0) return HG_OK;
  if (hg::ranges_clash(ranges, n_ranges)) return HG_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hg::ClipList list;
  for (uint32_t i = 0; i < n_tensors;) {
    list.n_items = list.units = 0;
    for (; i < n_tensors && list.n_items < (uint32_t)hg::ClipList::kMost; ++i) {
      if (grads[i].n_scalars == 0) continue;
      list.item[list.n_items++] = hg::ClipItem{grads[i].data, out ? out[i] : const_cast<void*>(grads[i].data), grads[i].n_scalars,
                                               list.units, grads[i].dtype};
      list.units += (uint32_t)hg::units_of(grads[i].n_scalars);
    }
    if (list.n_items == 0) break;
    const uint32_t groups = hg::deal_out(list);
    hipLaunchKernelGGL(hg::clip, dim3(groups), dim3(hg::kListThreads), 0, s, list, &stats->factor);
  }
  return hipGetLastError() == hipSuccess ? HG_OK : HG_ERR_DEVICE;
}
