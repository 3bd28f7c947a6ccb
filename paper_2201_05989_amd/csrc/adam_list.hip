// The optimiser step (adam_device.hpp) on all of a model's tensors in one launch, with what the gradient norm has decided read from
// device memory: the factor that clips the gradients, whether the step is taken at all, and its number.
//
// Memory bound, as the step on one array is (adam.hip): a scalar with a gradient costs 12 bytes of reads and 12 to 14 of writes
// beside its gradient, four in a row without one cost their gradient's bytes.  The clipped gradient is never stored.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "hashgrid.h"
#include "adam_device.hpp"
#include "tensor_list.hpp"

namespace hg {
namespace {

struct AdamItem {
  AdamState st;  // (p16: 16-bit copy of either type)
  void* grad;
  uint64_t n;
  uint32_t first, grad_dtype, copy_dtype;
  AdamArgs a;  // (inv_c1, inv_sqrt_c2: of the caller's step, where the device does not count)
};
using AdamList = TensorList<AdamItem, 36>;
static_assert(sizeof(AdamList) <= 3840, "with the other arguments at most 4 KB");

// beta^t by repeated squaring: 2 log2(t) roundings of 64 bits
__device__ __forceinline__ double power(double beta, uint32_t t) {
  double r = 1.0;
  for (; t; t >>= 1) {
    if (t & 1) r *= beta;
    beta *= beta;
  }
  return r;
}

// A scalar's gradient as the step uses it, 0 where it is to be passed over.
__device__ __forceinline__ float step_gradient(const float g, const float scale, const float l2, const float p) {
  return l2 != 0.0f ? fmaf(l2, p, g * scale) : g * scale;
}

// Scalars [begin, end) of one tensor.  taken: the step is taken; else only the gradient is cleared, where asked to.
template <typename G, typename C, bool ZERO_GRAD>
__device__ __forceinline__ void step_span(const AdamItem& it, const AdamArgs& a, const float scale, const bool taken, const uint64_t begin,
                                          const uint64_t end) {
  G* const grad = static_cast<G*>(it.grad) + begin;
  float* const p = it.st.p32 + begin;
  float* const m = it.st.m + begin;
  float* const v = it.st.v + begin;
  C* const copy = it.st.p16 ? reinterpret_cast<C*>(it.st.p16) + begin : nullptr;
  const uint64_t n4 = (end - begin) / 4;
  for (uint64_t q = threadIdx.x; q < n4; q += kListThreads) {
    const Vec<G, 4> raw = load_vec<G, 4>(grad + q * 4);
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) any |= (float)raw.v[j] != 0.0f;
    if (taken && (any || a.l2 != 0.0f)) {
      Vec<float, 4> pp = load_vec<float, 4>(p + q * 4), mm = load_vec<float, 4>(m + q * 4), vv = load_vec<float, 4>(v + q * 4);
      Vec<C, 4> cc;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float g = step_gradient((float)raw.v[j], scale, a.l2, pp.v[j]);
        if (g != 0.0f) adam_scalar(a, g, mm.v[j], vv.v[j], pp.v[j]);
        cc.v[j] = (C)pp.v[j];
      }
      store_vec<float, 4>(m + q * 4, mm);
      store_vec<float, 4>(v + q * 4, vv);
      store_vec<float, 4>(p + q * 4, pp);
      if (copy) store_vec<C, 4>(copy + q * 4, cc);
    }
    if (ZERO_GRAD && any) store_vec<G, 4>(grad + q * 4, Vec<G, 4>{});
  }
  const uint64_t at = n4 * 4 + threadIdx.x;
  if (at < end - begin) {
    const float raw = (float)grad[at];
    if (taken) {
      float pp = p[at];
      const float g = step_gradient(raw, scale, a.l2, pp);
      if (g != 0.0f) {
        float mm = m[at], vv = v[at];
        adam_scalar(a, g, mm, vv, pp);
        m[at] = mm;
        v[at] = vv;
        p[at] = pp;
        if (copy) copy[at] = (C)pp;
      }
    }
    if (ZERO_GRAD && raw != 0.0f) grad[at] = (G)0.0f;
  }
}

template <bool ZERO_GRAD>
__global__ __launch_bounds__(kListThreads) void adam_list(const AdamList list, const float grad_scale,
                                                          hashgrid_grad_stats* __restrict__ stats) {
  // every workgroup reads `step`, one writes `steps`: no workgroup reads what another writes
  const uint32_t step = stats ? stats->step : 1u;
  const float scale = stats ? grad_scale * stats->factor : grad_scale;
  if (stats && step && blockIdx.x == 0 && threadIdx.x == 0) stats->steps = step;
  if (!ZERO_GRAD && step == 0) return;
  for_spans(list, [&](const AdamItem& it, const uint64_t begin, const uint64_t end) {
    AdamArgs a = it.a;
    if (stats && step) {
      a.inv_c1 = (float)(1.0 / (1.0 - power((double)a.beta1, step)));
      a.inv_sqrt_c2 = (float)(1.0 / sqrt(1.0 - power((double)a.beta2, step)));
    }
    with_type(it.grad_dtype, [&](auto* g) {
      using G = std::remove_pointer_t<decltype(g)>;
      if (it.copy_dtype == HG_F16)
        step_span<G, _Float16, ZERO_GRAD>(it, a, scale, step != 0, begin, end);
      else
        step_span<G, __bf16, ZERO_GRAD>(it, a, scale, step != 0, begin, end);
    });
  });
}

bool misaligned(const void* p, uint32_t bytes) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

}  // namespace
}  // namespace hg

extern "C" hg_status hashgrid_adam_steps(uint32_t n_tensors, const hashgrid_adam_tensor* tensors, float grad_scale, int zero_grad,
                                         uint32_t step, hashgrid_grad_stats* stats, void* stream) {
  if (n_tensors > HG_MAX_TENSORS) return HG_ERR_UNSUPPORTED;
  if ((n_tensors && !tensors) || (step == 0) == (stats == nullptr)) return HG_ERR_INVALID_ARG;
  if (!(grad_scale > 0.0f && grad_scale < INFINITY) || (reinterpret_cast<uintptr_t>(stats) & 15)) return HG_ERR_INVALID_ARG;
  hg::Range ranges[5 * HG_MAX_TENSORS];
  uint32_t n_ranges = 0;
  uint64_t units = 0;
  for (uint32_t i = 0; i < n_tensors; ++i) {
    const hashgrid_adam_tensor& t = tensors[i];
    if (!hg::adam_config_ok(t.cfg) || t.grad_dtype > HG_BF16 || (t.params_half && t.half_dtype != HG_F16 && t.half_dtype != HG_BF16))
      return HG_ERR_INVALID_ARG;
    if (t.n_scalars > HG_MAX_TENSOR_SCALARS) return HG_ERR_UNSUPPORTED;
    if (t.n_scalars == 0) continue;
    if (hg::misaligned(t.params_master, 4) || hg::misaligned(t.m, 4) || hg::misaligned(t.v, 4) ||
        hg::misaligned(t.grad, hg::dtype_bytes(t.grad_dtype)) || (t.params_half && hg::misaligned(t.params_half, 2)))
      return HG_ERR_INVALID_ARG;
    auto add = [&](const void* p, uint32_t bytes, bool written) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(p);
      ranges[n_ranges++] = hg::Range{at, at + t.n_scalars * bytes, written};
    };
    add(t.params_master, 4, true);
    add(t.m, 4, true);
    add(t.v, 4, true);
    add(t.grad, hg::dtype_bytes(t.grad_dtype), zero_grad != 0);
    if (t.params_half) add(t.params_half, 2, true);
    units += hg::units_of(t.n_scalars);
  }
  if (units > UINT32_MAX) return HG_ERR_UNSUPPORTED;
  if (n_ranges == 0 && !stats) return HG_OK;
  if (hg::ranges_clash(ranges, n_ranges)) return HG_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hg::AdamList list;
  uint32_t i = 0;
  do {  // (once for an empty list too where the device counts the steps)
    list.n_items = list.units = 0;
    for (; i < n_tensors && list.n_items < (uint32_t)hg::AdamList::kMost; ++i) {
      const hashgrid_adam_tensor& t = tensors[i];
      if (t.n_scalars == 0) continue;
      list.item[list.n_items++] = hg::AdamItem{hg::AdamState{t.params_master, static_cast<_Float16*>(t.params_half), t.m, t.v}, t.grad,
                                               t.n_scalars, list.units, t.grad_dtype, t.half_dtype,
                                               hg::adam_args(t.cfg, step ? step : 1u)};
      list.units += (uint32_t)hg::units_of(t.n_scalars);
    }
    if (list.n_items == 0 && n_ranges) break;
    const uint32_t groups = hg::deal_out(list);
    if (zero_grad)
      hipLaunchKernelGGL(hg::adam_list<true>, dim3(groups), dim3(hg::kListThreads), 0, s, list, grad_scale, stats);
    else
      hipLaunchKernelGGL(hg::adam_list<false>, dim3(groups), dim3(hg::kListThreads), 0, s, list, grad_scale, stats);
  } while (i < n_tensors);
  return hipGetLastError() == hipSuccess ? HG_OK : HG_ERR_DEVICE;
}
