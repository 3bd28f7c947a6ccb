// The optimiser step (adam_device.hpp) on all of a model's tensors in one launch, with what the gradient norm has decided read from
// device memory: the factor that clips the gradients, whether the step is taken at all, and its number.
//
// Memory bound, as the step on one array is (adam.hip): a scalar with a gradient costs 12 bytes of reads and 12 to 14 of writes
// beside its gradient; the clipped gradient is never stored.  Scalars without a gradient keep every bit, but memory is read and
// written by the line: where one of the 32 scalars that share a line of each fp32 array has a gradient, all of the line is read
// and written back, past the caches where they do not hold it all from one step to the next.  Left out lane by lane, the
// stores leave lines with holes behind, which cost the memory more than whole ones (norm and step, fp32 gradients, three models in
// turn, whole lines and lane by lane: 58 M scalars of which 22 % have one 308 and 462 us, 408 M with 63 % 2.56 and 3.76 ms, 12 M with
// 95 % 73.6 and 74.3 us; 4, 16 or 64 lanes together instead of a line's eight: 310 to 311 us, 2.54 to 2.55 ms, 73.3 to 73.5 us).
// Lines in which no scalar has a gradient cost their gradient's bytes.
// (Step alone: 408 M scalars 2.3 ms, 12.2 GB in whole lines at 5.3 TB/s, where a large copy reaches 4.9; 12 M 63 us.)
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
  Place at;
  AdamArgs a;  // (inv_c1, inv_sqrt_c2: of the caller's step, where the device does not count)
};
using AdamList = TensorList<AdamItem, 48>;
static_assert(sizeof(AdamList) <= 4000, "with the other arguments at most 4 KB");

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

// Four scalars of an array of 32- or 16-bit scalars as they lie in memory (the latter in x and y), and as floats.  The load stands
// apart from the conversion: behind a branch on the type the compiler waits for what is used in it.
struct alignas(16) Bits4 {
  uint32_t w[4];
};
template <bool STREAM>
__device__ __forceinline__ Bits4 load_bits(const void* array, const uint32_t dtype, const uint64_t at) {
  Bits4 b;
  if (dtype == HG_F32) {
    b = __builtin_bit_cast(Bits4, load_vec<float, 4, STREAM>(static_cast<const float*>(array) + at));
  } else {
    const Scalars<uint16_t, 4> h = load_vec<uint16_t, 4, STREAM>(static_cast<const uint16_t*>(array) + at);
    const uint2 two = __builtin_bit_cast(uint2, h);
    b.w[0] = two.x;
    b.w[1] = two.y;
  }
  return b;
}
__device__ __forceinline__ Scalars<float, 4> to_floats(const Bits4& b, const uint32_t dtype) {
  Scalars<float, 4> f;
  if (dtype == HG_F32) {
    f = __builtin_bit_cast(decltype(f), b);
  } else if (dtype == HG_F16) {
    const Scalars<_Float16, 4> h = __builtin_bit_cast(decltype(h), make_uint2(b.w[0], b.w[1]));
#pragma unroll
    for (int j = 0; j < 4; ++j) f.v[j] = (float)h.v[j];
  } else {  // bf16: the upper half of a float
#pragma unroll
    for (int j = 0; j < 4; ++j) f.v[j] = __uint_as_float(j & 1 ? b.w[j / 2] & 0xffff0000u : b.w[j / 2] << 16);
  }
  return f;
}
__device__ __forceinline__ void store_zeros(void* array, const uint32_t dtype, const uint64_t at) {
  if (dtype == HG_F32)
    store_vec<float, 4>(static_cast<float*>(array) + at, Scalars<float, 4>{});
  else
    store_vec<uint16_t, 4>(static_cast<uint16_t*>(array) + at, Scalars<uint16_t, 4>{});
}
__device__ __forceinline__ void store_copy(void* array, const uint32_t dtype, const uint64_t at, const Scalars<float, 4>& p) {
  if (dtype == HG_F16) {
    Scalars<_Float16, 4> h;
#pragma unroll
    for (int j = 0; j < 4; ++j) h.v[j] = (_Float16)p.v[j];
    store_vec<_Float16, 4>(static_cast<_Float16*>(array) + at, h);
  } else {
    Scalars<__bf16, 4> h;
#pragma unroll
    for (int j = 0; j < 4; ++j) h.v[j] = (__bf16)p.v[j];
    store_vec<__bf16, 4>(static_cast<__bf16*>(array) + at, h);
  }
}

// Which arrays are read past the caches.  kState: values and moments, where a step's arrays are more than kResidentBytes: beyond
// that they do not survive until the next step (norm and step, three models in turn, of 4.5 M scalars, 81 MB each, 33.4 us past
// the caches and 29.9 through them; 6 M, 108 MB, 40.5 and 40.8; 12 M, 220 MB, 73.6 and 82.5; 14 M, 252 MB, 83.2 and 94.0.  One model of
// 12 M with nothing else running 73.3 and 71.2; in a clipped training step of 2^18 points, whose other passes need the caches, 317
// both ways, and with 58 M scalars 550 and 597).
// kAll: the gradients as well, where the norm has read them past the caches (kCacheBytes).
enum class Reach { kNone, kState, kAll };
constexpr uint64_t kResidentBytes = 96u << 20;

// Scalars [begin, end) of one tensor.  taken: the step is taken; else only the gradient is cleared, where asked to.
template <bool ZERO_GRAD, Reach REACH>
__device__ __forceinline__ void step_span(const AdamItem& it, const AdamArgs& a, const float scale, const bool taken, const uint64_t begin,
                                          const uint64_t end) {
  void* const grad = it.grad;
  void* const copy = it.st.p16;
  float *const p = it.st.p32, *const m = it.st.m, *const v = it.st.v;
  const uint32_t n = (uint32_t)(end - begin), n4 = n / 4, gt = it.at.dtype, ct = it.at.copy_dtype;
  // (two or eight vectors ahead instead of four: 74.2 and 76.5 us for 73.6 on 12 M scalars, norm included)
  for_vectors<4, kListThreads>(n4, threadIdx.x, [&](const uint32_t q0, auto many) __attribute__((always_inline)) {
    constexpr int K = decltype(many)::value;
    Bits4 bits[K];
    Scalars<float, 4> g[K], pp[K], mm[K], vv[K];
    bool any[K], run[K];
#pragma unroll
    for (int k = 0; k < K; ++k) bits[k] = load_bits<REACH == Reach::kAll>(grad, gt, begin + (q0 + k * kListThreads) * 4);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint64_t at = begin + (q0 + k * kListThreads) * 4;
      g[k] = to_floats(bits[k], gt);
      any[k] = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) any[k] |= g[k].v[j] != 0.0f;
      const bool near = (__ballot(any[k]) >> (threadIdx.x & 56) & 0xff) != 0;  // eight lanes: a cache line of each fp32 array
      run[k] = taken && (near || a.l2 != 0.0f);
      if (run[k]) {
        pp[k] = load_vec<float, 4, REACH != Reach::kNone>(p + at);
        mm[k] = load_vec<float, 4, REACH != Reach::kNone>(m + at);
        vv[k] = load_vec<float, 4, REACH != Reach::kNone>(v + at);
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint64_t at = begin + (q0 + k * kListThreads) * 4;
      if (run[k]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float h = step_gradient(g[k].v[j], scale, a.l2, pp[k].v[j]);
          if (h != 0.0f) adam_scalar(a, h, mm[k].v[j], vv[k].v[j], pp[k].v[j]);
        }
        store_vec<float, 4>(m + at, mm[k]);
        store_vec<float, 4>(v + at, vv[k]);
        store_vec<float, 4>(p + at, pp[k]);
        if (copy) store_copy(copy, ct, at, pp[k]);
      }
      if (ZERO_GRAD && any[k]) store_zeros(grad, gt, at);
    }
  });
  if (threadIdx.x < n - n4 * 4) {  // fewer than four scalars
    const uint64_t at = begin + n4 * 4 + threadIdx.x;
    const float raw = gt == HG_F32   ? static_cast<const float*>(grad)[at]
                      : gt == HG_F16 ? (float)static_cast<const _Float16*>(grad)[at]
                                     : (float)static_cast<const __bf16*>(grad)[at];
    if (taken) {
      float pp = p[at];
      const float h = step_gradient(raw, scale, a.l2, pp);
      if (h != 0.0f) {
        float mm = m[at], vv = v[at];
        adam_scalar(a, h, mm, vv, pp);
        m[at] = mm;
        v[at] = vv;
        p[at] = pp;
        if (copy && ct == HG_F16) static_cast<_Float16*>(copy)[at] = (_Float16)pp;
        if (copy && ct == HG_BF16) static_cast<__bf16*>(copy)[at] = (__bf16)pp;
      }
    }
    if (ZERO_GRAD && raw != 0.0f) {
      if (gt == HG_F32)
        static_cast<float*>(grad)[at] = 0.0f;
      else
        static_cast<uint16_t*>(grad)[at] = 0;
    }
  }
}

template <bool ZERO_GRAD, Reach REACH>
__global__ __launch_bounds__(kListThreads) void adam_list(const AdamList list, const float grad_scale,
                                                          hashgrid_grad_stats* __restrict__ stats) {
  // every workgroup reads `step`, one writes `steps`: no workgroup reads what another writes
  const uint32_t step = stats ? stats->step : 1u;
  const float scale = stats ? grad_scale * stats->factor : grad_scale;
  if (stats && step && blockIdx.x == 0 && threadIdx.x == 0) stats->steps = step;
  if (!ZERO_GRAD && step == 0) return;
  float beta1 = -1.0f, beta2 = -1.0f, inv_c1 = 0.0f, inv_sqrt_c2 = 0.0f;  // of the step that the device has counted
  for (Spans at(list, blockIdx.x, gridDim.x); at.within(list); at.advance()) {
    const AdamItem& it = list.item[at.i];
    AdamArgs a = it.a;
    if (stats && step) {
      if (a.beta1 != beta1 || a.beta2 != beta2) {
        beta1 = a.beta1;
        beta2 = a.beta2;
        // both at a time, one in the even lanes and one in the odd ones: the kernel's first loads wait for this
        const bool odd = threadIdx.x & 1;
        double c = 1.0 - power((double)(odd ? beta2 : beta1), step);
        if (odd) c = sqrt(c);
        const float inv = (float)(1.0 / c);
        inv_c1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(inv), 0));
        inv_sqrt_c2 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(inv), 1));
      }
      a.inv_c1 = inv_c1;
      a.inv_sqrt_c2 = inv_sqrt_c2;
    }
    step_span<ZERO_GRAD, REACH>(it, a, scale, step != 0, at.begin, at.end);
  }
}

using StepKernel = void (*)(AdamList, float, hashgrid_grad_stats*);
const StepKernel kernels[2][3] = {
    {adam_list<false, Reach::kNone>, adam_list<false, Reach::kState>, adam_list<false, Reach::kAll>},
    {adam_list<true, Reach::kNone>, adam_list<true, Reach::kState>, adam_list<true, Reach::kAll>}};

bool misaligned(const void* p, uint32_t bytes) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

}  // namespace
}  // namespace hg

extern "C" hg_status hashgrid_adam_steps(uint32_t n_tensors, const hashgrid_adam_tensor* tensors, float grad_scale, int zero_grad,
                                         uint32_t step, hashgrid_grad_stats* stats, void* stream) {
  if (n_tensors > HG_MAX_TENSORS) return HG_ERR_UNSUPPORTED;
  if ((n_tensors && !tensors) || (step == 0) == (stats == nullptr)) return HG_ERR_INVALID_ARG;
  if (!(grad_scale > 0.0f && grad_scale < INFINITY) || (reinterpret_cast<uintptr_t>(stats) & 15)) return HG_ERR_INVALID_ARG;
  uint64_t scalars = 0, bytes = 0;  // (of the gradients)
  for (uint32_t i = 0; i < n_tensors; ++i) {
    const hashgrid_adam_tensor& t = tensors[i];
    if (!hg::adam_config_ok(t.cfg) || t.grad_dtype > HG_BF16 || (t.params_half && t.half_dtype != HG_F16 && t.half_dtype != HG_BF16))
      return HG_ERR_INVALID_ARG;
    if (t.n_scalars > HG_MAX_TENSOR_SCALARS) return HG_ERR_UNSUPPORTED;
    if (t.n_scalars == 0) continue;
    if (hg::misaligned(t.params_master, 4) || hg::misaligned(t.m, 4) || hg::misaligned(t.v, 4) ||
        hg::misaligned(t.grad, hg::dtype_bytes(t.grad_dtype)) || (t.params_half && hg::misaligned(t.params_half, 2)))
      return HG_ERR_INVALID_ARG;
    const uint64_t size = t.n_scalars * hg::dtype_bytes(t.grad_dtype), four = 4 * t.n_scalars;
    if (hg::in_stats(t.params_master, four, stats) || hg::in_stats(t.m, four, stats) || hg::in_stats(t.v, four, stats) ||
        hg::in_stats(t.grad, size, stats) || (t.params_half && hg::in_stats(t.params_half, 2 * t.n_scalars, stats)))
      return HG_ERR_INVALID_ARG;
    scalars += t.n_scalars;
    bytes += size;
  }
  if (scalars > HG_MAX_TENSOR_SCALARS) return HG_ERR_UNSUPPORTED;
  if (scalars == 0 && !stats) return HG_OK;
  const bool clash = hg::ranges_clash<5>(n_tensors, [&](int kind, uint32_t i) {
    const hashgrid_adam_tensor& t = tensors[i];
    const void* const array = kind == 0 ? t.params_master : kind == 1 ? t.m : kind == 2 ? t.v : kind == 3 ? t.grad : t.params_half;
    const uintptr_t begin = reinterpret_cast<uintptr_t>(array);
    const uint64_t each = kind < 3 ? 4 : kind == 3 ? hg::dtype_bytes(t.grad_dtype) : t.params_half ? 2 : 0;
    return hg::Range{begin, begin + t.n_scalars * each, kind != 3 || zero_grad};
  });
  if (clash) return HG_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const uint64_t all = bytes + 14 * scalars;  // with value, moments and copy
  const hg::Reach reach = bytes > hg::kCacheBytes ? hg::Reach::kAll : all > hg::kResidentBytes ? hg::Reach::kState : hg::Reach::kNone;
  // Half as many workgroups where that still leaves each some ten units: with fewer streams open the memory is faster (norm and
  // step on 58 M scalars 308 us with 512 and 321 with 1024, on 12 M 74.8 and 73.6, on 7 M 46.6 and 45.9).
  const uint32_t most = scalars > (32u << 20) ? hg::kMaxListGroups / 2 : hg::kMaxListGroups;
  hg::AdamList list;
  list.unit = hg::step_unit_for(scalars);
  uint32_t i = 0;
  do {  // (once for an empty list too where the device counts the steps)
    list.n_items = list.units = 0;
    for (; i < n_tensors && list.n_items < (uint32_t)hg::AdamList::kMost; ++i) {
      const hashgrid_adam_tensor& t = tensors[i];
      if (t.n_scalars == 0) continue;
      list.item[list.n_items++] =
          hg::AdamItem{hg::AdamState{t.params_master, static_cast<_Float16*>(t.params_half), t.m, t.v}, t.grad,
                       hg::next_place(list, t.n_scalars, t.grad_dtype, t.half_dtype & 15),
                       step ? hg::adam_args(t.cfg, step)
                            : hg::AdamArgs{t.cfg.lr, t.cfg.beta1, t.cfg.beta2, t.cfg.eps, t.cfg.l2_reg, 0.0f, 0.0f}};
    }
    if (list.n_items == 0 && scalars) break;
    const uint32_t groups = hg::groups_of(list.units, most);
    const auto kernel = hg::kernels[zero_grad ? 1 : 0][(int)reach];
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(hg::kListThreads), 0, s, list, grad_scale, stats);
  } while (i < n_tensors);
  return hipGetLastError() == hipSuccess ? HG_OK : HG_ERR_DEVICE;
}
