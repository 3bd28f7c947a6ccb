// One training iteration of the whole model (paper Section 4, "Training") behind one call: which kernels a batch
// takes, and nothing else.
//
//   large batches   forward, counting for the sort (where the batch does not give every compute unit a full workgroup the plain
//                   forward and the count pass); network forward + loss + network backward; scan (the network's
//                   Adam step and the loss sum ride along); scatter; accumulate + Adam on the tables
//   small batches   forward; network; atomic additions into an array of zeros; Adam on what they touched
//
// Five or six, and four launches of dependent kernels, each 2.6 us after the one before at the earliest and 3 us of the
// caller's time: one call per pass of the method took eleven and ten, and read and wrote the gradient of every table entry.
//
// With the gradients clipped by their norm (hashgrid_train_step_clipped) the optimiser has to wait for the last of them:
//
//   large batches   ... scan (the weights' gradients and the loss sum ride along); scatter; accumulate, the tables' gradient into
//                   memory; norm over both; Adam on both
//   small batches   forward; network; atomic additions; the weights' gradients and the loss sum; norm; Adam
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "hashgrid.h"
#include "hashgrid_internal.hpp"
#include "adam_device.hpp"
#include "array_ranges.hpp"

namespace hg {
namespace {

constexpr int kJobThreads = 256;
__global__ __launch_bounds__(kJobThreads) void side_job(const SideJob job) {
  __shared__ float4 part[kJobThreads];
  run_side_job<kJobThreads>(job, blockIdx.x, part);
}

// What clipping by the norm needs beyond the state: see hashgrid_train_step_clipped.
struct Clip {
  float max_norm;
  hashgrid_grad_stats* stats;
  float* grads;  // the tables' and the weights', one after the other
};

// Whether arrays of a clipped step share memory (x and target are read only).  hashgrid_adam_steps looks at its own, but by then the
// backward pass has added to tables_zeros: what is refused is to be refused before anything is launched.
bool arrays_clash(const hashgrid* hg, const hashgrid_train_state& st, const Clip& clip, uint64_t n_net, uint32_t B, const float* x,
                  const float* target, const void* y, const void* dLdy, const void* workspace, uint64_t workspace_bytes) {
  const uint64_t n_tab = hg->total * hg->cfg.F, n_y = (uint64_t)B * hg->cfg.L * hg->cfg.F;
  const struct {
    const void* at;
    uint64_t bytes;
  } array[] = {{x, 4ull * B * hg->cfg.d}, {target, 4ull * B * st.n_out}, {y, 2 * n_y}, {dLdy, 2 * n_y}, {workspace, workspace_bytes},
               {clip.stats, sizeof(hashgrid_grad_stats)}, {clip.grads, 4 * (n_tab + n_net)}, {st.tables, 4 * n_tab},
               {st.tables_half, 2 * n_tab}, {st.tables_m, 4 * n_tab}, {st.tables_v, 4 * n_tab}, {st.tables_zeros, 4 * n_tab},
               {st.weights, 4 * n_net}, {st.weights_half, 2 * n_net}, {st.weights_m, 4 * n_net}, {st.weights_v, 4 * n_net},
               {st.loss_sum, sizeof(double)}, {st.scratch, HG_TRAIN_SCRATCH_BYTES}};
  return ranges_clash<1>(sizeof(array) / sizeof(array[0]), [&](int, uint32_t i) {
    const uintptr_t begin = reinterpret_cast<uintptr_t>(array[i].at);
    return Range{begin, begin + array[i].bytes, i >= 2};
  });
}

// One iteration, with the optimiser step `step`; clip: with the gradients clipped, and the step that the device counts.
hg_status train_step(const hashgrid* hg, const hashgrid_train_state* st, uint32_t B, const float* x, const float* target, void* y,
                     void* dLdy, void* workspace, uint64_t workspace_bytes, uint32_t step, const Clip* clip, void* stream) {
  if (!hg || !st || (step == 0 && !clip)) return HG_ERR_INVALID_ARG;
  if (B == 0) return HG_OK;
  if (B > HG_MAX_BATCH) return HG_ERR_UNSUPPORTED;
  const hashgrid_config& c = hg->cfg;
  const uint32_t n_in = c.L * c.F, n_out = st->n_out;
  if (!x || !target || !y || !dLdy || n_out == 0) return HG_ERR_INVALID_ARG;
  if (c.param_dtype != HG_F16 || c.io_dtype != HG_F16 || c.grad_dtype != HG_F32 || !hg->lv.T_is_pow2 || c.d < 2 ||
      n_in % 8 != 0 || n_in > 64 || n_out > 32)
    return HG_ERR_UNSUPPORTED;
  if (st->loss != HG_LOSS_L2 && st->loss != HG_LOSS_MAPE) return HG_ERR_INVALID_ARG;
  if (!(fabsf(st->loss_scale) < INFINITY)) return HG_ERR_INVALID_ARG;
  if (!adam_config_ok(st->tables_adam) || !adam_config_ok(st->weights_adam) || st->tables_adam.l2_reg != 0.0f)
    return HG_ERR_INVALID_ARG;
  auto bad = [](const void* p, uintptr_t a) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; };
  if (bad(x, 4) || bad(target, 4) || bad(y, 16) || bad(dLdy, 16) || bad(st->tables, 16) || bad(st->tables_half, c.F * 2 > 8 ? c.F * 2 : 8) ||
      bad(st->tables_m, 16) || bad(st->tables_v, 16) || bad(st->tables_zeros, 16) || bad(st->weights, 4) ||
      bad(st->weights_half, 8) || bad(st->weights_m, 4) || bad(st->weights_v, 4) || bad(st->loss_sum, 8) ||
      bad(st->scratch, 16))
    return HG_ERR_INVALID_ARG;
  // the gradients here are those of the summed loss times loss_scale; the norm is the mean loss's
  const float mean = (float)(1.0 / ((double)st->loss_scale * B * n_out));
  if (clip && (bad(clip->stats, 16) || bad(clip->grads, 16) || !(clip->max_norm >= 0.0f) || !(mean > 0.0f && mean < INFINITY)))
    return HG_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);

  const uint64_t need = hashgrid_bwd_workspace_bytes(hg, B);
  const bool sorted = need != 0 && workspace && hashgrid_bwd_ws_pays(hg, B);
  if (sorted && (workspace_bytes < need || bad(workspace, 256))) return HG_ERR_INVALID_ARG;
  const uint32_t n1 = 64 * n_in, n2 = 64 * 64, n3 = 64 * n_out;
  if (clip && arrays_clash(hg, *st, *clip, n1 + n2 + n3, B, x, target, y, dLdy, workspace, sorted ? need : 0))
    return HG_ERR_INVALID_ARG;
  bool counted = false;
  hg_status rc = HG_ERR_UNSUPPORTED;
  if (sorted) {
    rc = hashgrid_encode_fwd_ws(hg, B, x, st->tables_half, y, workspace, workspace_bytes, stream);
    counted = rc == HG_OK;
  }
  if (rc == HG_ERR_UNSUPPORTED) rc = hashgrid_encode_fwd(hg, B, x, st->tables_half, y, stream);
  if (rc != HG_OK) return rc;

  const _Float16* W = static_cast<const _Float16*>(st->weights_half);
  SideJob job{};
  rc = launch_mlp_train(B, n_in, n_out, y, W, W + n1, W + n1 + n2, target, st->loss, st->loss_scale, dLdy, &job, st->scratch, s);
  if (rc != HG_OK) return rc;
  job.loss_sum = st->loss_sum;
  if (!clip) {
    job.w = AdamState{st->weights, static_cast<_Float16*>(st->weights_half), st->weights_m, st->weights_v};
    job.a = adam_args(st->weights_adam, step);
    const AdamArgs a = adam_args(st->tables_adam, step);
    const AdamState tab{st->tables, static_cast<_Float16*>(st->tables_half), st->tables_m, st->tables_v};
    if (sorted) return launch_binned_adam(hg, B, x, dLdy, st->tables_zeros, workspace, counted, a, tab, job, s);
    rc = hashgrid_encode_bwd(hg, B, x, dLdy, st->tables_zeros, stream);
    return rc != HG_OK ? rc : launch_adam_touched(hg, B, x, st->tables_zeros, a, tab, job, s);
  }
  // The sorted pass writes the tables' gradient in full, into memory of its own (cleared for sums behind the optimiser instead, as
  // atomic additions want it: 326 us a step for 317 at 2^18 points and 12 M table scalars, 586 for 550 with 58 M).
  const uint64_t n_tab = hg->total * c.F, n_net = n1 + n2 + n3;
  float* const net_grad = clip->grads + n_tab;
  float* const tab_grad = sorted ? clip->grads : st->tables_zeros;
  job.w = AdamState{net_grad, nullptr, nullptr, nullptr};
  if (sorted) {
    rc = launch_binned_job(hg, B, x, dLdy, tab_grad, workspace, counted, job, s);
  } else {
    rc = hashgrid_encode_bwd(hg, B, x, dLdy, tab_grad, stream);
    if (rc == HG_OK) {
      hipLaunchKernelGGL(side_job, dim3(job.blocks), dim3(kJobThreads), 0, s, job);
      rc = hipGetLastError() == hipSuccess ? HG_OK : HG_ERR_DEVICE;
    }
  }
  if (rc != HG_OK) return rc;
  const hashgrid_grad grads[2] = {{tab_grad, n_tab, HG_F32, 0}, {net_grad, n_net, HG_F32, 0}};
  rc = hashgrid_grad_norm(2, grads, mean, clip->max_norm, clip->stats, stream);
  if (rc != HG_OK) return rc;
  const hashgrid_adam_tensor both[2] = {
      {st->tables, st->tables_half, tab_grad, st->tables_m, st->tables_v, n_tab, HG_F32, HG_F16, st->tables_adam, 0},
      {st->weights, st->weights_half, net_grad, st->weights_m, st->weights_v, n_net, HG_F32, HG_F16, st->weights_adam, 0}};
  return hashgrid_adam_steps(2, both, 1.0f, !sorted, 0, clip->stats, stream);
}

}  // namespace
}  // namespace hg

extern "C" hg_status hashgrid_train_step(const hashgrid_t* hg, const hashgrid_train_state* st, uint32_t B, const float* x,
                                         const float* target, void* y, void* dLdy, void* workspace,
                                         uint64_t workspace_bytes, uint32_t step, void* stream) {
  return hg::train_step(hg, st, B, x, target, y, dLdy, workspace, workspace_bytes, step, nullptr, stream);
}

extern "C" hg_status hashgrid_train_step_clipped(const hashgrid_t* hg, const hashgrid_train_state* st, float max_norm,
                                                 hashgrid_grad_stats* stats, float* grads, uint32_t B, const float* x,
                                                 const float* target, void* y, void* dLdy, void* workspace,
                                                 uint64_t workspace_bytes, void* stream) {
  const hg::Clip clip{max_norm, stats, grads};
  return hg::train_step(hg, st, B, x, target, y, dLdy, workspace, workspace_bytes, 0, &clip, stream);
}
