"""hashgrid_train_step_clipped refuses arrays that share memory before it launches anything, through the C ABI with made-up addresses: every
call here is turned down, so no device is needed.  (That it takes the same arrays side by side: test_gpu_train_step_clipped.py.)"""
import ctypes
import itertools

import pytest

from paper_2201_05989_amd import HashGrid, binding

L, F, T, N_OUT = 4, 2, 1 << 12, 3
NET = 64 * (L * F + 64 + N_OUT)


def layout(grid, B):
    """[name, bytes, written] of every array of a call, and where each lies: side by side, 4 KB and more apart."""
    tab = grid.n_entries * F
    sizes = {"tables": 4 * tab, "tables_half": 2 * tab, "tables_m": 4 * tab, "tables_v": 4 * tab, "tables_zeros": 4 * tab, "weights": 4 * NET,
             "weights_half": 2 * NET, "weights_m": 4 * NET, "weights_v": 4 * NET, "loss_sum": 8, "scratch": binding.HG_TRAIN_SCRATCH_BYTES,
             "stats": binding.HG_GRAD_STATS_BYTES, "grads": 4 * (tab + NET), "y": 2 * L * F * B, "dLdy": 2 * L * F * B,
             "workspace": grid.bwd_workspace_bytes(B), "x": 4 * 3 * B, "target": 4 * N_OUT * B}
    at, end = {}, 1 << 30
    for name, size in sizes.items():
        at[name] = end
        end += (size + 8191) // 4096 * 4096
    return sizes, at


def call(grid, at, B, workspace_bytes):
    adam = binding.hashgrid_adam_config(1e-2, 0.9, 0.99, 1e-15, 0.0)
    st = binding.hashgrid_train_state(n_out=N_OUT, loss=0, loss_scale=1.0, tables_adam=adam, weights_adam=adam,
                                      **{k: at[k] for k in ("tables", "tables_half", "tables_m", "tables_v", "tables_zeros", "weights",
                                                            "weights_half", "weights_m", "weights_v", "loss_sum", "scratch")})
    return grid._lib.hashgrid_train_step_clipped(grid._h, ctypes.byref(st), 1.0, at["stats"], at["grads"], B, at["x"], at["target"], at["y"],
                                                 at["dLdy"], at["workspace"], workspace_bytes, None)


@pytest.mark.parametrize("B", [300, 40000])  # gradients by atomic additions, and the sorted pass
def test_arrays_that_share_memory_are_refused_before_anything_is_launched(B):
    grid = HashGrid(3, L, F, T, 16, 128, "f16", "f16")
    assert grid.bwd_ws_pays(B) == (B == 40000)
    sizes, at = layout(grid, B)
    read = {"x", "target"}
    used = [n for n in sizes if n != "workspace" or B == 40000]
    for a, b in itertools.permutations(used, 2):
        if {a, b} == read:
            continue
        moved = dict(at)
        # b begins in the last bytes of a, as its alignment allows
        step = 256 if b == "workspace" else 16
        moved[b] = at[a] + (sizes[a] - 1) // step * step
        assert call(grid, moved, B, sizes["workspace"]) == 1, (a, b)
