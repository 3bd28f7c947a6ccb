"""A clipped training step that is refused leaves the model as it was, the array that has to be all zero between steps too."""
import ctypes

import pytest
import torch

from paper_2201_05989_amd import HashGridModel

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [500, 40000])  # gradients by atomic additions into that array, and the sorted pass
def test_arrays_that_share_memory(B):
    m = HashGridModel(3, 1, L=8, T=1 << 14, N_max=512, max_grad_norm=1.0)
    x, target = torch.rand((B, 3), device="cuda") * 0.9, torch.randn((B, 1), device="cuda")
    m.step(x, target)
    arrays = (m.tables, m.tables_half, m._tab_m, m._tab_v, m.weights, m.weights_half, m._net_m, m._net_v, m.grad_stats.memory)
    before = [a.clone() for a in arrays]
    need = m.grid.bwd_workspace_bytes(B)
    workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    for name, at in (("tables_v", m._tab_m), ("weights_v", m._net_m), ("tables_m", m._tab_zeros), ("weights_half", m.tables_half)):
        st = m._train_state(B)
        setattr(st, name, at.data_ptr())
        assert m.grid._lib.hashgrid_train_step_clipped(
            m.grid._h, ctypes.byref(st), 1.0, m.grad_stats.memory.data_ptr(), m._grads.data_ptr(), B, x.data_ptr(), target.data_ptr(),
            m._y.data_ptr(), m._dy.data_ptr(), workspace.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 1
    torch.cuda.synchronize()
    assert not m._tab_zeros.any() and all(torch.equal(a, b) for a, b in zip(arrays, before))
    m.step(x, target)
    assert int(m.grad_stats.steps) == 2
