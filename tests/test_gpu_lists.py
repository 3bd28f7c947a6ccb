"""Lists of tensors that change between two calls: what the calls read and write afterwards, on the device.  (What a list tells the library:
test_host_lists.py.)"""
import torch
import pytest

from paper_2201_05989_amd import AdamList, AdamTensor, GradStats, adam_steps, grad_norm

pytestmark = pytest.mark.gpu


def item(n, value):
    return AdamTensor(torch.zeros(n, device="cuda"), torch.full((n,), value, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"))


def test_norm_and_step_are_those_of_a_tensor_put_into_the_list():
    old, new = item(64, 3.0), item(64, 1.0)
    model, stats = AdamList([old]), GradStats()
    grad_norm(model.grads, stats)
    assert float(stats.norm) == 24.0
    model.tensors[0] = new
    grad_norm(model.grads, stats)
    assert float(stats.norm) == 8.0
    adam_steps(model, stats)
    assert not old.params_master.any() and not old.m.any() and bool((old.grad == 3.0).all())
    assert bool((new.params_master < 0).all()) and bool((new.m > 0).all()) and not new.grad.any()
