"""The optimizer's plan after a refused call, on the CPU: checks that come before the library is called."""
import ctypes

import pytest
import torch

from paper_2606_16907_amd import layer as L


class Plan(L.AdamW):
    """A plan over tensors of device 0, as far as the checks look at them."""

    def __init__(self, params):
        self.tensors = dict(param=params, grad=params, m=params, v=params)
        self.h, self.device = ctypes.c_void_p(4096), 0

    def __del__(self):
        pass


class OnDevice0(torch.Tensor):
    def get_device(self):
        return 0


def tensor(n, dtype=torch.float32):
    return torch.zeros(n, dtype=dtype).as_subclass(OnDevice0)


@pytest.fixture
def current(monkeypatch):
    device = {"now": 0}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device["now"])
    return device


def test_gradients_refused_on_another_device_leave_the_plan_as_it_was(current):
    plan = Plan([tensor(8)])
    kept = plan.tensors["grad"]
    current["now"] = 1
    with pytest.raises(ValueError, match="param 0: on"):
        plan.set_grads([tensor(8)])
    assert plan.device == 0 and plan.tensors["grad"] is kept and plan.h.value == 4096


@pytest.mark.parametrize("grads,word", [([tensor(7)], "contiguous"), ([tensor(8, torch.float16)], "dtype"), ([], "0 tensors")])
def test_other_refusals_leave_it_too(current, grads, word):
    plan = Plan([tensor(8)])
    kept = plan.tensors["grad"]
    with pytest.raises(ValueError, match=word):
        plan.set_grads(grads)
    assert plan.device == 0 and plan.tensors["grad"] is kept and plan.h.value == 4096
