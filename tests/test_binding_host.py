"""The binding hands addresses to kernels: tensors of the host are refused before any call of the library."""
import pytest
import torch

import paper_2510_26771_amd as st
from paper_2510_26771_amd import binding


class Calls:
    def __init__(self):
        self.names = []

    def __getattr__(self, name):
        def call(*arguments):
            self.names.append(name)
            return 0
        return call


@pytest.mark.parametrize("name,tensors", [("quantize_act", 5), ("linear_forward", 3), ("linear_forward_static", 2), ("linear_forward_q", 5), ("debug_gemm_acc", 3)])
def test_host_tensors_are_refused(monkeypatch, name, tensors):
    monkeypatch.setattr(binding, "_stream", lambda stream: None)
    plan = object.__new__(st.StampPlan)
    plan.lib, plan._h = Calls(), None
    host = torch.zeros(256, dtype=torch.uint8)

    class OnGpu:
        is_cuda = True

        def data_ptr(self):
            return 256

        def numel(self):
            return 256
    for i in range(tensors):
        with pytest.raises(ValueError):
            getattr(plan, name)(*(host if j == i else OnGpu() for j in range(tensors)))
        assert not plan.lib.names
    getattr(plan, name)(*(OnGpu() for _ in range(tensors)))
    assert len(plan.lib.names) == 1
