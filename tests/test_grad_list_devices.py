"""Lists of gradients whose tensors a kernel cannot read are refused in the binding: tensors in host memory, of several devices, of another device than the current one."""
import pytest
import torch

from paper_2105_13890_b200 import build, eoq
from test_float_operator_refusals import A

build.build_lib()


class On:
    """Stands in for a contiguous tensor on a device (-1: the host)."""

    dtype = torch.float32

    def __init__(self, device, n=8):
        self.device_, self.n = device, n

    def get_device(self):
        return self.device_

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 12


def calls(l):
    for call in (lambda: eoq.eoq_grad_norm(0, l, A, A, stream=0, check=False), lambda: eoq.eoq_grad_clip(0, l, 1.0, A, A, stream=0, check=False)):
        yield call


def test_tensors_in_host_memory():
    for l in (eoq.grad_list([torch.zeros(4)]), eoq.grad_list([torch.zeros(4)], [torch.zeros(4)]), eoq.grad_list([torch.zeros(4, device="meta")])):
        for call in calls(l):
            with pytest.raises(ValueError):
                call()


def test_tensors_of_several_devices():
    for tensors, out in (([On(0), On(-1)], None), ([On(0), On(1)], None), ([On(0)], [On(-1)]), ([On(0)], [On(1)])):
        with pytest.raises(ValueError):
            eoq.grad_list(tensors, out)
    # (a tensor without elements is left out, wherever it is)
    assert eoq.grad_list([On(0), On(-1, 0)], [On(0), On(1, 0)]).num == 2


def test_tensors_of_another_device(monkeypatch):
    monkeypatch.setattr(eoq, "_current_device", lambda: 0)
    for call in calls(eoq.grad_list([On(1)])):
        with pytest.raises(ValueError):
            call()
    for l in (eoq.grad_list([On(0)]), eoq.grad_list([On(-1, 0), On(3, 0)])):
        for call in calls(l):
            assert call() == eoq.EOQ_ERR_BAD_ARG          # all is well but the handle
