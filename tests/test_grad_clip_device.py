"""Norms that lie on another device than the handle are refused before a kernel could write to them (no GPU)."""
import pytest
import torch

from paper_2604_24708_b200 import binding as B


class _Norms:
    """What the binding asks a tensor."""
    is_cuda, shape, dtype = True, torch.Size([2]), torch.float32

    def __init__(self, device):
        self._device = device

    def get_device(self):
        return self._device

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000


@pytest.mark.parametrize("device", [0, 1])
def test_norms_on_another_device(device):
    h = B.hdet_create(B.hdet_config(n_replicas=2, n_groups=1, optimizer=B.HDET_OPT_SGD, grad_dtype=B.HDET_DTYPE_F32, sync_interval=1, device=device), [])
    for call in (lambda x: B.hdet_set_clip(h, 1.0, x), lambda x: B.hdet_grad_norm(h, x)):
        with pytest.raises(ValueError, match="the handle's CUDA device"):
            call(_Norms(1 - device))
    B.hdet_set_clip(h, 1.0, _Norms(device))
    with pytest.raises(B.HdetError, match="no tensors"):
        B.hdet_grad_norm(h, _Norms(device))
    B.hdet_destroy(h)
