"""Norms of gradients that are mostly zeros, and of ones so small that fp32 squares of them are zeros."""
import pytest
import torch

from paper_2604_24708_b200 import binding as B
from test_grad_clip import Run, _near, _stream


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("mean", [0, 1])
@pytest.mark.parametrize("align,shift", [(8, 0), (1, 3)])
def test_zeros(mean, align, shift, grad):
    run = Run(3, (70001, 33, 2048 * 9), grad, align=align, shift=shift, grad_mode=mean)
    gen = torch.Generator(device="cuda").manual_seed(5)
    out = torch.full((3,), 7.25, dtype=torch.float64, device="cuda")

    def norms():
        B.hdet_grad_norm(run.h, out, stream=_stream())
        g = torch.stack([run.gradient(r).double() for r in range(3)])
        if mean:
            g = g.mean(0, keepdim=True).float().double().expand(3, -1)
        return g.square().sum(1).sqrt()
    keep = run.grad.clone()
    for share in (0.0, 0.9, 0.9999):
        run.grad.copy_(torch.where(torch.rand(keep.shape, generator=gen, device="cuda") < share, torch.zeros_like(keep), keep))
        _near(out, norms(), torch.float64)
    run.grad.zero_()
    norms()
    assert (out == 0).all()
    run.grad.copy_(torch.where(torch.rand(keep.shape, generator=gen, device="cuda") < 0.5, torch.zeros_like(keep), -torch.zeros_like(keep)))
    norms()
    assert (out == 0).all()
    # squares below fp32's range, between zeros; the mean of three is three times as small again
    for size in (1e-18, 1e-25, 2.0 ** -110):
        run.grad.copy_(torch.where(torch.rand(keep.shape, generator=gen, device="cuda") < 0.99, torch.zeros_like(keep), (keep.float() * size).to(keep.dtype)))
        _near(out, norms(), torch.float64)
        assert (out > 0).all()
    run.close()
