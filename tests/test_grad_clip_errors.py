"""A call that the runtime refused is over when it has returned: the next norm, and the next clipped step, are not taken for failed."""
import pytest
import torch

from paper_2604_24708_b200 import binding as B
from test_grad_clip import Run, _config, _near, _stream


def _fail_create():
    t = B.hdet_tensor(param=0x1000, grad=0x2000, exp_avg=0x3000, exp_avg_sq=0x4000, numel=64, param_stride=64, grad_stride=64, state_stride=64)
    with pytest.raises(B.HdetError):
        B.hdet_create(_config(2, device=1000), [t])              # there is no such device


def _fail_static():
    with pytest.raises(B.HdetError):
        B.hdet_converge_static([B.hdet_tensor(param=0x1000, numel=64, param_stride=64)], 2, 60)


@pytest.mark.gpu
@pytest.mark.parametrize("failure", [_fail_create, _fail_static])
@pytest.mark.parametrize("opt", ["adamw", "sgd"])
def test_after_a_failed_call(opt, failure):
    run, ref = Run(2, opt=opt), Run(2, opt=opt)
    want = torch.stack([run.gradient(r).double().square().sum().sqrt() for r in range(2)])
    norms = torch.zeros(2, device="cuda")
    failure()
    B.hdet_grad_norm(run.h, norms, stream=_stream())
    _near(norms, want, torch.float32)
    for r in (run, ref):
        B.hdet_set_clip(r.h, float(want.min()) / 2)
        if r is run:
            failure()
        B.hdet_step(r.h, [0.0, 0.0], _stream())
        assert B.hdet_get_state(r.h).step == 1
    for x, y in zip(run.state(), ref.state()):
        assert torch.equal(x, y)
    run.close(), ref.close()
