"""Gradient norms against 64-bit sums, and clipped steps against plain steps on gradients that were clipped beforehand."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2604_24708_b200 import binding as B

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ODD = (1, 7, 8, 33, 1023, 1024, 2049, 4097, 32768, 32769, 70001, 5)


def _config(n, opt=B.HDET_OPT_ADAMW, grad="f32", **kw):
    kw = {**dict(alpha_lr=0.25, sync_interval=2, fuse_converge=1), **kw}
    return B.hdet_config(n_replicas=n, n_groups=1, optimizer=opt, grad_dtype=B.HDET_DTYPE_BF16 if grad == "bf16" else B.HDET_DTYPE_F32,
                         beta1=0.9, beta2=0.999, eps=1e-8, **kw)


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def test_refusals():
    lib, h = B.raw_library(), B.hdet_create(_config(2), [])
    f32, f64 = B.HDET_DTYPE_F32, B.HDET_DTYPE_F64
    assert lib.hdet_grad_norm(None, 0x1000, f32, None) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_set_clip(None, 1.0, None, f32) == B.HDET_ERR_INVALID_ARG
    for args, status in [((None, f32), B.HDET_ERR_INVALID_ARG), ((0x1000, B.HDET_DTYPE_BF16), B.HDET_ERR_INVALID_ARG), ((0x1002, f32), B.HDET_ERR_ALIGN),
                         ((0x1004, f64), B.HDET_ERR_ALIGN), ((0x1000, f32), B.HDET_ERR_UNSUPPORTED)]:
        assert lib.hdet_grad_norm(h, *args, None) == status, args
        assert lib.hdet_last_error(h).startswith(b"hdet_grad_norm: ")
    for bad in (-1.0, float("nan"), float("inf")):
        assert lib.hdet_set_clip(h, bad, None, f32) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_set_clip(h, 1.0, 0x1000, B.HDET_DTYPE_I32) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_set_clip(h, 1.0, 0x1004, f64) == B.HDET_ERR_ALIGN
    assert lib.hdet_last_error(h).startswith(b"hdet_set_clip: ")
    B.hdet_set_clip(h, 1.0)
    B.hdet_set_schedule(h, B.make_schedule(B.HDET_SCHED_CONSTANT, 10, [1e-2]))
    B.hdet_step(h)                      # a handle without tensors has nothing to clip
    B.hdet_set_clip(h, 0.0)
    for bad in (torch.zeros(2), torch.zeros(3)):
        with pytest.raises(ValueError):
            B.hdet_grad_norm(h, bad)
        with pytest.raises(ValueError):
            B.hdet_set_clip(h, 1.0, bad)
    B.hdet_destroy(h)


# ------------------------------------------------------------------------------------------------ a list of tensors
class Run:
    """Tensors of the given sizes in one allocation each for parameters, moments and gradients, and their handle."""

    def __init__(self, n, numels=ODD, grad="f32", opt="adamw", align=8, shift=0, shared_grad=False, shared_state=False, seed=0, **kw):
        self.n, self.numels, self.momentum = n, numels, kw.get("momentum", 0.0)
        adam = opt == "adamw"
        at, self.places = shift, []
        for k in numels:
            self.places.append((at, k))
            at += -(-k // align) * align
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda rows, scale: torch.randn((rows, at), generator=gen, device="cuda") * scale  # noqa: E731
        self.param, self.grad = rand(n, 0.02), rand(1 if shared_grad else n, 1e-2).to(DT[grad])
        rows = 1 if shared_state else n
        self.m, self.v = (rand(rows, 1e-3), rand(rows, 1e-3).square_()) if adam else ((rand(n, 1e-3), None) if self.momentum else (None, None))
        tensors = []
        for off, k in self.places:
            t = B.hdet_tensor(numel=k, param_stride=at, grad_stride=0 if shared_grad else at, state_stride=0 if shared_state else at)
            t.param, t.grad = self.param.data_ptr() + 4 * off, self.grad.data_ptr() + self.grad.element_size() * off
            if self.m is not None:
                t.exp_avg = self.m.data_ptr() + 4 * off
            if self.v is not None:
                t.exp_avg_sq = self.v.data_ptr() + 4 * off
            tensors.append(t)
        self.h = B.hdet_create(_config(n, B.HDET_OPT_ADAMW if adam else B.HDET_OPT_SGD, grad, **kw), tensors)
        B.hdet_set_schedule(self.h, B.make_schedule(B.HDET_SCHED_CONSTANT, 100, [1e-2], weight_decay=[0.1]))

    def gradient(self, r):
        g = self.grad[r if len(self.grad) > 1 else 0]
        return torch.cat([g[at:at + k] for at, k in self.places])

    def state(self):
        return [t.clone() for t in (self.param, self.m, self.v) if t is not None]

    def close(self):
        torch.cuda.synchronize()
        B.hdet_destroy(self.h)


def _stream():
    return torch.cuda.current_stream().cuda_stream


# Sums in fp64 of squares that are off by fp32's half step (and their sums over 16 bytes by eight of them): 9 x 2^-24 of the sum, half
# of that in the root; fp32 norms add half a step.
def _near(got, want, dtype):
    tol = 4.5 * 2.0 ** -24 + (2.0 ** -24 if dtype == torch.float32 else 0.0)
    assert ((got.double() - want).abs() <= tol * want.abs()).all(), (got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("n,numels,align,shift", [(1, (1,), 8, 0), (3, ODD, 8, 0), (2, ODD, 1, 1), (5, ODD, 1, 3), (4, (300001,), 4, 0), (2, (3, 1, 2), 1, 5),
                                                  (32, (2049, 40), 8, 0)])
def test_norms(n, numels, align, shift, grad):
    run = Run(n, numels, grad, align=align, shift=shift)
    want = torch.stack([run.gradient(r).double().square().sum().sqrt() for r in range(n)])
    for dtype in (torch.float32, torch.float64):
        out = torch.full((n + 2,), 7.25, dtype=dtype, device="cuda")
        before = B.hdet_kernel_launches(run.h)
        for _ in range(3):
            B.hdet_grad_norm(run.h, out[1:-1], stream=_stream())
        assert B.hdet_kernel_launches(run.h) == before + 3
        _near(out[1:-1], want, dtype)
        assert out[0] == 7.25 and out[-1] == 7.25
        first = out.clone()
        B.hdet_grad_norm(run.h, out[1:-1], stream=_stream())
        assert torch.equal(first, out)
    run.close()


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("n,align,shift,shared", [(4, 8, 0, False), (3, 1, 1, False), (5, 8, 0, True), (1, 4, 0, False)])
def test_norms_of_one_gradient_for_all(n, align, shift, shared, grad):
    """The replicas' mean, or the one gradient that they share: one norm, for every replica."""
    run = Run(n, grad=grad, align=align, shift=shift, shared_grad=shared, grad_mode=B.HDET_GRAD_AS_GIVEN if shared else B.HDET_GRAD_REPLICA_MEAN)
    total = sum(run.gradient(r).double() for r in range(n)) / n
    out = torch.empty(n, dtype=torch.float64, device="cuda")
    B.hdet_grad_norm(run.h, out, stream=_stream())
    # the mean is rounded to fp32: half a step of each element, so of the norm
    want = total.square().sum().sqrt().expand(n)
    assert ((out - want).abs() <= (4.5 + 1.0) * 2.0 ** -24 * want).all() and (out == out[0]).all()
    run.close()


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 32])
def test_norms_of_a_mean_whose_sum_is_out_of_range(n, grad):
    run = Run(n, (70001, 33, 5), grad, align=1, shift=1, grad_mode=B.HDET_GRAD_REPLICA_MEAN)
    out = torch.empty(n, dtype=torch.float64, device="cuda")
    for fill in (3.2e38, 2.0 ** -126, 2.0 ** -133):
        run.grad.fill_(fill)                    # equal in all replicas: their mean is exact but for one rounding of 1 / n
        B.hdet_grad_norm(run.h, out, stream=_stream())
        want = run.gradient(0).double().square().sum().sqrt().expand(n)
        assert ((out - want).abs() <= (4.5 + 1.0) * 2.0 ** -24 * want).all(), (fill, out[0], want[0])
    run.close()


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_norms_of_values_at_the_ends_of_the_range(grad):
    run = Run(2, (70001, 33), grad)
    out = torch.empty(2, dtype=torch.float64, device="cuda")
    for fill in (0.0, 1e-38, 1e-25, 3e-16, 1e-8, 1e8, 3e15, 1e25, 1e38):
        run.grad.fill_(fill)
        run.grad[1, ::2] *= -0.5
        B.hdet_grad_norm(run.h, out, stream=_stream())
        _near(out, torch.stack([run.gradient(r).double().square().sum().sqrt() for r in range(2)]), torch.float64)
    run.grad.zero_()
    run.grad[0, 70008] = float("inf")
    run.grad[1, 5] = float("nan")
    B.hdet_grad_norm(run.h, out, stream=_stream())
    assert out[0] == float("inf") and torch.isnan(out[1])
    run.close()


# ------------------------------------------------------------------------------------------------ clipped steps
def _clip_beforehand(run, ref, norms, max_norm, mean):
    """ref's fp32 gradients = run's, times the factors: what a clipped step of run has to do, as gradients of a plain step."""
    n = run.n
    factor = [np.float32(max_norm / x) if x > max_norm and np.isfinite(x) else np.float32(1.0) for x in norms.tolist()]
    if mean:
        total = torch.zeros_like(run.grad[0], dtype=torch.float64)
        for r in range(n):
            total += run.grad[r].double()
        ref.grad[0] = (total * (1.0 / n)).float() * float(factor[0])
        return
    for r in range(len(run.grad)):
        ref.grad[r] = run.grad[r].float() * float(factor[r])


CASES = [
    dict(opt="adamw", grad="f32"), dict(opt="adamw", grad="bf16"), dict(opt="adamw", grad="bf16", align=1, shift=1), dict(opt="sgd", grad="f32"),
    dict(opt="sgd", grad="bf16"), dict(opt="sgd", grad="bf16", momentum=0.9), dict(opt="sgd", grad="f32", momentum=0.9, align=1, shift=3),
    dict(opt="adamw", grad="bf16", grad_mode=B.HDET_GRAD_REPLICA_MEAN), dict(opt="adamw", grad="f32", grad_mode=B.HDET_GRAD_REPLICA_MEAN, align=1),
    dict(opt="sgd", grad="bf16", grad_mode=B.HDET_GRAD_REPLICA_MEAN), dict(opt="sgd", grad="f32", grad_mode=B.HDET_GRAD_REPLICA_MEAN, momentum=0.9),
    dict(opt="adamw", grad="bf16", shared_grad=True, shared_state=True), dict(opt="adamw", grad="f32", shared_grad=True, shared_state=True, align=1, shift=1),
    dict(opt="adamw", grad="bf16", grad_mode=B.HDET_GRAD_REPLICA_MEAN, shared_state=True), dict(opt="adamw", grad="f32", shared_grad=True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("fuse", [1, 0])
@pytest.mark.parametrize("case", CASES, ids=[" ".join(f"{k}={v}" for k, v in c.items()) for c in CASES])
def test_a_clipped_step_is_a_step_with_clipped_gradients(case, fuse):
    """Bit for bit, over steps with and without a converge, at norms on both sides of the largest."""
    n, mean = 3, case.get("grad_mode") == B.HDET_GRAD_REPLICA_MEAN
    run = Run(n, fuse_converge=fuse, **case)
    plain = {k: v for k, v in case.items() if k != "grad_mode"}
    ref = Run(n, fuse_converge=fuse, **{**plain, "grad": "f32", "shared_grad": mean or bool(case.get("shared_grad"))})
    for a, b in zip((ref.param, ref.m, ref.v), (run.param, run.m, run.v)):
        if a is not None:
            a.copy_(b)
    norms, again = torch.empty(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    B.hdet_grad_norm(run.h, norms, stream=_stream())
    limit = float(norms.median())
    B.hdet_set_clip(run.h, limit, again)
    for step, size in enumerate((1.0, 0.3, 4.0, 1.0)):
        run.grad.mul_(size).mul_(torch.tensor([1.0, 0.5, 2.0], device="cuda")[:len(run.grad), None])
        B.hdet_grad_norm(run.h, norms, stream=_stream())
        _clip_beforehand(run, ref, norms, limit, mean)
        assert B.hdet_step(run.h, stream=_stream()) == B.hdet_step(ref.h, stream=_stream())
        assert torch.equal(again, norms)
        for a, b in zip(run.state(), ref.state()):
            assert torch.equal(a, b), step
    # and off again
    B.hdet_set_clip(run.h, 0.0)
    _clip_beforehand(run, ref, norms * 0.0, 1.0, mean)
    B.hdet_step(run.h, stream=_stream()), B.hdet_step(ref.h, stream=_stream())
    assert all(torch.equal(a, b) for a, b in zip(run.state(), ref.state()))
    run.close(), ref.close()


@pytest.mark.gpu
def test_gradients_that_are_not_finite_clip_nothing():
    run = Run(3, opt="sgd")
    start = run.param.clone()
    run.grad[0, 9] = float("inf")
    run.grad[1, 9] = float("nan")
    norms = torch.empty(3, device="cuda")
    B.hdet_set_clip(run.h, 1e-3, norms)
    B.hdet_step(run.h, stream=_stream())
    torch.cuda.synchronize()
    assert norms[0] == float("inf") and torch.isnan(norms[1]) and torch.isfinite(norms[2])
    bad = ~torch.isfinite(run.param)
    assert bad[0, 9] and bad[1, 9] and bad.sum() == 2
    moved = (run.param - start)[2]
    assert float(moved.abs().max()) > 0
    assert B.hdet_get_state(run.h, raise_on_nonfinite=False).device_status == 1
    run.close()


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_every_form_of_the_step_clips_alike(grad):
    """From host memory, from device-resident scalars, from a captured graph, and on a stream of one's own."""
    n = 3
    runs = [Run(n, grad=grad) for _ in range(4)]
    outs = [torch.zeros(n, device="cuda") for _ in runs]
    for run, out in zip(runs, outs):
        B.hdet_set_clip(run.h, 0.5, out)
    a, b, c, d = runs
    host = a.grad.cpu().pin_memory()
    losses = torch.zeros(n, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    B.hdet_step_device(d.h, losses, stream=_stream())       # brings the scalar state to the device
    B.hdet_step_device(d.h, losses, stream=_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):       # a whole round
        for _ in range(2):
            B.hdet_step_device(d.h, losses, stream=_stream())
    outs[3].zero_()
    side.wait_stream(torch.cuda.current_stream())
    for k in range(2):
        B.hdet_step(a.h, stream=_stream())
        b.grad.zero_()
        B.hdet_step_host_grads(b.h, [host.data_ptr() + host.element_size() * at for at, _ in b.places], stream=_stream())
        with torch.cuda.stream(side):
            B.hdet_step(c.h, stream=_stream())
    torch.cuda.synchronize()
    for x, y in zip(a.state(), c.state()):
        assert torch.equal(x, y)
    for (at, k) in a.places:            # host gradients come without what lies between the tensors
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x[:, at:at + k], y[:, at:at + k])
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[3])        # the gradients, and so the norms, are the same
    graph.reset()
    for run in runs:
        run.close()


@pytest.mark.gpu
def test_device_resident_steps_clip_as_host_steps():
    """Their scalars agree to rounding of the math library, so the parameters to a few steps of fp32."""
    n = 3
    a, b = Run(n, grad="bf16"), Run(n, grad="bf16")
    norms, losses = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    for r in (a, b):
        B.hdet_set_clip(r.h, 0.5, norms)
    for _ in range(3):
        assert B.hdet_step(a.h, stream=_stream()) == B.hdet_step_device(b.h, losses, stream=_stream())
    torch.cuda.synchronize()
    for x, y in zip(a.state(), b.state()):
        assert float((x - y).abs().max()) <= 8 * 2.0 ** -24 * float(x.abs().max())
    a.close(), b.close()


@pytest.mark.gpu
def test_a_shard_clips_its_own_replicas():
    whole, part = Run(4), Run(2, n_replicas_global=4, replica_offset=2)
    for x, y in zip((part.param, part.m, part.v, part.grad), (whole.param, whole.m, whole.v, whole.grad)):
        x.copy_(y[2:])
    a, b = torch.empty(4, device="cuda"), torch.empty(2, device="cuda")
    B.hdet_set_clip(whole.h, 0.5, a)
    B.hdet_set_clip(part.h, 0.5, b)
    _, total = B.hdet_partial_layout(part.h, len(ODD))
    staging = torch.empty(total, device="cuda")
    assert not B.hdet_step(whole.h, stream=_stream()) and not B.hdet_step_sharded(part.h, None, staging, stream=_stream())
    assert torch.equal(a[2:], b)
    for x, y in zip(part.state(), whole.state()):
        assert torch.equal(x, y[2:])
    whole.close(), part.close()
