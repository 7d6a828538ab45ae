"""Errors of the vocabulary ends: a failed call is over when it has returned."""
import ctypes as C

import pytest
import torch

from paper_2604_24708_b200 import binding as B

NO_DEVICE = 1000


def _fail():
    """A call that the runtime refuses: there is no such device."""
    d = B.hdet_embedding(0x1000, 0x2000, 0x3000, 4, 10, 8, 4, 32, 8, 80, 8, 1.0, 2, B.HDET_DTYPE_I32, B.HDET_DTYPE_F32, B.HDET_DTYPE_F32, NO_DEVICE, 0)
    assert B.raw_library().hdet_embed(C.byref(d), None) == B.HDET_ERR_CUDA
    assert B.raw_library().hdet_embed_grad(C.byref(d), 0, 0x10000, 1 << 30, None) == B.HDET_ERR_CUDA
    a = B.hdet_token_loss_args(hidden=0x1000, weight=0x2000, targets=0x3000, loss=0x4000, n_tokens=4, vocab=10, width=8, hidden_stride=32, hidden_row=8,
                               weight_stride=80, weight_row=8, target_stride=4, grad_scale=1.0, n_replicas=2, hidden_dtype=B.HDET_DTYPE_BF16,
                               weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32, loss_dtype=B.HDET_DTYPE_F32, device=NO_DEVICE)
    assert B.raw_library().hdet_token_loss(C.byref(a), 0x10000, 1 << 30, None) == B.HDET_ERR_CUDA


@pytest.mark.gpu
@pytest.mark.parametrize("grads", [False, True])
def test_a_failed_call_is_not_the_next_ones(grads):
    """The loss, and calls that were there before it, after a failure on this thread."""
    h, w = torch.randn((2, 200, 64), device="cuda").bfloat16(), torch.randn((2, 300, 64), device="cuda").bfloat16()
    y, loss = torch.randint(0, 300, (2, 200), device="cuda", dtype=torch.int32), torch.empty(2, device="cuda")
    out = dict(d_hidden=torch.empty_like(h), d_weight=torch.empty_like(w)) if grads else {}
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, **out), dtype=torch.uint8, device="cuda")
    _fail()
    B.hdet_token_loss(h, w, y, loss, ws, stream=torch.cuda.current_stream().cuda_stream, **out)
    want = torch.nn.functional.cross_entropy((h.double() @ w.double().transpose(1, 2)).flatten(0, 1), y.flatten().long(), reduction="none")
    assert torch.allclose(loss.double(), want.view(2, 200).mean(1), rtol=1e-5)
    _fail()
    p = torch.randn((2, 64), device="cuda")
    mean = p.mean(0)
    t = B.hdet_tensor(param=p.data_ptr(), numel=64, param_stride=64)
    B.hdet_converge_static([t], 2, 0, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(p[0], mean) and torch.equal(p[1], mean)


# ------------------------------------------------------------------------------------------------ arguments (no GPU)
ARG, CUDA = B.HDET_ERR_INVALID_ARG, B.HDET_ERR_CUDA      # CUDA: nothing is wrong with the arguments, but there is no such device


def _embed_status(grad=False, **kw):
    d = B.hdet_embedding(0x1000, 0x2000, 0x3000, 4, 10, 8, 4, 32, 8, 80, 8, 1.0, 2, B.HDET_DTYPE_I32, B.HDET_DTYPE_F32, B.HDET_DTYPE_F32, NO_DEVICE, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    lib = B.raw_library()
    return lib.hdet_embed_grad(C.byref(d), 0, 0x10000, 1 << 50, None) if grad else lib.hdet_embed(C.byref(d), None)


def _loss_status(**kw):
    a = B.hdet_token_loss_args(
        hidden=0x1000, weight=0x2000, targets=0x3000, loss=0x4000, token_loss=0x5000, d_hidden=0x6000, d_weight=0x7000, n_tokens=4, vocab=10, width=8,
        hidden_stride=32, hidden_row=8, weight_stride=80, weight_row=8, target_stride=4, token_loss_stride=4, d_hidden_stride=32, d_hidden_row=8,
        d_weight_stride=80, d_weight_row=8, grad_scale=1.0, n_replicas=2, hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16,
        target_dtype=B.HDET_DTYPE_I32, loss_dtype=B.HDET_DTYPE_F32, d_hidden_dtype=B.HDET_DTYPE_BF16, d_weight_dtype=B.HDET_DTYPE_F32, device=NO_DEVICE)
    for k, v in kw.items():
        setattr(a, k, v)
    return B.raw_library().hdet_token_loss(C.byref(a), 0x10000, 1 << 50, None)


def test_what_is_refused_below_is_nothing_but_what_is_changed():
    assert _embed_status() == _embed_status(grad=True) == _loss_status() == CUDA


@pytest.mark.parametrize("stride", [1 << 60, (1 << 63) - 1, B.HDET_MAX_ROW_STRIDE + 1, 0x1C71C71C71C71C72])     # 9 x the last: 2^64 + 2
def test_row_strides_whose_offsets_pass_64_bits(stride):
    """With a stride of 2^64 / 9 a table of ten rows would seem to end behind its second element."""
    for name in ("table_row", "rows_row"):
        assert _embed_status(**{name: stride}) == _embed_status(grad=True, **{name: stride}) == ARG
    for name in ("hidden_row", "weight_row", "d_hidden_row", "d_weight_row"):
        assert _loss_status(**{name: stride}) == ARG


@pytest.mark.parametrize("stride", [1 << 60, (1 << 63) - 1, B.HDET_MAX_REPLICA_STRIDE + 1])
def test_replica_strides_whose_offsets_pass_64_bits(stride):
    for name in ("table_stride", "rows_stride", "token_stride"):
        assert _embed_status(**{name: stride}) == _embed_status(grad=True, **{name: stride}) == ARG
    for name in ("hidden_stride", "weight_stride", "target_stride", "token_loss_stride", "d_hidden_stride", "d_weight_stride"):
        assert _loss_status(**{name: stride}) == ARG


@pytest.mark.parametrize("scale", [1e39, -1e39, 1e300, float("inf"), float("nan")])
def test_scales_that_fp32_does_not_hold(scale):
    """They would turn into infinity, and zeros times that into NaN."""
    assert _embed_status(scale=scale) == _embed_status(grad=True, scale=scale) == _loss_status(grad_scale=scale) == ARG
    assert _embed_status(scale=3e38) == _loss_status(grad_scale=-3e38) == CUDA


def test_a_gradient_in_the_place_of_the_hidden_states_lies_on_them():
    same = dict(d_hidden=0x1000)
    assert _loss_status(**same) == CUDA
    assert _loss_status(**same, d_hidden_dtype=B.HDET_DTYPE_F32) == ARG
    assert _loss_status(**same, d_hidden_row=16, d_hidden_stride=64) == ARG
    assert _loss_status(**same, d_hidden_stride=40) == ARG
    assert _loss_status(**same, hidden_stride=0) == ARG             # one batch for all replicas, and a gradient for each
    assert _loss_status(**same, d_hidden_stride=40, n_replicas=1) == CUDA


@pytest.mark.parametrize("stride", [-1, -(1 << 62), 1 << 62, 3])
def test_one_replica_has_no_replica_strides(stride):
    """With one replica they are not looked at, whatever they hold."""
    names = ("table_stride", "rows_stride", "token_stride")
    assert _embed_status(n_replicas=1, **dict.fromkeys(names, stride)) == _embed_status(grad=True, n_replicas=1, **dict.fromkeys(names, stride)) == CUDA
    names = ("hidden_stride", "weight_stride", "target_stride", "token_loss_stride", "d_hidden_stride", "d_weight_stride")
    assert _loss_status(n_replicas=1, **dict.fromkeys(names, stride)) == CUDA
    need = []
    for s in (0, stride):
        a = B.hdet_token_loss_args(weight=0x2000, n_tokens=4, vocab=10, width=8, hidden_row=8, weight_row=8, grad_scale=1.0, n_replicas=1,
                                   hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32, **dict.fromkeys(names, s))
        size = C.c_int64(0)
        assert B.raw_library().hdet_token_loss_workspace(C.byref(a), C.byref(size)) == B.HDET_OK
        need.append(size.value)
    assert need[0] == need[1]
