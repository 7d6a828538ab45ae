"""What the workspace queries of the vocabulary ends look at, and what a workspace is enough for (host arithmetic, no GPU)."""
import ctypes as C

import pytest

from paper_2604_24708_b200 import binding as B


def _loss_args(R, T, V, D, grads=None, hidden=0x1000, hidden_pad=0, weight=0x2000, piece_bytes=0):
    """grads: None, or the dtypes of d_hidden and d_weight (None: not asked for)."""
    dh, dw = grads or (None, None)
    row = D + hidden_pad
    return B.hdet_token_loss_args(
        hidden=hidden, weight=weight, targets=0x3000, loss=0x4000, d_hidden=0x6000 if dh is not None else None,
        d_weight=0x7000 if dw is not None else None, n_tokens=T, vocab=V, width=D, hidden_stride=T * row, hidden_row=row, weight_stride=V * D, weight_row=D,
        target_stride=T, d_hidden_stride=T * D, d_hidden_row=D, d_weight_stride=V * D, d_weight_row=D, grad_scale=1.0, piece_bytes=piece_bytes,
        n_replicas=R, hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32, loss_dtype=B.HDET_DTYPE_F32,
        d_hidden_dtype=dh or 0, d_weight_dtype=dw or 0)


def _loss_bytes(*args, **kw):
    need = C.c_int64(0)
    assert B.raw_library().hdet_token_loss_workspace(C.byref(_loss_args(*args, **kw)), C.byref(need)) == B.HDET_OK
    return need.value


@pytest.mark.parametrize("R,T,V,D", [(1, 1, 1000, 64), (1, 4, 10000, 768), (3, 2, 300, 64), (32, 3, 5000, 64), (1, 1, 50257, 768), (1, 5, 1000, 64)])
def test_the_loss_workspace_does_not_depend_on_the_hidden_states_address_or_strides(R, T, V, D):
    sizes = {_loss_bytes(R, T, V, D, hidden=at, hidden_pad=pad) for at in (None, 0x1000, 0x1002, 0x1008) for pad in (0, 1, 8)}
    assert len(sizes) == 1, sizes


F32, BF16 = B.HDET_DTYPE_F32, B.HDET_DTYPE_BF16
NO_DEVICE = 1000        # no such device: a call that is not refused for its arguments ends there, before it looks at any pointer


def _up_to(T):
    return sorted({t for m in range(0, T + 65, 64) for t in (m - 1, m, m + 1) if 0 < t <= T} | {1, 2, 3, 4, 5})


@pytest.mark.parametrize("R,T,V,D,piece", [(8, 2048, 50257, 2048, 0), (16, 1024, 50257, 768, 0), (8, 1024, 50257, 768, 0), (4, 200, 50257, 64, 0),
                                           (3, 300, 4099, 520, 1), (3, 400, 1000, 64, 1000000), (1, 260, 700, 64, 1)])
@pytest.mark.parametrize("grads", [None, (BF16, BF16), (BF16, F32), (F32, F32), (None, BF16)])
def test_a_loss_workspace_is_enough_for_fewer_tokens(R, T, V, D, piece, grads):
    lib, size = B.raw_library(), _loss_bytes(R, T, V, D, grads, piece_bytes=piece)
    for t in _up_to(T):
        a = _loss_args(R, t, V, D, grads, piece_bytes=piece)
        a.device = NO_DEVICE
        assert lib.hdet_token_loss(C.byref(a), 0x10000, size, None) == B.HDET_ERR_CUDA, (t, lib.hdet_last_error(None))
        assert _loss_bytes(R, t, V, D, grads, piece_bytes=piece) <= size


def _embedding(R, T, V, D):
    return B.hdet_embedding(0x1000, 0x2000, 0x3000, T, V, D, T, T * D, D, V * D, D, 1.0, R, B.HDET_DTYPE_I32, F32, F32, NO_DEVICE, 0)


@pytest.mark.parametrize("R,T,V,D", [(1, 20000, 1000, 64), (2, 9441, 1000, 64), (8, 1000, 50257, 768), (16, 1200, 50257, 300), (32, 700, 100, 8), (1, 7, 3, 1)])
def test_an_embedding_workspace_is_enough_for_fewer_tokens(R, T, V, D):
    lib, need = B.raw_library(), C.c_int64(0)
    assert lib.hdet_embed_grad_workspace(C.byref(_embedding(R, T, V, D)), C.byref(need)) == B.HDET_OK
    for t in _up_to(T):
        assert lib.hdet_embed_grad(C.byref(_embedding(R, t, V, D)), 0, 0x10000, need.value, None) == B.HDET_ERR_CUDA, (t, lib.hdet_last_error(None))


def test_the_query_of_a_long_batch_takes_no_time():
    import time
    start = time.perf_counter()
    _loss_bytes(1, B.HDET_MAX_TOKENS, 50257, 64, (BF16, BF16))
    assert time.perf_counter() - start < 5
