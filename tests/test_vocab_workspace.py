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
