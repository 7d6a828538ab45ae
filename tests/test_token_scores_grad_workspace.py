"""The workspace of the gradients for given ones holds nothing of the loss's statistics (no GPU)."""
import ctypes as C

import pytest

from paper_2604_24708_b200 import binding as B


@pytest.mark.parametrize("R,T,V,D,tile", [(2, 256, 5000, 64, 128), (8, 2048, 50257, 64, 256), (1, 1000, 130000, 40, 256), (1, 100, 700, 64, 128)])
def test_a_loss_needs_more(R, T, V, D, tile):
    same = dict(hidden=0x1000, weight=0x2000, targets=0x3000, d_hidden=0x9000, d_weight=0xA000, n_tokens=T, vocab=V, width=D, hidden_stride=T * D,
                hidden_row=D, weight_stride=V * D, weight_row=D, target_stride=T, d_hidden_stride=T * D, d_hidden_row=D, d_weight_stride=V * D,
                d_weight_row=D, n_replicas=R, hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32,
                d_hidden_dtype=B.HDET_DTYPE_F32, d_weight_dtype=B.HDET_DTYPE_F32, piece_bytes=1 << 40)
    loss, given, lib = C.c_int64(0), C.c_int64(0), B.raw_library()
    assert lib.hdet_token_loss_workspace(C.byref(B.hdet_token_loss_args(loss=0x4000, grad_scale=1.0, **same)), C.byref(loss)) == B.HDET_OK
    assert lib.hdet_token_scores_grad_workspace(C.byref(B.hdet_token_scores_args(**same)), C.byref(given)) == B.HDET_OK
    # a maximum and a sum for each half tile of every row; of as much one number could be needed
    assert given.value <= loss.value - 4 * R * T * 2 * (V // tile)
