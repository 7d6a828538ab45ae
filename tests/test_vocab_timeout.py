"""Waits of the token loss that run out: made to happen without any fault, by a hand-over that is withheld, with a limit of some milliseconds."""
import ctypes as C

import pytest
import torch

from paper_2604_24708_b200 import binding as B


def test_it_refuses_what_the_loss_refuses():
    lib = B.raw_library()
    assert lib.hdet_selftest_token_loss_wait(None, 0x10000, 1 << 40, None) == B.HDET_ERR_INVALID_ARG
    a = B.hdet_token_loss_args(weight=0x2000, loss=0x4000, n_tokens=0, vocab=10, width=8, hidden_row=8, weight_row=8, grad_scale=1.0, n_replicas=1,
                               hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32)
    assert lib.hdet_selftest_token_loss_wait(C.byref(a), 0x10000, 16, None) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_last_error(None).startswith(b"hdet_selftest_token_loss_wait: ")


# single CTAs and pairs; more tiles than there are SMs, and fewer
@pytest.mark.gpu
@pytest.mark.parametrize("R,T,V", [(1, 60, 300), (2, 100, 20000), (2, 300, 2000), (2, 600, 9000)])
@pytest.mark.parametrize("dt,piece", [(None, 0), (torch.bfloat16, 0), (torch.bfloat16, 1000000), (torch.float32, 0)])
def test_a_wait_that_runs_out(R, T, V, dt, piece):
    D = 200
    gen = torch.Generator().manual_seed(T)
    h, w = torch.randn((R, T, D), generator=gen).bfloat16().cuda(), torch.randn((R, V, D), generator=gen).bfloat16().cuda()
    y = torch.randint(0, V, (R, T), generator=gen).int().cuda()
    out = dict(loss=torch.empty(R, device="cuda"))
    if dt:
        out.update(d_hidden=torch.empty((R, T, D), dtype=dt, device="cuda"), d_weight=torch.empty((R, V, D), dtype=dt, device="cuda"))
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=out.get("d_hidden"), d_weight=out.get("d_weight"), piece_bytes=piece),
                     dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    B.hdet_token_loss(h, w, y, workspace=ws, piece_bytes=piece, stream=st, **out)
    want = {k: v.clone() for k, v in out.items()}
    for _ in range(2):
        B.hdet_selftest_token_loss_wait(h, w, y, workspace=ws, piece_bytes=piece, stream=st, **out)
        torch.cuda.synchronize()
        assert torch.isnan(out["loss"]).all()
    B.hdet_token_loss(h, w, y, workspace=ws, piece_bytes=piece, stream=st, **out)
    assert all(torch.equal(out[k], want[k]) for k in want) and torch.isfinite(want["loss"]).all()


@pytest.mark.gpu
def test_the_kernel_for_few_tokens_has_no_wait():
    h, w = torch.zeros((1, 2, 64), device="cuda").bfloat16(), torch.zeros((1, 300, 64), device="cuda").bfloat16()
    y, loss = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y), dtype=torch.uint8, device="cuda")
    with pytest.raises(B.HdetError, match="waits for nothing"):
        B.hdet_selftest_token_loss_wait(h, w, y, loss, ws)
