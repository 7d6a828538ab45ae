"""Waits of the gradients for given ones that run out: made to happen without any fault, by a hand-over that is withheld, with a limit of some
milliseconds.  There is no loss that could tell, so the gradients' first elements do."""
import ctypes as C

import pytest
import torch

from paper_2604_24708_b200 import binding as B
from test_token_scores import inputs, strided


def test_it_refuses_what_the_gradient_refuses():
    lib = B.raw_library()
    assert lib.hdet_selftest_token_scores_grad_wait(None, 0x10000, 1 << 40, None) == B.HDET_ERR_INVALID_ARG
    a = B.hdet_token_scores_args(weight=0x2000, n_tokens=0, vocab=10, width=8, hidden_row=8, weight_row=8, n_replicas=1, d_weight=0x3000, d_weight_row=8,
                                 hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32)
    assert lib.hdet_selftest_token_scores_grad_wait(C.byref(a), 0x10000, 16, None) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_last_error(None).startswith(b"hdet_selftest_token_scores_grad_wait: ")


# single CTAs and pairs; more tiles than there are SMs, and fewer; sums in registers and not; pieces; rows and replicas apart, at odd elements
SHAPES = [(1, 60, 300, 200), (2, 1, 20000, 200), (2, 300, 2000, 1100), (3, 600, 9000, 72)]
CASES = [s + (dt, piece, "both", (0, 0, 0)) for s in SHAPES for dt, piece in ((torch.bfloat16, 0), (torch.bfloat16, 4000000), (torch.float32, 0))]
CASES += [(2, 300, 2000, 1100, dt, 0, which, (3, 5, 1)) for dt in (torch.bfloat16, torch.float32) for which in ("hidden", "weight")]


@pytest.mark.gpu
@pytest.mark.parametrize("R,T,V,D,dt,piece,which,layout", CASES)
def test_a_wait_that_runs_out(R, T, V, D, dt, piece, which, layout):
    h, w, y = inputs(R, T, V, D, seed=T, pad=0.3)
    stream = torch.cuda.current_stream().cuda_stream
    lse, entropy, logprob = (torch.empty((R, T), device="cuda") for _ in range(3))
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores(h, w, y, ws, logprob=logprob, entropy=entropy, lse=lse, stream=stream)
    gen = torch.Generator().manual_seed(1)
    given = dict(lse=lse, logprob=logprob, entropy=entropy, d_logprob=torch.randn((R, T), generator=gen).cuda(), d_entropy=torch.randn((R, T), generator=gen).cuda())
    out = {}
    if which != "weight":
        out["d_hidden"] = strided((R, T, D), dt, *layout, 0.0)[1]
    if which != "hidden":
        out["d_weight"] = strided((R, V, D), dt, *layout, 0.0)[1]
    ws = torch.empty(B.hdet_token_scores_grad_workspace(h, w, y, piece_bytes=piece, **out), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores_grad(h, w, y, ws, piece_bytes=piece, stream=stream, **given, **out)
    want = {k: v.clone() for k, v in out.items()}
    for _ in range(2):
        for v in out.values():
            v.zero_()
        B.hdet_selftest_token_scores_grad_wait(h, w, y, ws, piece_bytes=piece, stream=stream, **given, **out)
        torch.cuda.synchronize()
        for k, v in out.items():
            assert torch.isnan(v[:, 0, 0]).all(), k
    B.hdet_token_scores_grad(h, w, y, ws, piece_bytes=piece, stream=stream, **given, **out)
    assert all(torch.equal(out[k], want[k]) and torch.isfinite(want[k]).all() for k in want)
