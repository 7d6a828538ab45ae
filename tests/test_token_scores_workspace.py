"""One query for the most tokens and alternatives covers all calls with fewer (no GPU)."""
import ctypes as C
import random

import pytest

from paper_2604_24708_b200 import binding as B


def _need(R, T, V, D, n_top, shared):
    a = B.hdet_token_scores_args(hidden=0x1000, weight=0x2000 if D % 8 == 0 else 0x2002, n_tokens=T, vocab=V, width=D, hidden_stride=T * D, hidden_row=D,
                                 weight_stride=0 if shared else V * D, weight_row=D, n_replicas=R, n_top=n_top, hidden_dtype=B.HDET_DTYPE_BF16,
                                 weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32)
    need = C.c_int64(0)
    assert B.raw_library().hdet_token_scores_workspace(C.byref(a), C.byref(need)) == B.HDET_OK
    return need.value


@pytest.mark.parametrize("seed", range(8))
def test_fewer_alternatives_need_no_more(seed):
    rng = random.Random(seed)
    for i in range(40):
        R, T, V, D = rng.randint(1, 32), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 18)), rng.randint(1, 300)
        most = _need(R, T, V, D, min(20, V), i % 2)
        assert all(_need(R, t, V, D, k, i % 2) <= most for k in range(min(20, V) + 1) for t in (T, rng.randint(0, T)))


def test_a_table_asks_once(monkeypatch):
    import types

    import torch

    from paper_2604_24708_b200 import vocab
    asked = []
    fake = types.SimpleNamespace(HDET_DTYPE_BF16=B.HDET_DTYPE_BF16, hdet_embed_workspace=lambda *a, **k: 256, hdet_embed_grad_workspace=lambda *a, **k: 256,
                                 hdet_token_loss_workspace=lambda *a, **k: 256, hdet_token_scores_grad_workspace=lambda *a, **k: 256,
                                 hdet_token_scores_workspace=lambda *a, n_top=0, **k: asked.append(n_top) or 1024)
    monkeypatch.setattr(vocab, "B", fake)
    table = torch.zeros((2, 10, 4))
    arena = types.SimpleNamespace(numels=[40], n=2, device="cpu", shared_grad=False, param_view=lambda k, shape: table, grad_view=lambda k, shape: table)
    bound = vocab.TiedTable(arena, 0, 10, 4, 3, scores=True, n_top=20)
    assert asked == [10] and bound.n_top == 10 and bound.workspace.numel() == 1024
