"""A mean loss and an entropy term of one's own through the same table: the second gradient is added to the first."""
import pytest
import torch

from test_scores_training import _setup
from paper_2604_24708_b200 import binding as B


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_tables_gradients_add_up(dtype):
    n, T, V, D, beta = 2, 150, 600, 64, 0.05
    arena, h, table, ids, out, gen = _setup(n, T, V, D, dtype, B.HDET_OPT_SGD)
    hidden, y = torch.randn((n, T, D), generator=gen, device="cuda").bfloat16(), ids[:, 1:].contiguous()
    losses, d_first, d_second = torch.zeros(n, device="cuda"), torch.empty((n, T, D), dtype=dtype, device="cuda"), torch.empty((n, T, D), dtype=dtype, device="cuda")
    table.scores(hidden, y, **out)
    given = dict(logprob=out["logprob"], entropy=out["entropy"], d_entropy=torch.full((n, T), -beta / T, device="cuda"))
    table.scores_grad(hidden, y, out["lse"], d_second, **given)
    second = table.grad.clone()
    table.loss(hidden, y, losses, d_hidden=d_first)
    first = table.grad.clone()
    again = torch.empty_like(d_second)
    table.scores_grad(hidden, y, out["lse"], again, accumulate=True, **given)
    assert torch.equal(again, d_second)
    if dtype == torch.float32:
        assert torch.equal(table.grad, first + second)
    else:                                     # `second` was rounded before it could be added here, there the sum is
        off = (table.grad.double() - first.double() - second.double()).abs()
        assert (off <= 2.0 ** -8 * (second.double().abs() + table.grad.double().abs()) * 1.001).all()
    B.hdet_destroy(h)
