"""Logits that are large, up to the ends of fp32's range: what counts is how far they lie apart."""
import pytest
import torch

from paper_2604_24708_b200 import binding as B

SIZES = [(1, 4099), (2, 4099), (40, 4099), (300, 8200), (1400, 50257)]      # few tokens; kept logits in single CTAs and pairs; lists


def _run(h, w, y, n_top=3):
    T = h.shape[1]
    out = {k: torch.empty((1, T), device="cuda") for k in ("logprob", "entropy", "lse")}
    out.update(top_ids=torch.empty((1, T, n_top), dtype=torch.int32, device="cuda"), top_logprob=torch.empty((1, T, n_top), device="cuda"))
    plain = {k: torch.empty_like(v) for k, v in out.items() if not k.startswith("top")}
    for o, n in ((out, n_top), (plain, 0)):
        ws = torch.empty(B.hdet_token_scores_workspace(h, w, y, n_top=n), dtype=torch.uint8, device="cuda")
        B.hdet_token_scores(h, w, y, ws, stream=torch.cuda.current_stream().cuda_stream, **o)
    for k, v in plain.items():                            # without alternatives: other readers, the same sums but for their order
        assert ((v - out[k]).abs() <= 2.0 ** -16 * v.abs()).all(), k
    return {k: v[0] for k, v in out.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("size", [24.0, 250.0, 2000.0, -2992.0, 7936.0, 32640.0, -65280.0])
def test_exact_logits_far_from_zero(T, V, size):
    """All logits are `size` less at most 24, and exact in fp32: log probability and entropy are those of the differences."""
    gen = torch.Generator().manual_seed(1)
    gap = (8 + torch.randint(0, 64, (V,), generator=gen).double() / 8)           # multiples of an eighth below 16: exact
    gap[V // 3] = 0.0
    w = torch.zeros((1, V, 64), dtype=torch.bfloat16)
    w[0, :, 3], w[0, :, 40] = 1.0, -gap.bfloat16()
    h = torch.zeros((1, T, 64), dtype=torch.bfloat16)
    h[0, :, 3], h[0, :, 40] = size, 1.0
    assert float(h[0, 0, 3]) == size and torch.equal(w[0, :, 40].double(), -gap)
    out = _run(h.cuda(), w.cuda(), torch.full((1, T), V // 3, dtype=torch.int32, device="cuda"))
    delta = torch.exp(-gap).sum() - 1
    lp = -torch.log1p(delta)
    entropy = -lp + (torch.exp(-gap) * gap).sum() / (1 + delta)
    # exponentials of a difference d: 2^-22 of their value and d times half a step of fp32; sums by their additions (16 within 64 columns, one for every
    # 64, those of the parts)
    rel = (4 + 16) * 2.0 ** -22 + (16 + V / 64 + 60) * 2.0 ** -24
    assert ((out["logprob"].double() - lp).abs() <= rel * lp.abs()).all()
    assert ((out["entropy"].double() - entropy).abs() <= rel * entropy).all()
    assert ((out["lse"].double() - (size - lp)).abs() <= abs(size) * 2.0 ** -24 + rel).all()
    assert (out["top_ids"][:, 0] == V // 3).all() and torch.equal(out["top_logprob"][:, 0], out["logprob"])


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("top,rest", [(3e38, -3e38), (3e38, 0.0), (0.0, -3e38), (-1e37, -2e38), (-1e38, -3e38), (-2.6e38, -3e38), (1e36, -1e36), (3e38, 2.6e38)])
def test_logits_up_to_the_ends_of_the_range(T, V, top, rest):
    """Two classes share the probability; the others are so far below that nothing is left of them."""
    one = 2.0 ** 64
    w = torch.full((1, V, 64), 0.0)
    w[0, :, 7] = rest / one
    w[0, [5, V - 2], 7] = top / one
    h = torch.zeros((1, T, 64), dtype=torch.bfloat16)
    h[0, :, 7] = one
    w = w.bfloat16()
    high, low = float(w[0, 5, 7]) * one, float(w[0, 0, 7]) * one          # exact products
    assert torch.isfinite(torch.tensor([high, low])).all() and high > low
    out = _run(h.cuda(), w.cuda(), torch.full((1, T), 5, dtype=torch.int32, device="cuda"), n_top=2)
    log2 = torch.tensor(2.0, dtype=torch.float64).log()
    assert ((out["logprob"].double() + log2).abs() <= 2.0 ** -22).all() and ((out["entropy"].double() - log2).abs() <= 2.0 ** -22).all()
    assert ((out["lse"].double() - high).abs() <= abs(high) * 2.0 ** -24 + 1).all()
    assert (out["top_ids"] == torch.tensor([5, V - 2], device="cuda")).all() and ((out["top_logprob"].double() + log2).abs() <= 2.0 ** -22).all()
    # one class alone: certain
    w[0, V - 2, 7] = rest / one
    out = _run(h.cuda(), w.cuda(), torch.full((1, T), 5, dtype=torch.int32, device="cuda"), n_top=1)
    assert (out["logprob"] == 0).all() and (out["entropy"] == 0).all() and (out["top_ids"] == 5).all() and (out["top_logprob"] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("last", [2.8e38, -1e38])
def test_logits_that_rise_through_the_range(T, V, last):
    """Every maximum is left behind by a far larger one, in each part of the table."""
    one = 2.0 ** 64
    w = torch.zeros((1, V, 64))
    w[0, :, 7] = torch.linspace(-3e38 / one, last / one, V // 64 + 1).repeat_interleave(64)[:V]
    w[0, V - 1, 7] = 1.02 * w[0, :, 7].max() if last > 0 else 0.9 * w[0, :, 7].max()
    h = torch.zeros((1, T, 64), dtype=torch.bfloat16)
    h[0, :, 7] = one
    out = _run(h.cuda(), w.bfloat16().cuda(), torch.full((1, T), V - 1, dtype=torch.int32, device="cuda"), n_top=1)
    assert (out["logprob"] == 0).all() and (out["entropy"] == 0).all() and (out["top_ids"] == V - 1).all()
    assert ((out["lse"].double() - float(w.bfloat16()[0, V - 1, 7]) * one).abs() <= abs(last) * 2.0 ** -23).all()
