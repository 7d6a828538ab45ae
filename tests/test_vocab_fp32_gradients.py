"""What gradients in fp32 are good for: the softmax's gradient G goes into the products as three bf16 numbers, and their sums leave the
tensor cores, which cut instead of rounding, every 512 products.

Logits are small and exact in fp32 (multiples of 2^-6), so that neither they nor the exponentials' arguments (between -8 and 0) hide either.
"""
import pytest
import torch

from paper_2604_24708_b200 import binding as B

# An entry of G: ex2 (2^-22) and its argument (2^-22, times ln 2), its product with 1 / sum and that quotient (2^-23 together), the sum
# of exponentials, each off by 2^-21 as above and added in fewer than 64 steps (2^-24 each)
E_G = 2.0 ** -21 + 2.0 ** -23 + 2.0 ** -21 + 64 * 2.0 ** -24

ONE = 255 / 128        # eight bits, so that its products with G have sixteen: sums of them are cut


def _inputs(T, V, D, seed):
    gen = torch.Generator().manual_seed(seed)
    h = torch.randint(-4, 5, (1, T, D), generator=gen).float() / 8
    w = torch.randint(-1, 2, (1, V, D), generator=gen).float() / 8
    h[..., 0], w[..., 0] = ONE, 0.0
    return h.bfloat16().cuda(), w.bfloat16().cuda()


def _gradients(h, w, y):
    (_, T, D), V = h.shape, w.shape[1]
    loss, dh, dw = torch.empty(1, device="cuda"), torch.empty((1, T, D), device="cuda"), torch.empty((1, V, D), device="cuda")
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=dh, d_weight=dw), dtype=torch.uint8, device="cuda")
    B.hdet_token_loss(h, w, y, loss, ws, d_hidden=dh, d_weight=dw, stream=torch.cuda.current_stream().cuda_stream)
    z = h[0].double() @ w[0].double().t()
    assert float(z.max() - z.min()) < 5
    g = torch.softmax(z, 1)
    g[torch.arange(T, device="cuda"), y[0].long()] -= 1.0
    return dh[0].double(), dw[0].double(), g


@pytest.mark.gpu
@pytest.mark.parametrize("V", [300, 20000])
def test_three_terms(V):
    """One token: every row of the table's gradient is an entry of G times the hidden state.  Two bf16 numbers would be off by up to 2^-16,
    over four times the bound."""
    h, w = _inputs(1, V, 64, V)
    y = torch.tensor([[V // 2]], dtype=torch.int32, device="cuda")
    _, dw, g = _gradients(h, w, y)
    assert 2 * E_G < 2.0 ** -16
    ref = g.t() @ h[0].double()
    # three terms leave 2^-24, and are added up with fewer than eight steps of 2^-23
    assert ((dw - ref).abs() <= ref.abs() * (E_G + 2.0 ** -24 + 2.0 ** -20)).all(), float(((dw - ref).abs() / ref.abs().clamp(min=1e-30)).max())


@pytest.mark.gpu
def test_sums_of_one_sign():
    """30000 tokens that share a hidden state: a class that is nobody's target sums 30000 positive numbers, with 1875 cuts.  Bounded by the partial sums
    since the sum was last taken out; a sum left in the tensor cores would be some 4e-5 off."""
    T, V, D = 30000, 130, 16
    h, w = _inputs(T, V, D, 1)
    y = torch.randint(100, V, (1, T), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).int()
    _, dw, g = _gradients(h, w, y)
    p = g[:, :100] * ONE
    parts = torch.nn.functional.pad(p, (0, 0, 0, -T % 512)).view(-1, 32, 16, 100).sum(2)         # of 16 tokens, 32 of them a chunk
    cuts = parts.cumsum(1).sum((0, 1)) * 2.0 ** -23
    total = p.sum(0)
    # the two smaller terms' cuts are 2^-8 of these; the chunks of all three terms are added with half a step each, those of the small terms to
    # sums 2^-7 as large
    bound = cuts * (1 + 2.0 ** -7) + total * (len(parts) * (1 + 2.0 ** -6) * 2.0 ** -24 + E_G + 2.0 ** -22)
    got = dw[:100, 0] * T
    assert float((bound / total).max()) < 2e-5
    assert ((got - total).abs() <= bound).all(), float(((got - total).abs() / bound).max())
