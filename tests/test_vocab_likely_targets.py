"""Token loss where targets are likely and logits large: bounds relative to the loss and to the row of the softmax's gradient.

Hidden states and tables are small multiples of powers of two, so every logit is exact in fp32 whatever the order of its sum, and all
that is left to err is the softmax.  With d = log(sum of exp over the other classes) - z_target, loss = log(1 + exp d) and the
target's gradient is -1 / (1 + exp -d): both have the relative error that d has as an absolute one.
"""
import pytest
import torch

from paper_2604_24708_b200 import binding as B

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _inputs(R, T, V, D, seed):
    """Targets' logits lean from 0 to 8 times |w|^2: probabilities from 1 / V to 1 - 1e-40, logits up to some hundreds."""
    gen = torch.Generator().manual_seed(seed)
    w = torch.randint(-4, 5, (R, V, D), generator=gen).float() / 8
    y = torch.randint(0, V, (R, T), generator=gen)
    lean = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.5, 2.0, 4.0, 8.0])[torch.randint(0, 9, (R, T, 1), generator=gen)]
    rows = torch.stack([w[r][y[r]] for r in range(R)])
    h = torch.randint(-4, 5, (R, T, D), generator=gen).float() / 8 + (lean * rows * 8).round() / 8
    assert torch.equal(h, h.bfloat16().float()) and torch.equal(w, w.bfloat16().float())
    return h.bfloat16().cuda(), w.bfloat16().cuda(), y.int().cuda()


def _reference(h, w, y):
    """d, losses, G of one replica in 64 bits."""
    z, at = h.double() @ w.double().t(), torch.arange(len(y), device="cuda")
    own = z[at, y.long()]
    z[at, y.long()] = float("-inf")
    d = torch.logsumexp(z, 1) - own
    small = torch.log1p(torch.exp(-d.abs()))
    loss = d.clamp(min=0) + small
    g = torch.exp(z - (own + d.clamp(min=0) + small)[:, None])
    g[at, y.long()] = -torch.sigmoid(d)
    return d, loss, g


def _error_of_d(d, V):
    """What d may be off by.  The sum of exp: each term by ex2 (2^-22) and its argument's rounding, of which terms that count have one
    below 32 (2^-20), and fewer than 64 + V / 4096 additions in a row (2^-24 each); its logarithm, at most log2 V + 1, and z log2 e - k
    by 2^-24 each; log2 e as a constant, 2^-26 of the logits' distances, below 4 |d| + 64 here."""
    return 2.0 ** -22 + 2.0 ** -20 + (64 + V / 4096) * 2.0 ** -24 + (32 + 4 * d.abs()) * 2.0 ** -23


def _run(h, w, y, dt=None, piece_bytes=0):
    R, T, D, V = h.shape[0], h.shape[1], h.shape[2], w.shape[1]
    out = dict(loss=torch.empty(R, dtype=torch.float64, device="cuda"), token_loss=torch.empty((R, T), device="cuda"))
    if dt:
        out.update(d_hidden=torch.empty((R, T, D), dtype=DT[dt], device="cuda"), d_weight=torch.empty((R, V, D), dtype=DT[dt], device="cuda"))
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=out.get("d_hidden"), d_weight=out.get("d_weight"), piece_bytes=piece_bytes),
                     dtype=torch.uint8, device="cuda")
    B.hdet_token_loss(h, w, y, workspace=ws, piece_bytes=piece_bytes, stream=torch.cuda.current_stream().cuda_stream, **out)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 3, 4, 90, 300])
@pytest.mark.parametrize("V,D", [(2, 64), (1000, 128), (7001, 264)])
def test_losses(T, V, D):
    h, w, y = _inputs(2, T, V, D, seed=T + V)
    for dt in (None, "bf16"):                        # with gradients the loss takes another way
        out = _run(h, w, y, dt)
        for r in range(2):
            d, loss, _ = _reference(h[r], w[r], y[r])
            got = out["token_loss"][r].double()
            assert (got >= 0).all()
            # a relative error of e_d, and exp, log1p and the roundings of d <= |d| 2^-23 more; below 2^-126 fp32 has no full precision
            assert ((got - loss).abs() <= loss * (_error_of_d(d, V) + (8 + d.abs()) * 2.0 ** -23) + 2.0 ** -126).all()
            assert abs(float(out["loss"][r]) - float(loss.mean())) <= float((loss * (_error_of_d(d, V) + (8 + d.abs()) * 2.0 ** -23)).mean()) + 2.0 ** -126


@pytest.mark.gpu
@pytest.mark.parametrize("T", [90, 300])
@pytest.mark.parametrize("dt,piece", [("f32", 0), ("f32", 1), ("bf16", 0), ("bf16", 1)])
def test_gradients(T, dt, piece):
    R, V, D = 2, 3000, 128
    h, w, y = _inputs(R, T, V, D, seed=T)
    out = _run(h, w, y, dt, piece)
    for r in range(R):
        d, _, g = _reference(h[r], w[r], y[r])
        # an entry of G: as the loss, and its own exponential and its argument (of at most 126); G as operand: bf16, or three terms; bf16
        # only: numerators of 2^-11, and zero for those below 2^-61 of the row's largest
        e = _error_of_d(d, V) + (16 + 126 + d.abs()) * 2.0 ** -23 + (2.0 ** -24 if dt == "f32" else 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18)
        a, wa = g.abs(), w[r].double().abs()
        size = a @ wa
        flush = 0.0 if dt == "f32" else 2.0 ** -61 * V * a.amax(1, keepdim=True) * float(wa.max())
        # sums of V products: cut every 16 products, at most 2^-23 of the magnitudes, and one addition a chunk
        steps = V / 16 + 8
        ref = g @ w[r].double() / T
        got = out["d_hidden"][r].double()
        bound = (size * (e[:, None] + steps * 2.0 ** -23) + flush) / T + ref.abs() * (torch.finfo(DT[dt]).eps / 2 + 2.0 ** -22)
        # Below 2^-126 no relative error holds (targets with d < -80): ex2.approx.ftz gives zero there, and a term of G or the result has
        # fewer bits the smaller it is, a bf16 one none below 2^-133.  Each entry of G, and the result, is off by 2^-126 at most for that.
        bound += float(wa.sum(0).max()) * 2.0 ** -126 / T + 2.0 ** -126
        assert ((got - ref).abs() <= bound).all(), float(((got - ref).abs() / bound).max())
        # and in norm, each token's row beside its own (rows as small as 1e-17 of the others' among them)
        far = (got - ref).norm(dim=1) / ref.norm(dim=1)
        some = d > -60                               # what bf16 and fp32 hold with full precision after the division by T
        assert (far[some] <= (2.0 ** -7 if dt == "bf16" else 2.0 ** -14)).all(), float(far[some].max())
        if dt == "f32":
            ha = h[r].double().abs()
            ref = g.t() @ h[r].double() / T
            bound = ((a * e[:, None]).t() @ ha + (a.t() @ ha) * (T / 16 + 8) * 2.0 ** -23) / T + ref.abs() * 2.0 ** -22
            bound += float(ha.sum(0).max()) * 2.0 ** -126 / T + 2.0 ** -126
            assert ((out["d_weight"][r].double() - ref).abs() <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 20, 300])
def test_one_class_and_classes_without_weight(T):
    """One class: nothing to learn.  Classes of logit -inf beside a finite target: the same.  A target of logit -inf: an infinite loss; of
    +inf, or with no finite logit at all: NaN."""
    h = torch.ones((1, T, 8), dtype=torch.bfloat16, device="cuda")
    for V, w in [(1, torch.full((1, 1, 8), 3.0)), (300, torch.full((1, 300, 8), float("-inf")))]:
        w[0, 0] = 3.0
        out = _run(h, w.bfloat16().cuda(), torch.zeros((1, T), dtype=torch.int32, device="cuda"))
        assert (out["token_loss"] == 0).all() and float(out["loss"]) == 0
    out = _run(h, torch.full((1, 1, 8), 3.0).bfloat16().cuda(), torch.zeros((1, T), dtype=torch.int32, device="cuda"), "f32")
    assert not out["d_hidden"].any() and not out["d_weight"].any()
    for own, other, want in [(float("-inf"), 1.0, float("inf")), (float("inf"), 1.0, None), (float("-inf"), float("-inf"), None), (float("nan"), 1.0, None)]:
        w = torch.full((1, 300, 8), other)
        w[0, 5] = own
        out = _run(h, w.bfloat16().cuda(), torch.full((1, T), 5, dtype=torch.int32, device="cuda"))
        assert (torch.isnan(out["token_loss"]) if want is None else out["token_loss"] == want).all(), (own, other)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [90, 300])
@pytest.mark.parametrize("dt,piece", [("f32", 0), ("bf16", 0), ("bf16", 1)])
def test_gradients_of_unlikely_classes(T, dt, piece):
    """Every class's row of the table's gradient beside its own size, down to classes of probability 1e-25."""
    R, V, D = 1, 900, 128
    gen = torch.Generator().manual_seed(T)
    w = torch.randint(-4, 5, (R, V, D), generator=gen).float() / 8
    w *= torch.tensor([0.0, 0.5, 1.0, 2.0])[torch.randint(0, 4, (R, V, 1), generator=gen)]
    h = torch.randint(-4, 5, (R, T, D), generator=gen).float() / 2
    h[..., 0], w[..., 0] = 8.0, torch.randint(-4, 1, (R, V), generator=gen).float() / 2      # classes that are unlikely for every token
    h, w, y = h.bfloat16().cuda(), w.bfloat16().cuda(), torch.randint(0, V, (R, T), generator=gen).int().cuda()
    out = _run(h, w, y, dt, piece)
    d, _, g = _reference(h[0], w[0], y[0])
    a, ha = g.abs(), h[0].double().abs()
    assert float(a.amax(0).min()) < 1e-12 and float(a[a > 0].min()) < 1e-25
    e = _error_of_d(d, V) + (16 + 126 + d.abs()) * 2.0 ** -23 + (2.0 ** -24 if dt == "f32" else 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18)
    ref = g.t() @ h[0].double() / T
    bound = ((a * e[:, None]).t() @ ha + (a.t() @ ha) * (T / 16 + 8) * 2.0 ** -23) / T + ref.abs() * (torch.finfo(DT[dt]).eps / 2 + 2.0 ** -22)
    if dt == "bf16" and not piece:                   # what counts as zero: 2^-62 of a neighbour, twice that for its unit
        bound += (2.0 ** -61 * a.amax(1, keepdim=True)).expand_as(a).t() @ ha / T
    got = out["d_weight"][0].double()
    assert ((got - ref).abs() <= bound).all(), float(((got - ref).abs() / bound).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [None, "bf16", "f32"])
def test_wide_logits_of_one_sign(dt):
    """The tensor cores cut a sum towards zero after every 16 products, and where the products have one sign the cuts add up.  They are
    bounded by the partial sums since the last time the sum was taken out, every 16 x 64 products (8 x 64 for fp32 gradients)."""
    T, V, D = 40, 200, 4096
    gen = torch.Generator().manual_seed(1)
    w = (torch.randn((1, V, D), generator=gen) * 0.02).bfloat16()
    y = torch.randint(0, V, (1, T), generator=gen)
    lean = torch.where(torch.rand((1, T, 1), generator=gen) < 0.5, -1.0, 1.0) * (0.5 + torch.rand((1, T, D), generator=gen)) * 0.4
    h = (lean * torch.sign(w[0].float())[y]).bfloat16().cuda()                 # |z| of the targets about 25
    w, y = w.cuda(), y.int().cuda()
    out = _run(h, w, y, dt)
    chunk = 64 * (8 if dt == "f32" else 16)
    parts = (h[0].double()[:, None] * w[0].double()[None]).view(T, V, D // 16, 16).sum(-1)         # of 16 products
    cuts = parts.view(T, V, D // chunk, chunk // 16).cumsum(-1).abs()
    ez = cuts.sum((-1, -2)) * 2.0 ** -23 + cuts[..., -1].sum(-1) * 2.0 ** -24
    d, loss, g = _reference(h[0], w[0], y[0])
    at = torch.arange(T, device="cuda")
    own = ez[at, y[0].long()]
    others = torch.where(g > 0, g, 0.0)
    e = own + (others * ez).sum(1) / others.sum(1) + _error_of_d(d, V)
    got = out["token_loss"][0].double()
    assert float(d.min()) < -15 and float(d.max()) > 15
    bound = e * -g[at, y[0].long()] + loss * (8 + d.abs()) * 2.0 ** -23         # the derivative of the loss by d is that of -G's entry
    assert ((got - loss).abs() <= bound).all(), float(((got - loss).abs() / bound).max())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 20, 300])
@pytest.mark.parametrize("power", [10, 28, 31, 60, 120])
def test_huge_logits(T, power):
    """Logits that are whole multiples of a large power of two: the classes of the largest share all of the probability, and the losses of
    the others are the distances to it.  Neither is uncertain, whatever the logits' size."""
    V, D = 300, 64
    gen = torch.Generator().manual_seed(power)
    w = torch.zeros((1, V, D))
    w[0, :, 0] = torch.randint(-3, 4, (V,), generator=gen).float()
    h = torch.zeros((1, T, D))
    h[..., 0] = 2.0 ** power
    y = torch.randint(0, V, (1, T), generator=gen).int().cuda()
    top = w[0, :, 0] == 3
    for dt in (None, "f32", "bf16"):
        out = _run(h.bfloat16().cuda(), w.bfloat16().cuda(), y, dt)
        n = int(top.sum())
        steps = 3 - w[0, y[0].cpu().long(), 0].double()
        loss = torch.where(steps > 0, steps * 2.0 ** power, 0.0) + torch.log(torch.tensor(float(n)).double())
        got = out["token_loss"][0].double().cpu()
        assert ((got - loss).abs() <= loss * 2.0 ** -21).all()        # ex2, log, log1p, two additions: 2^-22 and four times 2^-24
        if dt:
            g = top.double().repeat(T, 1) / n
            g[torch.arange(T), y[0].cpu().long()] -= 1.0
            ref = g.t() @ h[0].double() / T
            bound = (g.abs().t() @ h[0].double() / T) * (2.0 ** -20 if dt == "f32" else 2.0 ** -8 + 2.0 ** -10) + ref.abs() * torch.finfo(DT[dt]).eps
            assert ((out["d_weight"][0].double().cpu() - ref).abs() <= bound).all()
