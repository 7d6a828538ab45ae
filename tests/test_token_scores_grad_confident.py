"""Gradients of rows whose distribution is nearly all in one class, against 64 bits and relative to each row's own gradient."""
import pytest
import torch

from paper_2604_24708_b200 import binding as B

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _confident(T, V, D, seed=7, least=10.0, most=36.0):
    """Hidden states that point at one row of the table each; the probability of that class goes up to 1 - 1e-12 (in wide tables)."""
    gen = torch.Generator().manual_seed(seed)
    w = (torch.randn((V, D), generator=gen) * 0.05).bfloat16().cuda()
    top = torch.randperm(V, generator=gen)[:T].cuda()
    row = w[top].float()
    want = torch.linspace(least, most, T, device="cuda")[:, None] if T > 1 else torch.full((1, 1), 30.0, device="cuda")
    return (row * want / row.square().sum(1, keepdim=True)).bfloat16(), w, top


def _exact(h, w, top, y, a, b):
    """G in 64 bits.  A row of G adds up to nothing, so the entry of the likely class is less the sum of the others: nothing is taken from 1."""
    z = h.double() @ w.double().t()
    lp = z - torch.logsumexp(z, 1, keepdim=True)
    p = lp.exp()
    at = top[:, None]
    others = torch.where(torch.arange(z.shape[1], device="cuda") == at, -float("inf"), z)
    likely = -torch.log1p(torch.exp(torch.logsumexp(others, 1) - z.gather(1, at)[:, 0]))
    entropy = -likely * likely.exp() - torch.where(torch.isinf(others), 0.0, p * lp).sum(1)
    g = -p * (a[:, None] + b[:, None] * (lp + entropy[:, None]))
    if y is not None:
        g[torch.arange(len(y), device="cuda"), y] += a
    g.scatter_(1, at, 0.0)
    g.scatter_(1, at, -g.sum(1, keepdim=True))
    return z, lp, g


def _check(h, w, top, y, use, dt, piece_bytes=0, R=1):
    """R replicas of one batch and one table each (the same values)."""
    T, D = h.shape
    V = w.shape[0]
    gen = torch.Generator().manual_seed(T + D)
    a = (0.5 + torch.rand(T, generator=gen)).cuda() if "a" in use else torch.zeros(T, device="cuda")
    b = (0.5 + torch.rand(T, generator=gen)).cuda() * (-1) ** torch.arange(T, device="cuda") if "b" in use else torch.zeros(T, device="cuda")
    hr, wr = h[None].expand(R, T, D).contiguous(), w[None].expand(R, V, D).contiguous()
    yr = None if y is None else y[None].expand(R, T).int().contiguous()
    per = lambda x: x[None].expand(R, T).contiguous()  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream
    lse, entropy, logprob = (torch.empty((R, T), device="cuda") for _ in range(3))
    ws = torch.empty(B.hdet_token_scores_workspace(hr, wr, yr), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores(hr, wr, yr, ws, logprob=None if y is None else logprob, entropy=entropy, lse=lse, stream=stream)
    dh, dw = torch.empty((R, T, D), dtype=DT[dt], device="cuda"), torch.empty((R, V, D), dtype=DT[dt], device="cuda")
    ws = torch.full((B.hdet_token_scores_grad_workspace(hr, wr, yr, d_hidden=dh, d_weight=dw, piece_bytes=piece_bytes),), 0xFF, dtype=torch.uint8, device="cuda")
    B.hdet_token_scores_grad(hr, wr, yr, ws, lse, logprob=None if y is None else logprob, entropy=entropy if "b" in use else None,
                             d_logprob=per(a) if "a" in use else None, d_entropy=per(b) if "b" in use else None, d_hidden=dh, d_weight=dw,
                             piece_bytes=piece_bytes, stream=stream)
    # An entry is the sum of a part of the log probability's gradient and one of the entropy's, which are rounded apart and may cancel (a + b (lp + H)
    # passes zero in rows that are not certain): what it may be off by is relative to the sum of their magnitudes.
    z, lp, g_a = _exact(h, w, top, y, a.double(), torch.zeros_like(b, dtype=torch.float64))
    g_b = _exact(h, w, top, y, torch.zeros_like(a, dtype=torch.float64), b.double())[2]
    g, size = g_a + g_b, g_a.abs() + g_b.abs()
    # An entry's probability is off by the errors of its own logit and of the normaliser, which holds those of the likely class's.  Each is a
    # sum of products, cut by up to a step of 2^-23 for every 16 of them in runs of 512 at most, then rounded; the forward call's and this one's
    # are formed apart.  The normaliser is rounded to fp32, exponentials and the sums of entries are off by some steps.
    ez = z.amax(1).abs() * (min(D, 1024) / 16 + D / 512 + 2) * 2.0 ** -23 + 2.0 ** -16
    rel = 4 * ez + z.amax(1).abs() * 2.0 ** -22 + 2.0 ** -14
    rounding = 2.0 ** -8 if dt == "bf16" else 2.0 ** -22            # of an entry that is an operand; the result's own
    wd, hd = w.double(), h.double()
    ref_h, size_h = g @ wd, size @ wd.norm(dim=1)
    ref_w = g.t() @ hd
    size_w = size * hd.norm(dim=1)[:, None]
    for r in range(R):
        for what, off, norm, bound in (
                ("d_hidden", (dh[r].double() - ref_h).norm(dim=1), ref_h.norm(dim=1), size_h * (rel + rounding)),
                ("d_weight", (dw[r].double() - ref_w).norm(dim=1)[top], ref_w.norm(dim=1)[top], (size_w * (rel + rounding)[:, None]).sum(0)[top])):
            assert (off <= bound + norm * rounding).all(), f"{what}: rows are up to {float((off / norm).max()):.3e} of their norm off"
    return dh, dw


SIZES = [(1, 50257, 64), (1, 4099, 1088), (2, 777, 520), (130, 50257, 64), (130, 4099, 1088), (130, 700, 448), (520, 4099, 1088), (300, 2000, 2048)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_entropies_alone_without_targets(T, V, D, dt):
    h, w, top = _confident(T, V, D)
    _check(h, w, top, None, "b", dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("use", ["b", "ab"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_targets_that_are_not_the_likely_class(T, V, D, use, dt):
    h, w, top = _confident(T, V, D)
    _check(h, w, top, (top + 1 + torch.arange(T, device="cuda") % 40) % V, use, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("use", ["a", "b", "ab"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_targets_that_are_the_likely_class(T, V, D, use, dt):
    h, w, top = _confident(T, V, D)
    _check(h, w, top, top, use, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("piece_bytes", [1, 700_000, 3_000_000])
def test_pieces_of_the_vocabulary_and_groups_of_replicas(piece_bytes, dt):
    h, w, top = _confident(200, 3001, 512)
    ref = _check(h, w, top, None, "b", dt, R=3)
    got = _check(h, w, top, None, "b", dt, piece_bytes, R=3)
    assert all(torch.equal(x[0], x[1]) and torch.equal(x[0], x[2]) for x in ref + got)
    for _ in range(2):
        again = _check(h, w, top, None, "b", dt, piece_bytes, R=3)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_one_class_has_no_gradient(dt):
    """A vocabulary of one: its probability is 1 whatever the logit, and nothing moves it."""
    h, w, _ = _confident(150, 400, 64)
    w1, zero = w[:1].contiguous(), torch.zeros(150, dtype=torch.int64, device="cuda")
    dh, dw = _check(h, w1, zero, None, "b", dt)
    assert (dh == 0).all() and (dw == 0).all()


@pytest.mark.gpu
def test_rows_from_certain_to_undecided():
    """Across the border where the likely class's entry is formed from the others: 64-bit gradients on both sides of it."""
    h, w, top = _confident(512, 900, 256, least=0.5, most=14.0)
    for dt in ("f32", "bf16"):
        z = h.double() @ w.double().t()
        _check(h, w, z.argmax(1), None, "b", dt)
        _check(h, w, z.argmax(1), z.argmin(1), "ab", dt)
