"""Gradients for given gradients of log probabilities and entropies against 64-bit formulas and differences; refusals."""
import ctypes as C

import pytest
import torch

from paper_2604_24708_b200 import binding as B
from test_token_scores import inputs, reference, strided

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = 7.25


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def _args(**kw):
    a = B.hdet_token_scores_args(
        hidden=0x1000, weight=0x2000, targets=0x3000, logprob=0x4000, entropy=0x5000, lse=0x6000, d_logprob=0x7000, d_entropy=0x8000,
        d_hidden=0x9000, d_weight=0xA000, n_tokens=4, vocab=10, width=8, hidden_stride=32, hidden_row=8, weight_stride=80, weight_row=8,
        target_stride=4, logprob_stride=4, entropy_stride=4, lse_stride=4, d_logprob_stride=4, d_entropy_stride=4, d_hidden_stride=32,
        d_hidden_row=8, d_weight_stride=80, d_weight_row=8, n_replicas=2, hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16,
        target_dtype=B.HDET_DTYPE_I32, d_hidden_dtype=B.HDET_DTYPE_BF16, d_weight_dtype=B.HDET_DTYPE_F32)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


ARG, ALIGN, UNSUP = B.HDET_ERR_INVALID_ARG, B.HDET_ERR_ALIGN, B.HDET_ERR_UNSUPPORTED
BAD = [
    (dict(n_replicas=0), ARG), (dict(n_tokens=-1), ARG), (dict(vocab=0), ARG), (dict(width=0), ARG), (dict(target_dtype=B.HDET_DTYPE_F32), ARG),
    (dict(hidden_dtype=B.HDET_DTYPE_F32), UNSUP), (dict(d_hidden_dtype=B.HDET_DTYPE_F64), ARG), (dict(d_weight_dtype=7), ARG), (dict(device=-1), ARG),
    (dict(piece_bytes=-1), ARG), (dict(hidden_row=7), ARG), (dict(d_hidden_row=7), ARG), (dict(d_weight_row=7), ARG),
    (dict(d_weight_row=B.HDET_MAX_ROW_STRIDE + 1), ARG), (dict(hidden=None), ARG), (dict(weight=None), ARG), (dict(d_hidden=None, d_weight=None), ARG),
    (dict(d_logprob=None, d_entropy=None), ARG), (dict(lse=None), ARG), (dict(logprob=None), ARG), (dict(entropy=None), ARG), (dict(targets=None), ARG),
    (dict(hidden_stride=31), ARG), (dict(weight_stride=79), ARG), (dict(target_stride=3), ARG), (dict(lse_stride=3), ARG), (dict(logprob_stride=1), ARG),
    (dict(entropy_stride=2), ARG), (dict(d_logprob_stride=3), ARG), (dict(d_entropy_stride=-4), ARG), (dict(d_hidden_stride=0), ARG), (dict(d_weight_stride=79), ARG),
    (dict(d_hidden=0x1000, d_hidden_dtype=B.HDET_DTYPE_F32), ARG), (dict(d_hidden=0x1000, d_hidden_row=16, d_hidden_stride=64), ARG),
    (dict(hidden=0x1001), ALIGN), (dict(weight=0x2001), ALIGN), (dict(targets=0x3002), ALIGN), (dict(logprob=0x4001), ALIGN), (dict(entropy=0x5002), ALIGN),
    (dict(lse=0x6002), ALIGN), (dict(d_logprob=0x7002), ALIGN), (dict(d_entropy=0x8001), ALIGN), (dict(d_hidden=0x9001), ALIGN), (dict(d_weight=0xA002), ALIGN),
]


@pytest.mark.parametrize("change,status", BAD, ids=[str(b[0]) for b in BAD])
def test_refusals(change, status):
    a, lib = _args(**change), B.raw_library()
    assert lib.hdet_token_scores_grad(C.byref(a), 0x10000, 1 << 50, None) == status
    assert lib.hdet_last_error(None).startswith(b"hdet_token_scores_grad: ")


def test_refusals_of_workspaces():
    lib, need, none = B.raw_library(), C.c_int64(0), C.c_int64(1)
    assert lib.hdet_token_scores_grad_workspace(C.byref(_args()), C.byref(need)) == B.HDET_OK and need.value >= 256
    assert lib.hdet_token_scores_grad(C.byref(_args()), None, need.value, None) == ARG
    assert lib.hdet_token_scores_grad(C.byref(_args()), 0x10000, 255, None) == ARG
    assert lib.hdet_token_scores_grad(C.byref(_args()), 0x10010, need.value, None) == ALIGN
    assert lib.hdet_token_scores_grad(None, 0x10000, need.value, None) == ARG
    assert lib.hdet_token_scores_grad_workspace(C.byref(_args()), None) == ARG
    assert lib.hdet_token_scores_grad_workspace(C.byref(_args(vocab=0)), C.byref(none)) == ARG and none.value == 0
    for t in (1, 2, 3, 63, 64):
        assert lib.hdet_token_scores_grad_workspace(C.byref(_args(n_tokens=t, n_replicas=1)), C.byref(none)) == B.HDET_OK
        assert none.value <= 1 << 30


# ------------------------------------------------------------------------------------------------ the formula
def _formula(z, y, a, b):
    """G of one replica's logits z [T, V] in 64 bits; y None or [T]."""
    lp = torch.log_softmax(z, 1)
    p = lp.exp()
    entropy = -(p * lp).sum(1, keepdim=True)
    g = -p * (a[:, None] + b[:, None] * (lp + entropy))
    if y is not None:
        g[torch.arange(len(y), device=z.device), y] += a
    return g, p, lp, entropy


def test_the_formula_is_the_gradient():
    gen = torch.Generator().manual_seed(0)
    z = torch.randn((5, 11), generator=gen, dtype=torch.float64) * 3
    y, a, b = torch.tensor([0, 3, 10, 3, 7]), torch.randn(5, generator=gen, dtype=torch.float64), torch.randn(5, generator=gen, dtype=torch.float64)

    def value(z):
        lp = torch.log_softmax(z, 1)
        return (a * lp[torch.arange(5), y]).sum() + (b * -(lp.exp() * lp).sum(1)).sum()
    g = _formula(z, y, a, b)[0]
    leaf = z.clone().requires_grad_()
    value(leaf).backward()
    assert (leaf.grad - g).abs().max() <= 1e-13
    for _ in range(4):
        d = torch.randn(z.shape, generator=gen, dtype=torch.float64)
        # the third derivative's part of a central difference is 1e-8 of the values; rounding 1e-16 / 1e-4
        assert abs(float((value(z + 1e-4 * d) - value(z - 1e-4 * d)) / 2e-4 - (g * d).sum())) <= 1e-6


# ------------------------------------------------------------------------------------------------ against 64 bits
def _reference(h, w, y, a, b, h_two, w_two):
    T, D = h.shape
    V = w.shape[0]
    fwd, tol_f, *_ = reference(h, w, y, 0)
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if y is None else (y >= 0) & (y < V)
    t = keep.nonzero()[:, 0]
    dh, e_dh = torch.zeros((T, D), dtype=torch.float64, device="cuda"), torch.zeros((T, D), dtype=torch.float64, device="cuda")
    dw, e_dw = torch.zeros((V, D), dtype=torch.float64, device="cuda"), torch.zeros((V, D), dtype=torch.float64, device="cuda")
    if len(t) == 0:
        return dh, e_dh, dw, e_dw
    hd, wd, a, b = h[t].double(), w.double(), a[t].double(), b[t].double()
    z = hd @ wd.t()
    g, p, lp, entropy = _formula(z, None if y is None else y[t].long(), a, b)
    # what a logarithm, the entropy and the given token's logarithm may be off by, as the forward call left them and as they are formed again
    e_lp = (hd.abs() @ wd.abs().t()) * D * 2.0 ** -23 + tol_f["lse"][t][:, None] + fwd["lse"][t].abs()[:, None] * 2.0 ** -23
    e_h = tol_f["entropy"][t][:, None] + entropy * 2.0 ** -23
    steps = (4 + lp.abs()) * 2.0 ** -22                   # of the exponential and of what it is multiplied with
    size = p * (a.abs()[:, None] + b.abs()[:, None] * (lp.abs() + entropy))
    e_g = size * (steps + e_lp) + p * b.abs()[:, None] * (e_lp + e_h)
    if y is not None:
        rows = torch.arange(len(t), device="cuda")
        yy = y[t].long()
        e_g[rows, yy] += p[rows, yy] * a.abs() * tol_f["logprob"][t] + a.abs() * 2.0 ** -22
    e_gh = e_g + g.abs() * (2.0 ** -16 if h_two else 2.0 ** -8)
    e_gw = e_g + g.abs() * (2.0 ** -16 if w_two else 2.0 ** -8)
    dh[t] = g @ wd
    e_dh[t] = e_gh @ wd.abs() + (g.abs() @ wd.abs()) * V * 2.0 ** -23
    dw = g.t() @ hd
    e_dw = e_gw.t() @ hd.abs() + (g.abs().t() @ hd.abs()) * len(t) * 2.0 ** -23
    return dh, e_dh, dw, e_dw


def _within(got, ref, tol, dtype, what, two):
    got = got.double()
    assert torch.isfinite(got).all(), what
    far = (got - ref).abs() - (tol + ref.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -22))
    assert (far <= 0).all(), f"{what}: {float(far.max()):.3e} over the bound"
    # worst cases; errors that are independent add up to far less: bf16 has two roundings of 2^-8 at most, fp32 gradients sums of steps of 2^-24
    norm = float(ref.norm())
    if norm > 0:
        assert float((got - ref).norm()) <= norm * (2.0 ** -15 if two else 2.0 ** -7), what


def _given(R, T, y, V, seed):
    """Gradients whose values at padding are NaN."""
    gen = torch.Generator().manual_seed(seed)
    a, b = torch.randn((R, T), generator=gen).cuda() / T, (torch.randn((R, T), generator=gen).cuda() * 0.3 / T)
    if y is not None:
        some = (y >= 0) & (y < V)
        a, b = torch.where(some, a, float("nan")), torch.where(some, b, float("nan"))
    return a, b


def _run(h, w, y, dh_dt="bf16", dw_dt="bf16", use="ab", layout=(0, 0, 0), accumulate=False, piece_bytes=0, in_place=False, seed=0, ws_fill=None):
    R = max(h.shape[0] if h.dim() == 3 else 1, w.shape[0] if w.dim() == 3 else 1)
    T, D, V = h.shape[-2], h.shape[-1], w.shape[-2]
    stream = torch.cuda.current_stream().cuda_stream
    lse, entropy, logprob = (torch.empty((R, T), device="cuda") for _ in range(3))
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores(h, w, y, ws, logprob=None if y is None else logprob, entropy=entropy, lse=lse, stream=stream)
    a, b = _given(R, T, y, V, seed)
    if y is not None:                                     # nothing is read at padding
        some = (y >= 0) & (y < V)
        lse, entropy, logprob = (torch.where(some, x, float("nan")) for x in (lse, entropy, logprob))
    pad_row, pad_rep, shift = layout
    dh = dw = start = None
    bufs = []
    hidden = h
    if dh_dt:
        buf, dh = strided((R, T, D), DT[dh_dt], pad_row, pad_rep, shift, GUARD)
        bufs.append((buf, dh))
        dh.fill_(float("nan"))
        if in_place:
            dh.copy_(h)
            hidden = dh
    if dw_dt:
        buf, dw = strided((R, V, D), DT[dw_dt], pad_row, pad_rep, shift, GUARD)
        bufs.append((buf, dw))
        gen = torch.Generator().manual_seed(3)
        dw.copy_(torch.randn(dw.shape, generator=gen) * 1e-2 if accumulate else torch.full((1,), float("nan")))
        start = dw.double() if accumulate else None
    ws = torch.empty(B.hdet_token_scores_grad_workspace(hidden, w, y, d_hidden=dh, d_weight=dw, piece_bytes=piece_bytes), dtype=torch.uint8, device="cuda")
    if ws_fill is not None:
        ws.fill_(ws_fill)
    B.hdet_token_scores_grad(hidden, w, y, ws, lse, logprob=None if y is None else logprob, entropy=entropy if "b" in use else None,
                             d_logprob=a if "a" in use else None, d_entropy=b if "b" in use else None, d_hidden=dh, d_weight=dw,
                             accumulate=accumulate, piece_bytes=piece_bytes, stream=stream)
    two_h, two_w = dh_dt == "f32", dw_dt == "f32"
    zero = torch.zeros_like(a)
    a, b = a if "a" in use else zero, b if "b" in use else zero
    for r in range(R):
        one = lambda t, dims: t if t is None or t.dim() == dims else t[r]  # noqa: E731
        ref = _reference(one(h, 2), one(w, 2), one(y, 1), a[r], b[r], two_h, two_w)
        if dh is not None:
            _within(dh[r], ref[0], ref[1], dh.dtype, "d_hidden", two_h)
        if dw is not None:
            want = ref[2] + start[r] if accumulate else ref[2]
            tol = ref[3] + (want.abs() * 2.0 ** -8 if accumulate and piece_bytes and not two_w else 0)      # rounded once more, at most
            _within(dw[r], want, tol, dw.dtype, "d_weight", two_w)
    for buf, view in bufs:                                # nothing beside the rows is written
        mask = torch.ones_like(buf, dtype=torch.bool)
        mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
        assert (buf[mask] == GUARD).all()
    return dh, dw


SHAPES = [      # R, T, V, D
    (1, 1, 64, 8), (1, 1, 1000, 64), (2, 2, 129, 33), (3, 7, 500, 40), (1, 48, 5000, 256), (3, 129, 4099, 520), (2, 200, 257, 130), (1, 300, 3000, 1100),
    (5, 257, 1, 24), (1, 1000, 20, 64), (4, 300, 8200, 64), (2, 600, 2048, 136),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dh,dw", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", None), (None, "bf16")])
@pytest.mark.parametrize("R,T,V,D", SHAPES)
def test_gradients(R, T, V, D, dh, dw):
    h, w, y = inputs(R, T, V, D, seed=R * 1000 + T + V)
    _run(h, w, y, dh, dw, ws_fill=0xFF)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("use", ["a", "b", "ab"])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_either_of_the_given_gradients(T, use, dt):
    h, w, y = inputs(2, T, 1030, 72, seed=T)
    _run(h, w, y, dt, dt, use=use)
    if use == "b":
        _run(h.nan_to_num(0.25), w, None, dt, dt, use=use)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_layouts_pieces_and_sums(dt):
    h, w, y = inputs(2, 270, 1500, 88, seed=4)
    _run(h, w, y, dt, dt, layout=(3, 5, 1))
    _run(h, w, y, dt, dt, layout=(8, 64, 8), accumulate=True)
    _run(h, w, y, dt, dt, piece_bytes=300_000)
    _run(h, w, y, dt, dt, piece_bytes=300_000, accumulate=True, layout=(1, 0, 0))
    _run(h, w[0].contiguous(), y, dt, dt)
    _run(h[0].nan_to_num(0.25), w, None, dt, dt, use="b")
    _, h2 = strided(h.shape, torch.bfloat16, 3, 1, 1, float("nan"))
    _, w2 = strided(w.shape, torch.bfloat16, 5, 1, 1, float("nan"))
    h2.copy_(h), w2.copy_(w)
    got, ref = _run(h2, w2, y.long(), dt, dt), _run(h, w, y, dt, dt)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    if dt == "bf16":
        got = _run(h, w, y, dt, dt, in_place=True)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 30, 300])
def test_padding_alone(T):
    h, w, _ = inputs(2, T, 333, 64, seed=1, pad=0.0)
    h[0] = float("nan")
    y = torch.stack([torch.full((T,), -1), torch.full((T,), 332)]).int().cuda()
    dh, dw = _run(h, w, y, "f32", "f32")
    assert (dh[0] == 0).all() and (dw[0] == 0).all()
    y[1] = 333
    h[1] = float("nan")
    dh, dw = _run(h, w, y, "bf16", "bf16")
    assert (dh == 0).all() and (dw == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("accumulate", [True, False])
def test_no_tokens(accumulate):
    h, w, y = inputs(2, 4, 100, 64, seed=1)
    h, y, none, stream = h[:, :0], y[:, :0], torch.empty((2, 0), device="cuda"), torch.cuda.current_stream().cuda_stream
    dw = torch.full(w.shape, GUARD, device="cuda")
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y, n_top=3), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores(h, w, y, ws, logprob=none, entropy=none, lse=none, top_ids=torch.empty((2, 0, 3), dtype=torch.int32, device="cuda"), stream=stream)
    ws = torch.empty(B.hdet_token_scores_grad_workspace(h, w, y, d_weight=dw), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores_grad(h, w, y, ws, none, logprob=none, d_logprob=none, d_weight=dw, accumulate=accumulate, stream=stream)
    assert (dw == (GUARD if accumulate else 0.0)).all()


@pytest.mark.gpu
def test_gradients_are_what_differences_say():
    """Central differences of the 64-bit value along random directions of the hidden states and of the table."""
    R, T, V, D = 1, 60, 900, 64
    h, w, y = inputs(R, T, V, D, seed=12, pad=0.0)
    dh, dw = _run(h, w, y, "f32", "f32", seed=5)
    a, b = _given(R, T, y, V, 5)

    def value(hd, wd):
        lp = torch.log_softmax(hd @ wd.t(), 1)
        return (a[0].double() * lp.gather(1, y[0].long()[:, None])[:, 0]).sum() - (b[0].double() * (lp.exp() * lp).sum(1)).sum()
    hd, wd = h[0].double(), w[0].double()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        u, v = torch.randn(hd.shape, generator=gen, device="cuda").double(), torch.randn(wd.shape, generator=gen, device="cuda").double()
        # the third derivative's part is (1e-4)^2 of values of the size of the sums of magnitudes; fp32 gradients are 2^-15 of their norm off
        for along, grad, got in ((u, dh[0], (value(hd + 1e-4 * u, wd) - value(hd - 1e-4 * u, wd)) / 2e-4),
                                 (v, dw[0], (value(hd, wd + 1e-5 * v) - value(hd, wd - 1e-5 * v)) / 2e-5)):
            size = float((grad.double().norm() * along.norm()))
            assert abs(float(got - (grad.double() * along).sum())) <= 2.0 ** -15 * size + 1e-6


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 260])
def test_what_is_not_finite_reaches_its_own_gradients(T):
    """A token whose normaliser is NaN has a gradient of NaN, and so has the table; the other tokens' gradients stay."""
    h, w, y = inputs(1, T, 500, 64, seed=3, pad=0.0)
    R, stream = 1, torch.cuda.current_stream().cuda_stream
    h[0, 0, 5] = float("nan")
    lse, entropy, logprob = (torch.empty((R, T), device="cuda") for _ in range(3))
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores(h, w, y, ws, logprob=logprob, entropy=entropy, lse=lse, stream=stream)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    ws = torch.empty(B.hdet_token_scores_grad_workspace(h, w, y, d_hidden=dh, d_weight=dw), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores_grad(h, w, y, ws, lse, logprob=logprob, entropy=entropy, d_logprob=torch.ones((R, T), device="cuda"), d_hidden=dh, d_weight=dw,
                             stream=stream)
    assert torch.isnan(dh[0, 0]).all() and torch.isnan(dw).all() and torch.isfinite(dh[0, 1:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_same_bits_captured_and_on_another_stream(dt):
    R, T, V, D = 2, 300, 2000, 64
    h, w, y = inputs(R, T, V, D, seed=8)
    ref = _run(h, w, y, dt, dt)
    stream = torch.cuda.current_stream().cuda_stream
    lse, entropy, logprob = (torch.empty((R, T), device="cuda") for _ in range(3))
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores(h, w, y, ws, logprob=logprob, entropy=entropy, lse=lse, stream=stream)
    a, b = _given(R, T, y, V, 0)
    dh, dw = torch.empty((R, T, D), dtype=DT[dt], device="cuda"), torch.empty((R, V, D), dtype=DT[dt], device="cuda")
    ws = torch.empty(B.hdet_token_scores_grad_workspace(h, w, y, d_hidden=dh, d_weight=dw), dtype=torch.uint8, device="cuda")

    def call():
        B.hdet_token_scores_grad(h, w, y, ws, lse, logprob=logprob, entropy=entropy, d_logprob=a, d_entropy=b, d_hidden=dh, d_weight=dw,
                                 stream=torch.cuda.current_stream().cuda_stream)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert torch.equal(dh, ref[0]) and torch.equal(dw, ref[1])
    with torch.cuda.graph(graph):
        call()
    dh.zero_(), dw.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dh, ref[0]) and torch.equal(dw, ref[1])
