"""Softmax cross entropy over the table and its gradients against 64-bit formulas, and the refusals of their arguments."""
import ctypes as C

import pytest
import torch

from paper_2604_24708_b200 import binding as B

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = 7.25


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def _args(**kw):
    a = B.hdet_token_loss_args(
        hidden=0x1000, weight=0x2000, targets=0x3000, loss=0x4000, token_loss=0x5000, d_hidden=0x6000, d_weight=0x7000,
        n_tokens=4, vocab=10, width=8, hidden_stride=32, hidden_row=8, weight_stride=80, weight_row=8, target_stride=4,
        token_loss_stride=4, d_hidden_stride=32, d_hidden_row=8, d_weight_stride=80, d_weight_row=8, grad_scale=1.0,
        n_replicas=2, hidden_dtype=B.HDET_DTYPE_BF16, weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32,
        loss_dtype=B.HDET_DTYPE_F32, d_hidden_dtype=B.HDET_DTYPE_BF16, d_weight_dtype=B.HDET_DTYPE_F32)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


ARG, ALIGN, UNSUP = B.HDET_ERR_INVALID_ARG, B.HDET_ERR_ALIGN, B.HDET_ERR_UNSUPPORTED
BAD = [
    (dict(n_replicas=0), ARG), (dict(n_replicas=33), ARG), (dict(n_tokens=-1), ARG), (dict(n_tokens=B.HDET_MAX_TOKENS + 1), ARG),
    (dict(vocab=0), ARG), (dict(vocab=B.HDET_MAX_VOCAB + 1), ARG), (dict(width=0), ARG), (dict(width=B.HDET_MAX_WIDTH + 1), ARG),
    (dict(target_dtype=B.HDET_DTYPE_F32), ARG), (dict(loss_dtype=B.HDET_DTYPE_BF16), ARG), (dict(hidden_dtype=B.HDET_DTYPE_F32), UNSUP),
    (dict(weight_dtype=B.HDET_DTYPE_F32), UNSUP), (dict(weight_dtype=B.HDET_DTYPE_I32), ARG), (dict(d_hidden_dtype=B.HDET_DTYPE_F64), ARG),
    (dict(d_weight_dtype=7), ARG), (dict(device=-1), ARG), (dict(grad_scale=float("nan")), ARG), (dict(grad_scale=float("inf")), ARG),
    (dict(piece_bytes=-1), ARG), (dict(hidden_row=7), ARG), (dict(weight_row=7), ARG), (dict(d_hidden_row=7), ARG), (dict(d_weight_row=7), ARG),
    (dict(hidden=None), ARG), (dict(weight=None), ARG), (dict(targets=None), ARG), (dict(loss=None), ARG),
    (dict(hidden_stride=31), ARG), (dict(weight_stride=79), ARG), (dict(target_stride=3), ARG), (dict(token_loss_stride=0), ARG),
    (dict(d_hidden_stride=0), ARG), (dict(d_weight_stride=0), ARG), (dict(d_weight_stride=-80), ARG),
    (dict(hidden=0x1001), ALIGN), (dict(weight=0x2001), ALIGN), (dict(targets=0x3002), ALIGN), (dict(loss=0x4004, loss_dtype=B.HDET_DTYPE_F64), ALIGN),
    (dict(token_loss=0x5002), ALIGN), (dict(d_hidden=0x6001), ALIGN), (dict(d_weight=0x7002), ALIGN),
]


@pytest.mark.parametrize("change,status", BAD, ids=[str(b[0]) for b in BAD])
def test_refusals(change, status):
    a, lib = _args(**change), B.raw_library()
    assert lib.hdet_token_loss(C.byref(a), 0x10000, 1 << 50, None) == status
    assert lib.hdet_last_error(None).startswith(b"hdet_token_loss: ")


def test_refusals_of_workspaces():
    lib, need = B.raw_library(), C.c_int64(0)
    assert lib.hdet_token_loss_workspace(C.byref(_args()), C.byref(need)) == B.HDET_OK and need.value >= 256
    assert lib.hdet_token_loss(C.byref(_args()), None, need.value, None) == ARG
    assert lib.hdet_token_loss(C.byref(_args()), 0x10000, need.value - 1, None) == ARG
    assert lib.hdet_token_loss(C.byref(_args()), 0x10010, need.value, None) == ALIGN
    assert lib.hdet_token_loss(None, 0x10000, need.value, None) == ARG
    assert lib.hdet_token_loss_workspace(C.byref(_args()), None) == ARG
    assert lib.hdet_token_loss_workspace(C.byref(_args(vocab=0)), C.byref(need)) == ARG


def test_workspace_follows_the_piece():
    lib = B.raw_library()

    def need(**kw):
        n = C.c_int64(0)
        a = _args(n_tokens=4096, vocab=50257, width=2048, n_replicas=1, hidden_row=2048, weight_row=2048, d_hidden_row=2048,
                  d_weight_row=2048, d_weight_dtype=B.HDET_DTYPE_BF16, **kw)
        assert lib.hdet_token_loss_workspace(C.byref(a), C.byref(n)) == B.HDET_OK
        return n.value
    whole, part, loss_only = need(piece_bytes=1 << 40), need(piece_bytes=64 << 20), need(d_hidden=None, d_weight=None)
    assert loss_only < part < whole
    assert whole - loss_only >= 4096 * 50257 * 2            # the whole softmax gradient
    assert part - loss_only <= (64 << 20) + 4 * 4 * 4096 * 2048 * 4


def test_the_struct_matches_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["token_loss", "n_tokens", "d_weight_row", "grad_scale", "piece_bytes", "hidden_dtype", "accumulate", "device"]
    (tmp_path / "t.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hdet.h"\nint main(void) {'
                                  'printf("%zu", sizeof(hdet_token_loss_args));'
                                  + "".join(f'printf(" %zu", offsetof(hdet_token_loss_args, {n}));' for n in names) + 'return 0; }')
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    got = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()
    A = B.hdet_token_loss_args
    assert [int(x) for x in got] == [C.sizeof(A)] + [getattr(A, n).offset for n in names]


def test_binding_refuses_wrong_shapes():
    h, w, y, l = torch.zeros(2, 3, 8).bfloat16(), torch.zeros(2, 5, 8).bfloat16(), torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2)
    ws = torch.zeros(1)
    for bad in [dict(), dict(hidden=h[..., :7]), dict(targets=y[:, :2]), dict(loss=torch.zeros(3)), dict(weight=w[..., ::2].repeat(1, 1, 2)[..., ::2])]:
        with pytest.raises(ValueError):                 # the first: not on a CUDA device
            B.hdet_token_loss(**{**dict(hidden=h, weight=w, targets=y, loss=l, workspace=ws), **bad})


# ------------------------------------------------------------------------------------------------ inputs and reference
def _strided(shape, dtype, pad_row, pad_rep, shift, fill):
    n, rows, width = shape
    row = width + pad_row
    rep = rows * row + pad_rep
    buf = torch.full((shift + n * rep + 16,), fill, dtype=dtype, device="cuda")
    return buf, buf.as_strided((n, rows, width), (rep, row, 1), shift)


def _inputs(R, T, V, D, seed, pad=0.2, target_dtype=torch.int32, lean=4.0):
    gen = torch.Generator().manual_seed(seed)
    w = (torch.randn((R, V, D), generator=gen) * 0.05).bfloat16()
    y = torch.randint(0, V, (R, T), generator=gen)
    h = torch.randn((R, T, D), generator=gen)
    for r in range(R):
        h[r] += torch.rand((T, 1), generator=gen) * lean * w[r][y[r]].float() / 0.05 / max(1.0, D ** 0.5)
    h = h.bfloat16()
    if pad and T > 1:
        at = torch.rand((R, T), generator=gen) < pad
        bad = torch.tensor([-100, -1, V, 2 ** 31 - 1])
        y = torch.where(at, bad[torch.randint(0, 4, (R, T), generator=gen)], y)
        h[at] = float("nan")            # what hidden states hold at padding reaches no output
    return h.cuda(), w.cuda(), y.to(target_dtype).cuda()


def _reference(h, w, y, grad_scale, hidden_two, weight_two):
    """64-bit values of one replica and, beside each, what it may be off by (see below), all on the GPU."""
    T, D = h.shape
    V = w.shape[0]
    keep = (y >= 0) & (y < V)
    t = keep.nonzero()[:, 0]
    yy = y[t].long()
    hd, wd = h[t].double(), w.double()
    n = len(t)
    z = hd @ wd.t()
    # fp32 sums of exact products: at most D additions, each off by at most a step (2^-23) of the sum of magnitudes
    ez = (hd.abs() @ wd.abs().t()) * D * 2.0 ** -23
    out = dict(loss=torch.zeros((), dtype=torch.float64, device="cuda"), token=torch.zeros(T, dtype=torch.float64, device="cuda"),
               dh=torch.zeros((T, D), dtype=torch.float64, device="cuda"), dw=torch.zeros((V, D), dtype=torch.float64, device="cuda"))
    tol = {k: torch.zeros_like(v) for k, v in out.items()}
    if n == 0:
        return out, tol
    lse = torch.logsumexp(z, 1)
    rows = torch.arange(n, device="cuda")
    each = lse - z[rows, yy]
    p = torch.exp(z - lse[:, None])
    # fp32 exponentials, logarithms and their arguments: a few steps of 1 + |z| + |lse|
    fp = (4 + z.abs() + lse.abs()[:, None]) * 2.0 ** -22
    e_lse = (p * ez).sum(1) + fp.amax(1)
    e_each = e_lse + ez[rows, yy] + fp.amax(1)
    g = p.clone()
    g[rows, yy] -= 1.0
    eg = p * (ez + e_lse[:, None] + fp) + 2.0 ** -23
    out["loss"], tol["loss"] = each.mean(), e_each.mean() + each.mean().abs() * 2.0 ** -24
    out["token"][t], tol["token"][t] = each, e_each
    c = grad_scale / n
    # G rounded to bf16 (half a step, 2^-8), or to a pair of them (2^-8 of 2^-8)
    egh = eg + g.abs() * (2.0 ** -16 if hidden_two else 2.0 ** -8)
    egw = eg + g.abs() * (2.0 ** -16 if weight_two else 2.0 ** -8)
    # fp32 sums over the vocabulary and over the tokens: as for z
    out["dh"][t] = c * (g @ wd)
    tol["dh"][t] = abs(c) * (egh @ wd.abs() + (g.abs() @ wd.abs()) * V * 2.0 ** -23)
    out["dw"] = c * (g.t() @ hd)
    tol["dw"] = abs(c) * (egw.t() @ hd.abs() + (g.abs().t() @ hd.abs()) * n * 2.0 ** -23)
    return out, tol


def _within(got, ref, tol, dtype, what):
    got = got.double()
    # the product with the scale (a step of fp32) and the output's rounding
    bound = tol + ref.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -22)
    far = (got - ref).abs() - bound
    assert torch.isfinite(got).all(), what
    assert (far <= 0).all(), f"{what}: {float(far.max()):.3e} over the bound"


def _close_in_norm(got, ref, dtype, what, two):
    """The bounds above are worst cases; errors that are independent add up to far less.  fp32: sums of 2^-24 steps and pairs
    of 2^-17 stay below 2^-16 together; bf16: two roundings of 2^-8 at most, as G and as output."""
    norm = float(ref.norm())
    if norm > 0:
        assert float((got.double() - ref).norm()) <= norm * (2.0 ** -16 if two else 2.0 ** -7), what


def _run(h, w, y, dh_dt=None, dw_dt=None, layout=(0, 0, 0), grad_scale=1.0, accumulate=False, piece_bytes=0, loss_dtype=torch.float32,
         token=True, ws_fill=None):
    """Runs the operator with outputs inside guarded buffers and compares everything with 64 bits."""
    R = max(h.shape[0] if h.dim() == 3 else 1, w.shape[0] if w.dim() == 3 else 1, y.shape[0] if y.dim() == 2 else 1)
    T, D, V = h.shape[-2], h.shape[-1], w.shape[-2]
    pad_row, pad_rep, shift = layout
    loss = torch.full((R,), GUARD, dtype=loss_dtype, device="cuda")
    tbuf, tl = _strided((R, 1, T), torch.float32, 0, pad_rep, 0, GUARD)
    tl = tl[:, 0]
    dh = dw = start = None
    if dh_dt:
        hbuf, dh = _strided((R, T, D), DT[dh_dt], pad_row, pad_rep, shift, GUARD)
        dh.fill_(float("nan"))
    if dw_dt:
        wbuf, dw = _strided((R, V, D), DT[dw_dt], pad_row, pad_rep, shift, GUARD)
        gen = torch.Generator().manual_seed(3)
        dw.copy_(torch.randn(dw.shape, generator=gen) * 1e-2 if accumulate else torch.full((1,), float("nan")))
        start = dw.double() if accumulate else None
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=dh, d_weight=dw, piece_bytes=piece_bytes), dtype=torch.uint8, device="cuda")
    if ws_fill is not None:
        ws.fill_(ws_fill)
    B.hdet_token_loss(h, w, y, loss, ws, token_loss=tl if token else None, d_hidden=dh, d_weight=dw, grad_scale=grad_scale,
                      accumulate=accumulate, piece_bytes=piece_bytes, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for r in range(R):
        ref, tol = _reference(h if h.dim() == 2 else h[r], w if w.dim() == 2 else w[r], y if y.dim() == 1 else y[r], grad_scale,
                              dh_dt == "f32", dw_dt == "f32")
        _within(loss[r], ref["loss"], tol["loss"], loss_dtype, "loss")
        if token:
            _within(tl[r], ref["token"], tol["token"], torch.float32, "token_loss")
        if dh_dt:
            _within(dh[r], ref["dh"], tol["dh"], DT[dh_dt], "d_hidden")
            _close_in_norm(dh[r], ref["dh"], DT[dh_dt], "d_hidden", dh_dt == "f32")
        if dw_dt:
            if accumulate:
                tol["dw"] += ref["dw"].abs() * 2.0 ** -22
                ref["dw"] = ref["dw"] + start[r]
            _within(dw[r], ref["dw"], tol["dw"], DT[dw_dt], "d_weight")
            _close_in_norm(dw[r], ref["dw"], DT[dw_dt], "d_weight", dw_dt == "f32")
    copies = (loss, tl.clone(), None if dh is None else dh.clone(), None if dw is None else dw.clone())
    for buf, view in [(tbuf, tl)] + ([(hbuf, dh)] if dh_dt else []) + ([(wbuf, dw)] if dw_dt else []):
        view.fill_(GUARD)
        assert (buf == GUARD).all(), "written outside its place"
    return copies


# ------------------------------------------------------------------------------------------------ values
# one CTA a tile (up to 128 tokens), then pairs; sizes on both sides of the tiles'; widths that cannot be copied in boxes
SMALL = [(1, 1, 1, 1), (1, 1, 300, 64), (2, 5, 257, 72), (1, 128, 1000, 128), (3, 100, 130, 33), (1, 127, 129, 136)]
PAIRS = [(1, 129, 255, 64), (2, 300, 513, 200), (1, 256, 256, 256), (1, 512, 5000, 768), (2, 257, 1025, 129)]


@pytest.mark.gpu
@pytest.mark.parametrize("size", SMALL + PAIRS, ids=str)
def test_loss(size):
    R, T, V, D = size
    _run(*_inputs(R, T, V, D, seed=T + V))
    _run(*_inputs(R, T, V, D, seed=T + V + 1, target_dtype=torch.int64, pad=0.0), loss_dtype=torch.float64, token=False)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("V,D", [(1, 8), (33, 64), (5000, 776), (50257, 264)])
def test_loss_of_few_tokens(T, V, D):
    for R, shared, pad in [(1, False, 0.0), (3, False, 0.5), (2, True, 0.5)]:
        h, w, y = _inputs(R, T, V, D, seed=T + V, pad=pad, target_dtype=torch.int64 if shared else torch.int32)
        if T == 3:
            y[0] = -100
        _run(h, w[0] if shared else w, y)
        _, hs = _strided((R, T, D), torch.bfloat16, 8, 8, 8, float("nan"))
        hs.copy_(h)
        _run(hs, w[0] if shared else w, y, token=False, loss_dtype=torch.float64, ws_fill=255)


@pytest.mark.gpu
@pytest.mark.parametrize("dh_dt,dw_dt", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", None), (None, "bf16"),
                                         ("f32", None), (None, "f32")])
@pytest.mark.parametrize("size", SMALL + PAIRS, ids=str)
def test_gradients(size, dh_dt, dw_dt):
    R, T, V, D = size
    _run(*_inputs(R, T, V, D, seed=T + V), dh_dt, dw_dt, grad_scale=1.0 if dh_dt == dw_dt else 64.0)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [(8, 0, 0), (0, 8, 8), (4, 0, 0), (1, 3, 1)], ids=str)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_strides_and_accumulation(layout, dt):
    pad_row, pad_rep, shift = layout
    for R, T, V, D in [(2, 90, 140, 72), (2, 200, 300, 72)]:
        h, w, y = _inputs(R, T, V, D, seed=9)
        _, hs = _strided((R, T, D), torch.bfloat16, pad_row, pad_rep, shift, float("nan"))
        _, wst = _strided((R, V, D), torch.bfloat16, pad_row, pad_rep, shift, float("nan"))
        hs.copy_(h)
        wst.copy_(w)
        _run(hs, wst, y, dt, dt, layout=layout, accumulate=True, grad_scale=0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size,piece", [((2, 100, 1000, 136), 1), ((2, 100, 1000, 136), 100000), ((3, 300, 2000, 264), 1),
                                        ((3, 300, 2000, 264), 512 * 700 * 2), ((5, 300, 600, 64), 512 * 768 * 2 * 2 * 2)], ids=str)
def test_pieces_of_the_vocabulary(size, piece, dt):
    _run(*_inputs(*size, seed=12), dt, dt, piece_bytes=piece, ws_fill=255)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(1, 20, 150, 4168), (2, 150, 300, 4200), (1, 70000, 130, 40), (1, 9000, 20000, 64)], ids=str)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_long_sums(size, dt):
    """Sums over the width, the tokens or the vocabulary that leave the tensor cores in several chunks."""
    _run(*_inputs(*size, seed=13), dt, dt)


@pytest.mark.gpu
def test_one_table_one_batch_for_all_replicas():
    for T in (60, 260):
        h, w, y = _inputs(3, T, 500, 96, seed=20)
        _run(h, w[0], y, "bf16", "bf16")
        _run(h, w[0], y, "f32", "f32")
        y0, h0 = y[0], h[0]
        out = _run(h0, w, y0, "bf16", "bf16")
        assert len(out[0]) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 70, 300])
def test_as_many_replicas_as_there_can_be(T):
    h, w, y = _inputs(B.HDET_MAX_REPLICAS, T, 90, 72, seed=25)
    y[5] = -1
    _run(h, w, y)
    _run(h, w, y, "bf16", "bf16")
    _run(h, w, y, "f32", "f32", piece_bytes=1)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [70, 300])
def test_the_gradient_in_the_place_of_the_hidden_states(T):
    h, w, y = _inputs(2, T, 500, 96, seed=26)
    loss, apart = torch.empty(2, device="cuda"), torch.empty_like(h)
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=apart), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    B.hdet_token_loss(h, w, y, loss, ws, d_hidden=apart, stream=st)
    B.hdet_token_loss(h, w, y, loss, ws, d_hidden=h, stream=st)
    assert torch.equal(h, apart)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 400])
def test_replicas_without_a_target_and_no_tokens(T):
    h, w, y = _inputs(3, T, 200, 64, seed=21)
    y[1] = -100
    h[1] = float("nan")
    loss, tl, dh, dw = _run(h, w, y, "bf16", "f32")
    assert float(loss[1]) == 0 and not tl[1].any() and not dh[1].any() and not dw[1].any()
    empty = torch.empty((3, 0), dtype=torch.int32, device="cuda")
    loss, _, _, dw = _run(torch.empty((3, 0, 64), dtype=torch.bfloat16, device="cuda"), w, empty, "bf16", "f32")
    assert not loss.any() and not dw.any()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [30, 300])
def test_large_and_infinite_logits(T):
    """Logits far above what exp holds; classes with logit -inf (probability 0); a NaN token makes its replica's loss NaN."""
    h, w, y = _inputs(2, T, 300, 64, seed=22, pad=0.0)
    _run((h * 64).bfloat16(), w, y, "bf16", "bf16")
    h = h.abs()
    w[0, 7] = float("-inf")                          # every logit of class 7 is -inf
    y[y == 7] = 8
    loss = torch.empty(2, device="cuda")
    tl = torch.empty((2, T), device="cuda")
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    B.hdet_token_loss(h, w, y, loss, ws, token_loss=tl, stream=st)
    z = h[0].double() @ w[0].double().nan_to_num(neginf=0.0).t()
    z[:, 7] = float("-inf")
    want = torch.logsumexp(z, 1) - z[torch.arange(T), y[0].long()]
    assert ((tl[0].double() - want).abs() <= 1e-4 * (1 + want.abs())).all()     # 64 x 2^-23 of sums of some tens, and fp32 steps
    h[1, 3] = float("nan")
    B.hdet_token_loss(h, w, y, loss, ws, token_loss=tl, stream=st)
    assert torch.isfinite(loss[0]) and torch.isnan(loss[1]) and torch.isnan(tl[1, 3]) and torch.isfinite(tl[1, 4:]).all()


# ------------------------------------------------------------------------------------------------ behaviour
@pytest.mark.gpu
@pytest.mark.parametrize("size", [(2, 100, 700, 80), (2, 300, 3000, 200)], ids=str)
def test_the_same_bits_whatever_the_workspace_held(size):
    h, w, y = _inputs(*size, seed=30)
    first = _run(h, w, y, "bf16", "f32", ws_fill=0)
    for fill in (255, 127):
        again = _run(h, w, y, "bf16", "f32", ws_fill=fill)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.gpu
def test_gradients_agree_with_differences_of_the_loss():
    """Central differences of the operator's own loss.  Third derivatives of the loss along one coordinate are at most the
    third central moment of that coordinate of the table, below (2 max|w|)^3; the loss itself is off by a few 1e-6."""
    R, T, V, D = 1, 3, 40, 64
    h, w, y = _inputs(R, T, V, D, seed=31, pad=0.0)
    dh, dw = torch.empty((R, T, D), device="cuda"), torch.empty((R, V, D), device="cuda")
    loss = torch.empty(1, dtype=torch.float64, device="cuda")
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=dh, d_weight=dw), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    B.hdet_token_loss(h, w, y, loss, ws, d_hidden=dh, d_weight=dw, stream=st)

    def at(h, w):
        B.hdet_token_loss(h, w, y, loss, ws, stream=st)
        return float(loss)
    for t, c in [(0, 0), (1, 17), (2, 63)]:
        up, down = h.clone(), h.clone()
        up[0, t, c] += 0.25
        down[0, t, c] -= 0.25
        step = float(up[0, t, c]) - float(down[0, t, c])
        bound = (step / 2) ** 2 / 6 * (2 * float(w.abs().max())) ** 3 / T + 2 * 4e-6 / step
        assert abs((at(up, w) - at(down, w)) / step - float(dh[0, t, c])) <= bound
    for v, c in [(int(y[0, 0]), 5), (3, 40)]:
        up, down = w.clone(), w.clone()
        up[0, v, c] += 2.0 ** -4
        down[0, v, c] -= 2.0 ** -4
        step = float(up[0, v, c]) - float(down[0, v, c])
        bound = (step / 2) ** 2 / 6 * (2 * float(h.float().abs().max())) ** 3 + 2 * 4e-6 / step
        assert abs((at(h, up) - at(h, down)) / step - float(dw[0, v, c])) <= bound


@pytest.mark.gpu
@pytest.mark.parametrize("T", [70, 270])
def test_captured_and_replayed_on_another_stream(T):
    h, w, y = _inputs(2, T, 600, 128, seed=40)
    loss, tl = torch.empty(2, device="cuda"), torch.empty((2, T), device="cuda")
    dh, dw = torch.empty((2, T, 128), device="cuda"), torch.empty((2, 600, 128), device="cuda").bfloat16()
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=dh, d_weight=dw), dtype=torch.uint8, device="cuda")

    def call():
        B.hdet_token_loss(h, w, y, loss, ws, token_loss=tl, d_hidden=dh, d_weight=dw, stream=torch.cuda.current_stream().cuda_stream)
    call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    h2, w2, y2 = _inputs(2, T, 600, 128, seed=41)
    h.copy_(h2), w.copy_(w2), y.copy_(y2)
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in (loss, tl, dh, dw)]
    call()
    assert all(torch.equal(a, b) for a, b in zip(replayed, (loss, tl, dh, dw)))


@pytest.mark.gpu
def test_two_calls_at_once_with_their_own_workspaces():
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets, alone = [], []
    for k in range(2):
        h, w, y = _inputs(2, 300, 2000, 256, seed=50 + k)
        out = dict(loss=torch.empty(2, device="cuda"), d_hidden=torch.empty((2, 300, 256), device="cuda").bfloat16(),
                   d_weight=torch.empty((2, 2000, 256), device="cuda").bfloat16())
        ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=out["d_hidden"], d_weight=out["d_weight"]), dtype=torch.uint8, device="cuda")
        sets.append((h, w, y, out, ws))
        B.hdet_token_loss(h, w, y, workspace=ws, stream=torch.cuda.current_stream().cuda_stream, **out)
        torch.cuda.synchronize()
        alone.append({n: t.clone() for n, t in out.items()})
    for _ in range(5):
        for st, (h, w, y, out, ws) in zip(streams, sets):
            B.hdet_token_loss(h, w, y, workspace=ws, stream=st.cuda_stream, **out)
    torch.cuda.synchronize()
    for (_, _, _, out, _), want in zip(sets, alone):
        assert all(torch.equal(out[n], want[n]) for n in want)


@pytest.mark.gpu
def test_tables_behind_2_to_the_31_elements():
    """24 replicas of a 50257 x 2048 table: the last replica's values equal those of a call of its own."""
    R, T, V, D = 24, 2, 50257, 2048
    w = torch.empty((R, V, D), dtype=torch.bfloat16, device="cuda")
    for r in range(R):
        w[r].normal_(0, 0.02)
    h = torch.randn((R, T, D), device="cuda").bfloat16()
    y = torch.randint(0, V, (R, T), device="cuda", dtype=torch.int32)
    y[:, 0] = V - 1
    st = torch.cuda.current_stream().cuda_stream
    dw, dh, loss = torch.empty_like(w), torch.empty_like(h), torch.empty(R, device="cuda")
    ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=dh, d_weight=dw), dtype=torch.uint8, device="cuda")
    B.hdet_token_loss(h, w, y, loss, ws, d_hidden=dh, d_weight=dw, stream=st)
    one = torch.empty((1, V, D), device="cuda").bfloat16(), torch.empty((1, T, D), device="cuda").bfloat16(), torch.empty(1, device="cuda")
    for r in (0, R - 1):
        B.hdet_token_loss(h[r:r + 1], w[r:r + 1], y[r:r + 1], one[2], ws, d_hidden=one[1], d_weight=one[0], stream=st)
        ref, tol = _reference(h[r], w[r], y[r], 1.0, False, False)
        _within(loss[r], ref["loss"], tol["loss"], torch.float32, "loss")
        _within(dw[r], ref["dw"], tol["dw"], torch.bfloat16, "d_weight")
        _within(dh[r], ref["dh"], tol["dh"], torch.bfloat16, "d_hidden")
        assert float((one[0][0].double() - ref["dw"]).norm()) <= 2.0 ** -7 * float(ref["dw"].norm())
