"""Log probabilities, entropies and best alternatives against 64-bit formulas, and the refusals of their arguments."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2604_24708_b200 import binding as B

GUARD = 7.25


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def _args(**kw):
    a = B.hdet_token_scores_args(
        hidden=0x1000, weight=0x2000, targets=0x3000, logprob=0x4000, entropy=0x5000, lse=0x6000, top_ids=0x7000, top_logprob=0x8000,
        n_tokens=4, vocab=10, width=8, hidden_stride=32, hidden_row=8, weight_stride=80, weight_row=8, target_stride=4, logprob_stride=4,
        entropy_stride=4, lse_stride=4, top_ids_stride=12, top_logprob_stride=12, n_replicas=2, n_top=3, hidden_dtype=B.HDET_DTYPE_BF16,
        weight_dtype=B.HDET_DTYPE_BF16, target_dtype=B.HDET_DTYPE_I32)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


ARG, ALIGN, UNSUP = B.HDET_ERR_INVALID_ARG, B.HDET_ERR_ALIGN, B.HDET_ERR_UNSUPPORTED
BAD = [
    (dict(n_replicas=0), ARG), (dict(n_replicas=33), ARG), (dict(n_tokens=-1), ARG), (dict(n_tokens=B.HDET_MAX_TOKENS + 1), ARG),
    (dict(vocab=0), ARG), (dict(vocab=B.HDET_MAX_VOCAB + 1), ARG), (dict(width=0), ARG), (dict(width=B.HDET_MAX_WIDTH + 1), ARG),
    (dict(n_top=-1), ARG), (dict(n_top=B.HDET_MAX_TOP + 1, vocab=100), ARG), (dict(n_top=11), ARG), (dict(n_top=0), ARG), (dict(top_ids=None), ARG),
    (dict(n_top=0, top_ids=None), ARG), (dict(targets=None), ARG), (dict(n_top=0, top_ids=None, top_logprob=None, logprob=None, entropy=None, lse=None), ARG),
    (dict(target_dtype=B.HDET_DTYPE_F32), ARG), (dict(hidden_dtype=B.HDET_DTYPE_F32), UNSUP), (dict(weight_dtype=B.HDET_DTYPE_F32), UNSUP),
    (dict(weight_dtype=B.HDET_DTYPE_I32), ARG), (dict(device=-1), ARG), (dict(hidden_row=7), ARG), (dict(weight_row=7), ARG),
    (dict(hidden_row=B.HDET_MAX_ROW_STRIDE + 1), ARG), (dict(weight_stride=B.HDET_MAX_REPLICA_STRIDE + 1), ARG), (dict(hidden=None), ARG), (dict(weight=None), ARG),
    (dict(hidden_stride=31), ARG), (dict(weight_stride=79), ARG), (dict(target_stride=3), ARG), (dict(logprob_stride=3), ARG), (dict(entropy_stride=0), ARG),
    (dict(lse_stride=-4), ARG), (dict(top_ids_stride=11), ARG), (dict(top_logprob_stride=0), ARG),
    (dict(hidden=0x1001), ALIGN), (dict(weight=0x2001), ALIGN), (dict(targets=0x3002), ALIGN), (dict(targets=0x3004, target_dtype=B.HDET_DTYPE_I64), ALIGN),
    (dict(logprob=0x4002), ALIGN), (dict(entropy=0x5001), ALIGN), (dict(lse=0x6002), ALIGN), (dict(top_ids=0x7002), ALIGN), (dict(top_logprob=0x8002), ALIGN),
]


@pytest.mark.parametrize("change,status", BAD, ids=[str(b[0]) for b in BAD])
def test_refusals(change, status):
    a, lib = _args(**change), B.raw_library()
    assert lib.hdet_token_scores(C.byref(a), 0x10000, 1 << 50, None) == status
    assert lib.hdet_last_error(None).startswith(b"hdet_token_scores: ")


def test_refusals_of_workspaces():
    lib, need, none = B.raw_library(), C.c_int64(0), C.c_int64(1)
    assert lib.hdet_token_scores_workspace(C.byref(_args()), C.byref(need)) == B.HDET_OK and need.value >= 256
    assert lib.hdet_token_scores(C.byref(_args()), None, need.value, None) == ARG
    assert lib.hdet_token_scores(C.byref(_args()), 0x10000, 255, None) == ARG
    assert lib.hdet_token_scores(C.byref(_args()), 0x10010, need.value, None) == ALIGN
    assert lib.hdet_token_scores(None, 0x10000, need.value, None) == ARG
    assert lib.hdet_token_scores_workspace(C.byref(_args()), None) == ARG
    assert lib.hdet_token_scores_workspace(C.byref(_args(vocab=0)), C.byref(none)) == ARG and none.value == 0
    assert lib.hdet_selftest_token_scores_wait(C.byref(_args(n_tokens=1, n_replicas=1)), 0x10000, 1 << 50, None) == UNSUP
    assert lib.hdet_token_scores(C.byref(_args(n_tokens=0)), 0x10000, need.value, None) == B.HDET_OK       # nothing to do


def test_workspaces_are_enough_for_fewer_tokens():
    lib, need, less = B.raw_library(), C.c_int64(0), C.c_int64(0)
    for kw in (dict(vocab=50257), dict(vocab=300, n_top=1), dict(n_replicas=7, vocab=4099, weight_stride=4099 * 8, hidden_stride=1 << 20)):
        kw = {**dict(n_replicas=1), **kw}
        assert lib.hdet_token_scores_workspace(C.byref(_args(n_tokens=3000, **kw)), C.byref(need)) == B.HDET_OK
        for t in (0, 1, 2, 3, 100, 192, 193, 256, 1000, 2999):
            assert lib.hdet_token_scores_workspace(C.byref(_args(n_tokens=t, **kw)), C.byref(less)) == B.HDET_OK
            assert less.value <= need.value


def test_the_struct_matches_the_header(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    A = B.hdet_token_scores_args
    names = [f[0] for f in A._fields_]
    (tmp_path / "t.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hdet.h"\nint main(void) {'
                                  'printf("%zu %d", sizeof(hdet_token_scores_args), HDET_MAX_TOP);'
                                  + "".join(f'printf(" %zu", offsetof(hdet_token_scores_args, {n}));' for n in names) + 'return 0; }')
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    got = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [C.sizeof(A), B.HDET_MAX_TOP] + [getattr(A, n).offset for n in names]


def test_binding_refuses_wrong_shapes():
    h, w, y = torch.zeros(2, 3, 8).bfloat16(), torch.zeros(2, 5, 8).bfloat16(), torch.zeros((2, 3), dtype=torch.int32)
    ws, e = torch.zeros(1), torch.zeros(2, 3)
    for bad in [dict(), dict(hidden=h[..., :7]), dict(targets=y[:, :2]), dict(weight=w[..., ::2].repeat(1, 1, 2)[..., ::2])]:
        with pytest.raises(ValueError):                 # the first: not on a CUDA device
            B.hdet_token_scores(**{**dict(hidden=h, weight=w, targets=y, workspace=ws, entropy=e), **bad})


# ------------------------------------------------------------------------------------------------ inputs and reference
def strided(shape, dtype, pad_row, pad_rep, shift, fill):
    n, rows, width = shape
    row = width + pad_row
    rep = rows * row + pad_rep
    buf = torch.full((shift + n * rep + 16,), fill, dtype=dtype, device="cuda")
    return buf, buf.as_strided((n, rows, width), (rep, row, 1), shift)


def inputs(R, T, V, D, seed, pad=0.2, target_dtype=torch.int32, lean=4.0):
    """Hidden states that lean towards their token's row; what they hold at padding is NaN."""
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
        h[at] = float("nan")
    return h.cuda(), w.cuda(), y.to(target_dtype).cuda()


def reference(h, w, y, n_top):
    """64-bit values of one replica (y None: every token counts) and, beside each, what it may be off by."""
    T, D = h.shape
    V = w.shape[0]
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if y is None else (y >= 0) & (y < V)
    t = keep.nonzero()[:, 0]
    hd, wd = h[t].double(), w.double()
    z = hd @ wd.t()
    ez = (hd.abs() @ wd.abs().t()) * D * 2.0 ** -23       # fp32 sums: at most D additions, each off by at most a step of the sum of magnitudes
    out = {k: torch.zeros(T, dtype=torch.float64, device="cuda") for k in ("lse", "entropy", "logprob")}
    tol = {k: torch.zeros_like(v) for k, v in out.items()}
    ids = torch.full((T, n_top), -1, dtype=torch.int32, device="cuda")
    top, e_top = torch.zeros((T, n_top), dtype=torch.float64, device="cuda"), torch.zeros((T, n_top), dtype=torch.float64, device="cuda")
    if len(t) == 0:
        return out, tol, ids, top, e_top
    lse = torch.logsumexp(z, 1, keepdim=True)
    lp = z - lse
    p = lp.exp()
    entropy = -(p * lp).sum(1)
    d = (z.amax(1, keepdim=True) - z)
    # an exponential is off by 2^-22 of its value and by the rounding of its argument; sums by their additions: 16 within 64 columns, one
    # for every 64, and those of the parts
    adds = 16 + V / 64 + 60
    rel = (4 + d) * 2.0 ** -22 + adds * 2.0 ** -24
    out["lse"][t], tol["lse"][t] = lse[:, 0], (p * (ez + rel)).sum(1) + lse[:, 0].abs() * 2.0 ** -23
    out["entropy"][t] = entropy
    tol["entropy"][t] = (p * ((lp + entropy[:, None]).abs() * ez + (d + 1) * rel)).sum(1) + 3 * ez.amax(1) ** 2 + entropy * 2.0 ** -22
    e_lp = ez + (p * (ez + rel)).sum(1, keepdim=True) + lp.abs() * 2.0 ** -22
    if y is not None:
        at = y[t].long()[:, None]
        out["logprob"][t], tol["logprob"][t] = lp.gather(1, at)[:, 0], e_lp.gather(1, at)[:, 0]
    if n_top:
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :n_top]
        ids[t], top[t], e_top[t] = order.int(), lp.gather(1, order), e_lp.gather(1, order)
    return out, tol, ids, top, e_top


def within(got, ref, tol, what):
    assert torch.isfinite(got).all(), what
    far = (got.double() - ref).abs() - (tol + ref.abs() * 2.0 ** -24)
    assert (far <= 0).all(), f"{what}: {float(far.max()):.3e} over the bound"
    # The bounds are worst cases: a logit is cut once for every 16 products, not for each, and by half a step on average.
    assert float((got.double() - ref).norm()) <= 2.0 ** -16 * float(ref.norm()) + float(tol.norm()) * 2.0 ** -5, what


def run(h, w, y, n_top=0, want=("logprob", "entropy", "lse"), top_logprob=True, rep_pad=0, ws_fill=None, check=True):
    """Runs the operator with outputs inside guarded buffers, twice, and compares everything with 64 bits."""
    R = max(h.shape[0] if h.dim() == 3 else 1, w.shape[0] if w.dim() == 3 else 1, y.shape[0] if y is not None and y.dim() == 2 else 1)
    T, V = h.shape[-2], w.shape[-2]
    bufs, out = {}, {}
    for k in want:
        if k == "logprob" and y is None:
            continue
        bufs[k], v = strided((R, 1, T), torch.float32, 0, rep_pad, 0, GUARD)
        out[k] = v[:, 0]
    if n_top:
        for k, dt in (("top_ids", torch.int32),) + ((("top_logprob", torch.float32),) if top_logprob else ()):
            bufs[k], v = strided((R, 1, T * n_top), dt, 0, rep_pad, 0, int(GUARD) if dt == torch.int32 else GUARD)
            out[k] = v[:, 0].unflatten(1, (T, n_top))
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y, n_top=n_top), dtype=torch.uint8, device="cuda")
    if ws_fill is not None:
        ws.fill_(ws_fill)
    call = lambda: B.hdet_token_scores(h, w, y, ws, stream=torch.cuda.current_stream().cuda_stream, **out)  # noqa: E731
    call()
    first = {k: v.clone() for k, v in bufs.items()}
    call()
    for k, v in bufs.items():
        assert torch.equal(first[k].view(torch.int32), v.view(torch.int32)), k          # the same bits (NaN too)
        rep = T * (n_top if k.startswith("top") else 1) + rep_pad
        rest = v[: R * rep].view(R, rep)[:, rep - rep_pad:] if rep_pad else v[R * rep:]
        assert (rest == int(GUARD) if v.dtype == torch.int32 else rest == GUARD).all(), k
    if not check:
        return out
    for r in range(R):
        one = lambda t, dims: t if t is None or t.dim() == dims else t[r]  # noqa: E731
        ref, tol, ids, top, e_top = reference(one(h, 2), one(w, 2), one(y, 1), n_top)
        for k in out:
            if k == "top_ids":
                assert torch.equal(out[k][r], ids), (k, r)
            elif k == "top_logprob":
                within(out[k][r], top, e_top, k)
            else:
                within(out[k][r], ref[k], tol[k], k)
    return out


# ------------------------------------------------------------------------------------------------ values
SHAPES = [      # R, T, V, D, n_top
    (1, 1, 50257, 768, 20), (1, 1, 64, 8, 5), (1, 1, 1, 16, 1), (3, 1, 1000, 64, 8), (2, 2, 4099, 96, 20), (32, 1, 777, 64, 3), (1, 2, 50257, 64, 1),
    (1, 1, 1000, 63, 7), (1, 3, 500, 40, 4), (2, 5, 129, 33, 20), (1, 48, 5000, 256, 8), (1, 128, 2000, 64, 20), (1, 129, 999, 72, 5), (3, 150, 257, 130, 2),
    (2, 200, 4099, 520, 6), (1, 192, 300, 1, 20), (1, 193, 300, 2, 20), (1, 1000, 20, 64, 20), (5, 257, 1, 24, 1), (4, 300, 8200, 64, 16), (16, 256, 1030, 136, 3),
    (1, 300, 3000, 1025, 4), (2, 130, 600, 2048, 20), (1, 20, 700, 1100, 9), (8, 513, 4099, 64, 0), (1, 1, 3000, 64, 0), (1, 700, 65, 640, 0), (1, 2500, 16411, 128, 12),
    # too many logits to be kept: lists of 16 and of 32, pairs of CTAs and single ones, sums in several chunks, short vocabularies
    (1, 1400, 50257, 64, 8), (1, 1400, 50257, 72, 20), (4, 400, 50257, 1100, 6), (32, 64, 50257, 32, 12), (3, 190, 130000, 40, 13), (1, 120000, 600, 16, 12),
    (2, 60000, 700, 8, 20),
]


@pytest.mark.gpu
@pytest.mark.parametrize("R,T,V,D,n_top", SHAPES)
def test_values(R, T, V, D, n_top):
    h, w, y = inputs(R, T, V, D, seed=R * 1000 + T)
    run(h, w, y, n_top, rep_pad=5, ws_fill=0xFF)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 7, 300])
def test_every_token_counts_without_targets(T):
    h, w, _ = inputs(2, T, 1001, 64, seed=T, pad=0.0)
    run(h, w, None, 5)
    run(h, w, None, 0, want=("entropy",))
    run(h, w, None, 20, want=(), top_logprob=False)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 9, 260])
def test_one_table_one_batch_and_wide_ids(T):
    h, w, y = inputs(3, T, 700, 64, seed=T, target_dtype=torch.int64)
    run(h, w[1].contiguous(), y, 4)                      # one table for all
    run(h, w, y[0], 4) if T == 1 else run(h.nan_to_num(0.5), w, y[0].contiguous(), 4)      # one list of targets for all
    run(h[0].nan_to_num(0.5), w, y, 4)                   # one batch for all
    run(h[0].nan_to_num(0.5), w[0], y[0], 4)             # no replica axis


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 40, 300])
@pytest.mark.parametrize("pad_row,pad_rep,shift", [(8, 64, 8), (1, 3, 1), (4, 4, 4), (2, 6, 0)])
def test_layouts(T, pad_row, pad_rep, shift):
    h0, w0, y = inputs(2, T, 515, 88, seed=5)
    _, h = strided(h0.shape, torch.bfloat16, pad_row, pad_rep, shift, float("nan"))
    _, w = strided(w0.shape, torch.bfloat16, pad_row, pad_rep, shift, float("nan"))
    h.copy_(h0), w.copy_(w0)
    a, b = run(h, w, y, 6), run(h0, w0, y, 6)
    assert torch.equal(a["top_ids"], b["top_ids"])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 30, 400])
def test_padding(T):
    """All of it, none of it, and the last tokens; ids at the ends of the table."""
    h, w, _ = inputs(2, T, 333, 64, seed=1, pad=0.0)
    for y in (torch.full((2, T), -1), torch.full((2, T), 332), torch.zeros((2, T)), torch.where(torch.arange(T) < T // 2, 332, 333).expand(2, T)):
        run(h, w, y.int().cuda().contiguous(), 3)


SIZES = [(1, 5000), (2, 5000), (30, 5000), (400, 5000), (1400, 50257), (100, 700_000)]      # the last two: too many logits to be kept


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("n_top", [3, 20])
def test_equal_logits_go_by_their_ids(T, V, n_top):
    """Rows of the table that are the same, more of them than a list holds, near and far apart; and a hidden state of zeros."""
    gen = torch.Generator().manual_seed(3)
    h, w, _ = inputs(1, T, V, 72, seed=2, pad=0.0)
    for count in (2, 7, 40, 600):
        at = torch.randperm(V, generator=gen)[:count]
        w2 = w.clone()
        w2[0, at] = w[0, int(at[0])] * 4
        run(h, w2, None, n_top)
    run(h, w[:, :1].expand(1, V, 72).contiguous(), None, n_top)
    run(torch.zeros_like(h), w, None, n_top)
    steps = (torch.arange(V, device="cuda") // (V // 135)).float().bfloat16()        # falling and rising plateaus
    for s in (steps, -steps):
        w2 = torch.zeros_like(w)
        w2[0, :, 0] = s
        run(h.abs(), w2, None, n_top)


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", [(1, 20000), (2, 20000), (30, 20000), (400, 20000), (1400, 50257), (100, 700_000)])
@pytest.mark.parametrize("n_top", [12, 20])
def test_logits_that_fall_and_rise_along_the_table(T, V, n_top):
    """A table in falling order fills the lists at once; one in rising order replaces every entry of them, again and again."""
    h, w, _ = inputs(1, T, V, 64, seed=4, pad=0.0)
    size = torch.linspace(0.0, 3.0, V, device="cuda")[:, None]
    for s in (size, size.flip(0)):
        w2 = (w[0].abs().float() * 0.01 + s).bfloat16()[None].contiguous()
        run(h.abs(), w2, None, n_top)


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", [(1, 700), (2, 700), (30, 700), (300, 700), (1400, 50257)])
def test_values_that_are_not_finite(T, V):
    inf, nan = float("inf"), float("nan")
    D = 64
    _, w, _ = inputs(1, T, V, D, seed=6, pad=0.0)
    h = torch.ones((1, T, D), device="cuda").bfloat16()
    y = torch.zeros((1, T), dtype=torch.int32, device="cuda")
    for value, places in ((nan, [V - 1]), (nan, [0]), (inf, [300]), (inf, [3, 690])):
        w2 = w.clone()
        w2[0, places, 5] = value
        out = run(h, w2, y, 4, check=False)
        for k in ("logprob", "entropy", "lse", "top_logprob"):
            assert torch.isnan(out[k]).all(), (k, value)
        assert (out["top_ids"] == -1).all()
    # a class with the logit -inf has probability 0: as if the table had none
    gone = (0, 130, V - 1)
    w2, left = w.clone(), torch.tensor([i for i in range(V) if i not in gone], device="cuda")
    w2[0, list(gone), 5] = -inf
    out, ref = run(h, w2, y, 4, check=False), run(h, w2[:, left].contiguous(), None, 4)
    for k in ("entropy", "lse"):
        assert ((out[k] - ref[k]).abs() <= 2.0 ** -18 * ref[k].abs()).all(), k
    assert (out["logprob"] == -inf).all() and torch.equal(left[ref["top_ids"].long()].int(), out["top_ids"])
    # fewer of them than are asked for, and none
    w2[0, 2:, 5] = -inf
    out = run(h, w2, y + 1, 4, check=False)
    assert (out["top_ids"] == torch.tensor([1, -1, -1, -1], device="cuda")).all() and (out["top_logprob"][..., 1:] == -inf).all()
    assert (out["top_logprob"][..., 0] == 0).all() and (out["logprob"] == 0).all() and (out["entropy"] == 0).all()
    w2[0, :, 5] = -inf
    out = run(h, w2, y, 4, check=False)
    assert torch.isnan(out["lse"]).all() and (out["top_ids"] == -1).all()
    # one token's alone
    if T > 1:
        h2 = h.clone()
        h2[0, T - 1, 3] = nan
        out, ref = run(h2, w, y, 4, check=False), run(h, w, y, 4)
        assert torch.isnan(out["lse"][0, T - 1]) and torch.equal(out["lse"][0, :-1], ref["lse"][0, :-1])


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,D", [(T, V, D) for T in (1, 2, 130, 520) for V, D in ((50257, 64), (4099, 1088))] + [(1400, 50257, 64)])
def test_likely_tokens_keep_their_relative_precision(T, V, D):
    """Probabilities up to 1 - 1e-12: log probability and entropy are off by no more, relatively, than the logits' errors make them."""
    gen = torch.Generator().manual_seed(7)
    w = (torch.randn((1, V, D), generator=gen) * 0.05).bfloat16().cuda()
    y = torch.randint(0, V, (1, T), generator=gen).cuda()
    row = w[0][y[0]].float()
    want = torch.linspace(10.0, 36.0, T, device="cuda")[:, None]              # the target's logit
    h = (row * want / row.square().sum(1, keepdim=True)).bfloat16()[None]
    out = run(h, w, y.int(), 3, check=False)
    z = h[0].double() @ w[0].double().t()
    others = z.clone()
    others.scatter_(1, y[0][:, None], -float("inf"))
    gap = torch.logsumexp(others, 1) - z.gather(1, y[0][:, None])[:, 0]
    lp = -torch.log1p(torch.exp(gap))
    # with q the others' probability, entropy = -lp (1 - q) - sum of p log p over them
    logp = z - torch.logsumexp(z, 1, keepdim=True)
    rest = torch.where(torch.isinf(others), 0.0, logp.exp() * logp).sum(1)
    entropy = -lp * torch.exp(lp) - rest
    # a logit's error, as in the bounds above but of its own sum: products of one sign, cut by up to a step of 2^-23 for every 16 of them in
    # runs of 1024, then rounded; it multiplies the others' share.  The others' own errors are those of sums near zero.
    ez = z.amax(1).abs() * (min(D, 1024) / 16 + D / 1024 + 2) * 2.0 ** -23 + 2.0 ** -16
    assert ((out["logprob"][0].double() - lp).abs() <= lp.abs() * (2 * ez + 2.0 ** -14)).all()
    assert ((out["entropy"][0].double() - entropy).abs() <= entropy * (2 * ez + 2.0 ** -14)).all()
    assert (out["top_ids"][0, :, 0] == y[0]).all() and (out["top_logprob"][0, :, 0] == out["logprob"][0]).all()
    assert (out["logprob"] < 0).all() and (out["entropy"] > 0).all()


@pytest.mark.gpu
def test_the_order_is_that_of_sums_in_64_bits():
    """Rows that differ by less than an fp32 sum's error: large terms that cancel, and a small one that decides."""
    gen = torch.Generator().manual_seed(9)
    V, D = 3000, 512
    for T in (1, 2, 40, 300):
        h = torch.randn((1, T, D), generator=gen).bfloat16()
        w = torch.randn((1, V, D), generator=gen).bfloat16() * 0.01
        big = (torch.randn(D // 2, generator=gen) * 4).bfloat16()
        at = torch.randperm(V, generator=gen)[:4]
        h[..., 1::2] = h[..., ::2]                        # what row + big and row - big meet is equal
        for i, v in enumerate(at.tolist()):
            w[0, v] = 0.0
            w[0, v, ::2], w[0, v, 1::2] = big, -big
            w[0, v, 0] += 4.0                             # far above the rest for a positive first element
            w[0, v, 1] += 2.0 ** -8 * (i % 2)
        h[..., 0] = h[..., 1] = 1.0
        run(h.cuda(), w.cuda(), None, 8)


# ------------------------------------------------------------------------------------------------ streams, graphs, waits
@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 300])
def test_captured_and_on_another_stream(T):
    h, w, y = inputs(2, T, 2000, 64, seed=8)
    ref = run(h, w, y, 5)
    out = {k: torch.zeros_like(v) for k, v in ref.items()}
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y, n_top=5), dtype=torch.uint8, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.hdet_token_scores(h, w, y, ws, stream=side.cuda_stream, **out)
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], ref[k]) for k in out)
    with torch.cuda.graph(graph):
        B.hdet_token_scores(h, w, y, ws, stream=torch.cuda.current_stream().cuda_stream, **out)
    for v in out.values():
        v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], ref[k]) for k in out)


@pytest.mark.gpu
@pytest.mark.parametrize("R,T,V,D", [(1, 40, 2000, 64), (2, 600, 5000, 1088), (3, 300, 4099, 128), (1, 1400, 50257, 64)])
def test_a_wait_that_runs_out_marks_every_token(R, T, V, D):
    h, w, y = inputs(R, T, V, D, seed=11)
    ref = run(h, w, y, 4)
    out = {k: torch.zeros_like(v) for k, v in ref.items()}
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y, n_top=4), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    B.hdet_selftest_token_scores_wait(h, w, y, ws, stream=stream, **out)
    some = (y >= 0) & (y < V)
    for k in ("logprob", "entropy", "lse"):
        assert torch.equal(torch.isnan(out[k]), some), k
    assert (out["top_ids"] == -1).all() and torch.equal(torch.isnan(out["top_logprob"]).all(-1), some)
    B.hdet_token_scores(h, w, y, ws, stream=stream, **out)
    assert all(torch.equal(out[k], ref[k]) for k in out)
