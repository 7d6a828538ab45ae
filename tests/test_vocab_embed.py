"""Embedding lookup and its gradient against plain sums in 64 bits, and the refusals of their arguments."""
import ctypes as C

import pytest
import torch

from paper_2604_24708_b200 import binding as B

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = 7.25   # what the places around an output hold before and after a call


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def _desc(**kw):
    d = B.hdet_embedding(0x1000, 0x2000, 0x3000, 4, 10, 8, 4, 32, 8, 80, 8, 1.0, 2, B.HDET_DTYPE_I32, B.HDET_DTYPE_F32,
                         B.HDET_DTYPE_F32, 0, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD = [
    (dict(n_replicas=0), B.HDET_ERR_INVALID_ARG), (dict(n_replicas=33), B.HDET_ERR_INVALID_ARG),
    (dict(n_tokens=-1), B.HDET_ERR_INVALID_ARG), (dict(n_tokens=B.HDET_MAX_TOKENS + 1), B.HDET_ERR_INVALID_ARG),
    (dict(vocab=0), B.HDET_ERR_INVALID_ARG), (dict(vocab=B.HDET_MAX_VOCAB + 1), B.HDET_ERR_INVALID_ARG),
    (dict(width=0), B.HDET_ERR_INVALID_ARG), (dict(width=B.HDET_MAX_WIDTH + 1), B.HDET_ERR_INVALID_ARG),
    (dict(token_dtype=B.HDET_DTYPE_F32), B.HDET_ERR_INVALID_ARG), (dict(rows_dtype=B.HDET_DTYPE_F64), B.HDET_ERR_INVALID_ARG),
    (dict(table_dtype=9), B.HDET_ERR_INVALID_ARG), (dict(device=-1), B.HDET_ERR_INVALID_ARG),
    (dict(scale=float("nan")), B.HDET_ERR_INVALID_ARG), (dict(scale=float("inf")), B.HDET_ERR_INVALID_ARG),
    (dict(table_row=7), B.HDET_ERR_INVALID_ARG), (dict(rows_row=7), B.HDET_ERR_INVALID_ARG),
    (dict(tokens=None), B.HDET_ERR_INVALID_ARG), (dict(rows=None), B.HDET_ERR_INVALID_ARG),
    (dict(table=None), B.HDET_ERR_INVALID_ARG), (dict(token_stride=3), B.HDET_ERR_INVALID_ARG),
    (dict(table_stride=79), B.HDET_ERR_INVALID_ARG), (dict(rows_stride=31), B.HDET_ERR_INVALID_ARG),
    (dict(token_stride=-1), B.HDET_ERR_INVALID_ARG), (dict(rows=0x2002), B.HDET_ERR_ALIGN),
    (dict(table=0x3001), B.HDET_ERR_ALIGN), (dict(tokens=0x1004, token_dtype=B.HDET_DTYPE_I64), B.HDET_ERR_ALIGN),
]


@pytest.mark.parametrize("change,status", BAD, ids=[str(b[0]) for b in BAD])
def test_refusals(change, status):
    d, lib = _desc(**change), B.raw_library()
    assert lib.hdet_embed(C.byref(d), None) == status
    assert b"hdet_embed" in lib.hdet_last_error(None)
    assert lib.hdet_embed_grad(C.byref(d), 0, 0x4000, 1 << 40, None) == status


def test_refusals_of_one_direction():
    lib, need = B.raw_library(), C.c_int64(0)
    # one output for all replicas
    assert lib.hdet_embed(C.byref(_desc(rows_stride=0)), None) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_embed_grad(C.byref(_desc(table_stride=0)), 0, 0x4000, 1 << 40, None) == B.HDET_ERR_INVALID_ARG
    # workspaces
    assert lib.hdet_embed_grad_workspace(C.byref(_desc()), C.byref(need)) == B.HDET_OK and need.value >= 256
    assert lib.hdet_embed_grad(C.byref(_desc()), 0, None, need.value, None) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_embed_grad(C.byref(_desc()), 0, 0x4000, need.value - 1, None) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_embed_grad(C.byref(_desc()), 0, 0x4010, need.value, None) == B.HDET_ERR_ALIGN
    assert lib.hdet_embed_grad_workspace(C.byref(_desc()), None) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_embed_grad_workspace(C.byref(_desc(width=0)), C.byref(need)) == B.HDET_ERR_INVALID_ARG
    assert lib.hdet_embed(None, None) == B.HDET_ERR_INVALID_ARG


def test_nothing_to_look_up_needs_no_device():
    assert B.raw_library().hdet_embed(C.byref(_desc(n_tokens=0)), None) == B.HDET_OK


def test_the_struct_matches_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    (tmp_path / "t.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hdet.h"\nint main(void) {'
                                  'printf("%zu %zu %zu %zu", sizeof(hdet_embedding), offsetof(hdet_embedding, scale), '
                                  'offsetof(hdet_embedding, table_row), offsetof(hdet_embedding, device)); return 0; }')
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    got = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()
    E = B.hdet_embedding
    assert [int(x) for x in got] == [C.sizeof(E), E.scale.offset, E.table_row.offset, E.device.offset]


# ------------------------------------------------------------------------------------------------ inputs
def _tokens(gen, R, T, V, kind, dtype):
    if kind == "same":
        t = torch.full((R, T), V // 2)
    elif kind == "zipf":
        t = ((V + 1.0) ** torch.rand((R, T), generator=gen) - 1).long().clamp(0, V - 1)
    elif kind == "distinct":
        t = torch.stack([torch.randperm(max(V, T), generator=gen)[:T] for _ in range(R)])
    else:
        t = torch.randint(0, V, (R, T), generator=gen)
    if kind == "padded":
        bad = torch.tensor([-1, -100, V, V + 1, 2 ** 31 - 1, -2 ** 31])
        at = torch.rand((R, T), generator=gen) < 0.3
        t = torch.where(at, bad[torch.randint(0, len(bad), (R, T), generator=gen)], t)
        if dtype == torch.int64:
            t[at] += 0
            t.view(-1)[:1] = 2 ** 32 + 1     # not row 1
    if kind == "empty":
        t = torch.full((R, T), -1)
    return t.to(dtype)


def _strided(shape, dtype, pad_row, pad_rep, shift, fill):
    """A view [N, rows, width] inside a larger buffer filled with ``fill``: rows pad_row apart, replicas pad_rep, shifted."""
    n, rows, width = shape
    row = width + pad_row
    rep = rows * row + pad_rep
    buf = torch.full((shift + n * rep + 16,), fill, dtype=dtype, device="cuda")
    return buf, buf.as_strided((n, rows, width), (rep, row, 1), shift)


# width, row padding, replica padding, shift (elements): vector widths 8, 4, 2, 1 by width, stride or address
LAYOUTS = [(64, 0, 0, 0), (768, 8, 0, 8), (36, 0, 4, 0), (100, 2, 0, 0), (33, 0, 0, 0), (1, 0, 0, 0), (264, 0, 8, 1), (40, 0, 1, 0)]


# ------------------------------------------------------------------------------------------------ lookup
@pytest.mark.gpu
@pytest.mark.parametrize("table_dt,out_dt", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_lookup(table_dt, out_dt, layout):
    D, pad_row, pad_rep, shift = layout
    gen = torch.Generator().manual_seed(D)
    for R, T, V, kind, tdt, shared in [(1, 1, 1, "any", torch.int32, False), (3, 37, 50, "padded", torch.int64, False),
                                       (2, 130, 1000, "padded", torch.int32, True)]:
        tok = _tokens(gen, R, T, V, kind, tdt)
        _, table = _strided((1 if shared else R, V, D), DT[table_dt], pad_row, pad_rep, shift, float("nan"))
        table.copy_(torch.randn(table.shape, generator=gen))
        buf, out = _strided((R, T, D), DT[out_dt], pad_row, pad_rep, shift, GUARD)
        B.hdet_embed(tok.cuda(), table[0] if shared else table, out, scale=1.7, stream=torch.cuda.current_stream().cuda_stream)
        some = (tok >= 0) & (tok < V)
        at = torch.where(some, tok, 0).long()
        ref = torch.stack([table[0 if shared else r].cpu().double()[at[r]] for r in range(R)]) * 1.7 * some[..., None]
        got = out.cpu().double()
        # scale to fp32, product in fp32, output: three roundings
        assert ((got - ref).abs() <= ref.abs() * (half_step(DT[out_dt]) + 2 * 2.0 ** -24) * 1.001).all()
        assert (got[~some] == 0).all()
        out.fill_(GUARD)
        assert (buf == GUARD).all()


@pytest.mark.gpu
def test_lookup_one_batch_for_all_replicas_and_far_offsets():
    """Tokens without a replica axis; a table whose last rows lie behind 2^32 bytes and 2^31 elements."""
    V, D = 1_100_000, 2048
    table = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    tok = torch.tensor([V - 1, 0, V // 2, 1_048_577], dtype=torch.int32, device="cuda")
    want = torch.randn((4, D), device="cuda").bfloat16()
    table[tok.long()] = want
    out = torch.empty((2, 4, D), dtype=torch.float32, device="cuda")
    B.hdet_embed(tok, table, out, stream=torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out[0], want.float()) and torch.equal(out[1], want.float())


# ------------------------------------------------------------------------------------------------ gradient
def _grad_reference(tok, rows, V, scale, start):
    """(sums, sums of magnitudes) by row in 64 bits."""
    R, T = tok.shape
    total = torch.zeros((R, V, rows.shape[-1]), dtype=torch.float64)
    size = torch.zeros_like(total)
    for r in range(R):
        keep = (tok[r] >= 0) & (tok[r] < V)
        x = rows[r].double()[keep] * scale
        total[r].index_add_(0, tok[r][keep].long(), x)
        size[r].index_add_(0, tok[r][keep].long(), x.abs())
    if start is not None:
        size += start.abs()
        total += start
    return total, size


def _check_grad(tok, rows, out, start, V, scale, longest):
    ref, size = _grad_reference(tok, rows, V, scale, start)
    got = out.cpu().double()
    # n - 1 additions, the scale, its product and the last addition in fp32, each at most half a step of a partial sum that
    # the sum of magnitudes bounds; then the output's rounding
    tol = size * (longest + 3) * 2.0 ** -24 + ref.abs() * half_step(out.dtype) * 1.001
    assert ((got - ref).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows_dt,table_dt", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_gradient(rows_dt, table_dt, layout):
    D, pad_row, pad_rep, shift = layout
    gen = torch.Generator().manual_seed(100 + D)
    for R, T, V, kind, tdt, acc in [(1, 1, 3, "any", torch.int32, False), (2, 33, 5, "any", torch.int64, False),
                                    (3, 300, 40, "padded", torch.int32, True), (2, 257, 500, "padded", torch.int64, False),
                                    (1, 64, 70, "empty", torch.int32, False)]:
        tok = _tokens(gen, R, T, V, kind, tdt)
        _, rows = _strided((R, T, D), DT[rows_dt], pad_row, pad_rep, shift, float("nan"))
        rows.copy_(torch.randn(rows.shape, generator=gen))
        pad = (tok < 0) | (tok >= V)
        rows[pad.cuda()] = float("nan")        # what padding holds reaches no output
        buf, table = _strided((R, V, D), DT[table_dt], pad_row, pad_rep, shift, GUARD)
        table.copy_(torch.randn(table.shape, generator=gen) if acc else torch.full(table.shape, float("nan")))
        start = table.cpu().double() if acc else None
        ws = torch.empty(B.hdet_embed_grad_workspace(tok.cuda(), rows, table), dtype=torch.uint8, device="cuda")
        B.hdet_embed_grad(tok.cuda(), rows, table, ws, scale=0.7, accumulate=acc, stream=torch.cuda.current_stream().cuda_stream)
        longest = max([1] + [int(torch.bincount(tok[r][~pad[r]].long(), minlength=1).max()) for r in range(R) if (~pad[r]).any()])
        _check_grad(tok, torch.nan_to_num(rows.cpu().float()), table, start, V, 0.7, longest)
        table.fill_(GUARD)
        assert (buf == GUARD).all()


# token counts on both sides of the chunks' and the merges' sizes; runs of equal tokens that cover many blocks
@pytest.mark.gpu
@pytest.mark.parametrize("R,T,V,kind", [(1, 1023, 300, "zipf"), (2, 1024, 50257, "zipf"), (1, 1025, 4000, "distinct"),
                                        (2, 2048, 100, "any"), (1, 2049, 2000, "zipf"), (1, 5000, 3, "any"),
                                        (2, 16384, 50257, "zipf"), (1, 16385, 50257, "padded"), (1, 40000, 7, "same"),
                                        (1, 300000, 50257, "zipf")])
def test_gradient_of_long_batches(R, T, V, kind):
    D = 24
    gen = torch.Generator().manual_seed(T)
    tok = _tokens(gen, R, T, V, kind, torch.int32)
    # small integers: every order of additions gives the same fp32 sums, so the result has to be exact
    rows = torch.randint(-8, 9, (R, T, D), generator=gen).float()
    table = torch.empty((R, V, D), device="cuda")
    ws = torch.empty(B.hdet_embed_grad_workspace(tok.cuda(), rows.cuda(), table), dtype=torch.uint8, device="cuda")
    B.hdet_embed_grad(tok.cuda(), rows.cuda(), table, ws, stream=torch.cuda.current_stream().cuda_stream)
    ref, _ = _grad_reference(tok, rows, V, 1.0, None)
    assert torch.equal(table.cpu().double(), ref)


@pytest.mark.gpu
def test_gradient_repeats_its_bits_and_keeps_the_order_of_tokens():
    gen = torch.Generator().manual_seed(5)
    R, T, V, D = 2, 3000, 64, 72
    tok = _tokens(gen, R, T, V, "zipf", torch.int64).cuda()
    rows = torch.randn((R, T, D), generator=gen).cuda()
    table = torch.empty((R, V, D), device="cuda")
    ws = torch.empty(B.hdet_embed_grad_workspace(tok, rows, table), dtype=torch.uint8, device="cuda")
    seen = []
    for k in range(3):
        ws.fill_(255 * (k % 2))
        B.hdet_embed_grad(tok, rows, table, ws, stream=torch.cuda.current_stream().cuda_stream)
        seen.append(table.clone())
    assert torch.equal(seen[0], seen[1]) and torch.equal(seen[0], seen[2])


@pytest.mark.gpu
def test_gradient_shared_batch_and_shared_rows():
    """One batch of tokens and one gradient for all replicas; no tokens at all."""
    gen = torch.Generator().manual_seed(6)
    tok = _tokens(gen, 1, 100, 30, "padded", torch.int32)[0]
    rows = torch.randint(-4, 5, (100, 16), generator=gen).float()
    table = torch.full((3, 30, 16), 2.0, device="cuda")
    ws = torch.empty(B.hdet_embed_grad_workspace(tok.cuda(), rows.cuda(), table), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    B.hdet_embed_grad(tok.cuda(), rows.cuda(), table, ws, accumulate=True, stream=st)
    ref, _ = _grad_reference(tok[None], rows[None], 30, 1.0, None)
    for r in range(3):
        assert torch.equal(table[r].cpu().double(), ref[0] + 2.0)
    none = torch.empty((3, 0), dtype=torch.int32, device="cuda")
    B.hdet_embed_grad(none, torch.empty((3, 0, 16), device="cuda"), table, ws, stream=st)
    assert (table == 0).all()


@pytest.mark.gpu
def test_gradient_agrees_with_differences_of_the_lookup():
    """d/dw of <lookup(table), g>: the lookup is linear in the table, so a difference is exact up to rounding."""
    gen = torch.Generator().manual_seed(7)
    R, T, V, D = 2, 50, 9, 12
    tok = _tokens(gen, R, T, V, "padded", torch.int32).cuda()
    g = torch.randint(-4, 5, (R, T, D), generator=gen).float().cuda()
    base = torch.zeros((R, V, D), device="cuda")
    out, out1 = torch.empty((R, T, D), device="cuda"), torch.empty((R, T, D), device="cuda")
    grad = torch.empty((R, V, D), device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    ws = torch.empty(B.hdet_embed_grad_workspace(tok, g, grad), dtype=torch.uint8, device="cuda")
    B.hdet_embed_grad(tok, g, grad, ws, scale=0.5, stream=st)
    B.hdet_embed(tok, base, out, scale=0.5, stream=st)
    for r, v, c in [(0, 0, 0), (1, 8, 11), (0, 4, 5), (1, 2, 3)]:
        moved = base.clone()
        moved[r, v, c] += 2.0
        B.hdet_embed(tok, moved, out1, scale=0.5, stream=st)
        assert float(((out1 - out) * g).sum()) / 2.0 == float(grad[r, v, c])


@pytest.mark.gpu
def test_captured_and_replayed_on_another_stream():
    gen = torch.Generator().manual_seed(8)
    R, T, V, D = 2, 500, 300, 64
    tok = _tokens(gen, R, T, V, "zipf", torch.int32).cuda()
    table = torch.randn((R, V, D), generator=gen).cuda()
    out, grad = torch.empty((R, T, D), device="cuda"), torch.empty((R, V, D), device="cuda")
    ws = torch.empty(B.hdet_embed_grad_workspace(tok, out, grad), dtype=torch.uint8, device="cuda")

    def both():
        st = torch.cuda.current_stream().cuda_stream
        B.hdet_embed(tok, table, out, scale=2.0, stream=st)
        B.hdet_embed_grad(tok, out, grad, ws, stream=st)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    tok.copy_(_tokens(gen, R, T, V, "zipf", torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    first = (out.clone(), grad.clone())
    both()
    assert torch.equal(first[0], out) and torch.equal(first[1], grad)


def test_binding_refuses_wrong_shapes():
    t = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        B.hdet_embed(t, torch.zeros(2, 5, 8), torch.zeros(2, 3, 8))            # not on a CUDA device
    with pytest.raises(ValueError):
        B.hdet_embed(t, torch.zeros(2, 5, 8), torch.zeros(3, 8))
    with pytest.raises(ValueError):
        B.hdet_embed(t, torch.zeros(2, 5, 9), torch.zeros(2, 3, 8))
    with pytest.raises(ValueError):
        B.hdet_embed(t, torch.zeros(3, 5, 8), torch.zeros(2, 3, 8))
    with pytest.raises(ValueError):
        B.hdet_embed(t, torch.zeros(2, 5, 8).half(), torch.zeros(2, 3, 8))
    with pytest.raises(ValueError):
        B.hdet_embed(t, torch.zeros(2, 5, 16)[..., ::2], torch.zeros(2, 3, 8))
