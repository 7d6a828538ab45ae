"""Rows that are nearly certain among others and among padding: they are packed first, and every gradient has to end up at its own token."""
import pytest
import torch

from paper_2604_24708_b200 import binding as B
from test_token_scores import strided
from test_token_scores_grad_confident import DT, _confident, _exact


def _batch(R, T, V, D, seed):
    """Per replica: half of the tokens point at a class, the others at none; a third is padding, where everything is NaN."""
    gen = torch.Generator().manual_seed(seed)
    h, w, y, top = [], [], [], []
    for r in range(R):
        h1, w1, top1 = _confident(T, V, D, seed=seed + r, least=14.0, most=30.0)
        sure = (torch.rand(T, generator=gen) < 0.5).cuda()
        h1 = torch.where(sure[:, None], h1, torch.randn((T, D), generator=gen).bfloat16().cuda())
        y1 = torch.randint(0, V, (T,), generator=gen).cuda()
        own = (torch.rand(T, generator=gen) < 0.3).cuda()
        y1 = torch.where(own, top1, y1)
        pad = (torch.rand(T, generator=gen) < 0.33).cuda()
        h.append(torch.where(pad[:, None], float("nan"), h1.float()).bfloat16())
        y.append(torch.where(pad, -100, y1))
        w.append(w1)
        top.append((h1.double() @ w1.double().t()).argmax(1))
    return torch.stack(h), torch.stack(w), torch.stack(y).int(), torch.stack(top)


def _call(h, w, y, a, b, out, piece_bytes=0, accumulate=False):
    R, T = y.shape
    stream = torch.cuda.current_stream().cuda_stream
    lse, entropy, logprob = (torch.empty((R, T), device="cuda") for _ in range(3))
    ws = torch.empty(B.hdet_token_scores_workspace(h, w, y), dtype=torch.uint8, device="cuda")
    B.hdet_token_scores(h, w, y, ws, logprob=logprob, entropy=entropy, lse=lse, stream=stream)
    some = y >= 0
    lse, entropy, logprob = (torch.where(some, x, float("nan")) for x in (lse, entropy, logprob))
    ws = torch.full((B.hdet_token_scores_grad_workspace(h, w, y, piece_bytes=piece_bytes, **out),), 0xFF, dtype=torch.uint8, device="cuda")
    go = lambda: B.hdet_token_scores_grad(h, w, y, ws, lse, logprob=logprob, entropy=entropy, d_logprob=a, d_entropy=b, piece_bytes=piece_bytes,  # noqa: E731
                                          accumulate=accumulate, stream=torch.cuda.current_stream().cuda_stream, **out)
    go()
    return go


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("R,T,V,D,layout,piece_bytes", [
    (1, 9, 700, 64, (0, 0, 0), 0), (3, 200, 4099, 264, (3, 5, 1), 0), (2, 700, 1500, 520, (8, 64, 8), 0), (2, 700, 1500, 520, (0, 0, 0), 1_500_000),
    (1, 3000, 3001, 64, (0, 0, 0), 0), (2, 300, 8200, 1096, (1, 0, 0), 3_000_000)])
def test_every_gradient_is_its_own_tokens(R, T, V, D, layout, piece_bytes, dt):
    h, w, y, top = _batch(R, T, V, D, seed=T)
    gen = torch.Generator().manual_seed(2)
    a, b = torch.randn((R, T), generator=gen).cuda() * 1e-3, torch.randn((R, T), generator=gen).cuda()      # the entropies' part is what counts
    b[:, ::5] = 0.0
    some = y >= 0
    a, b = torch.where(some, a, float("nan")), torch.where(some, b, float("nan"))
    out = dict(d_hidden=strided((R, T, D), DT[dt], *layout, 0.0)[1], d_weight=strided((R, V, D), DT[dt], *layout, 0.0)[1])
    go = _call(h, w, y, a, b, out, piece_bytes)
    first = {k: v.clone() for k, v in out.items()}
    for r in range(R):
        t = some[r].nonzero()[:, 0]
        hd, wd, yy, tt = h[r, t].double(), w[r].double(), y[r, t].long(), top[r, t]
        zero = torch.zeros_like(hd[:, 0])
        z, lp, g_a = _exact(h[r, t], w[r], tt, yy, a[r, t].double(), zero)
        g_b = _exact(h[r, t], w[r], tt, yy, zero, b[r, t].double())[2]
        g, size = g_a + g_b, g_a.abs() + g_b.abs()
        # as beside the same bound for certain rows alone; the others' logarithms and entropies are off by the logits' errors, too, which in entries
        # near zero is relative to |lp| + H, not to their sum
        ez = z.abs().amax(1) * (min(D, 1024) / 16 + D / 512 + 2) * 2.0 ** -23 + 2.0 ** -16
        rel = 4 * ez + z.abs().amax(1) * 2.0 ** -22 + 2.0 ** -14
        p = lp.exp()
        entropy = -(p * lp).sum(1, keepdim=True)
        unsure = (entropy > 0.2).double()
        size = size + unsure * p * b[r, t].double().abs()[:, None] * (lp.abs() + entropy)
        rounding = 2.0 ** -8 if dt == "bf16" else 2.0 ** -22
        ref_h, ref_w = torch.zeros((T, D), dtype=torch.float64, device="cuda"), g.t() @ hd
        ref_h[t] = g @ wd
        bound_h = torch.zeros(T, dtype=torch.float64, device="cuda")
        bound_h[t] = (size @ wd.norm(dim=1)) * rel + (g.abs() @ wd.norm(dim=1)) * rounding
        bound_w = (size * hd.norm(dim=1)[:, None] * rel[:, None]).sum(0) + (g.abs() * hd.norm(dim=1)[:, None]).sum(0) * rounding
        assert ((first["d_hidden"][r].double() - ref_h).norm(dim=1) <= bound_h + ref_h.norm(dim=1) * rounding).all()
        # one ordinary sum over tokens more, in fp32
        assert ((first["d_weight"][r].double() - ref_w).norm(dim=1) <= bound_w + ref_w.norm(dim=1) * rounding + 1e-30).all()
    # the same bits on another stream and from a graph, over a workspace that another call has used
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], first[k]) for k in out)
    with torch.cuda.graph(graph):
        go()
    for v in out.values():
        v.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], first[k]) for k in out)


@pytest.mark.gpu
def test_added_to_what_is_there():
    h, w, y, _ = _batch(2, 260, 900, 136, seed=3)
    a, b = torch.full((2, 260), 1e-3, device="cuda"), torch.full((2, 260), 0.5, device="cuda")
    dw, start = torch.empty((2, 900, 136), device="cuda"), torch.randn((2, 900, 136), device="cuda")
    _call(h, w, y, a, b, dict(d_weight=dw))
    both = start.clone()
    _call(h, w, y, a, b, dict(d_weight=both), accumulate=True)
    assert torch.equal(both, start + dw)
