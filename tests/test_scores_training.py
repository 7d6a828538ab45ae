"""The operators together: a step on weighted tokens with an entropy term, between the two ends of a tied table, clipped and captured."""
import pytest
import torch

from paper_2604_24708_b200 import binding as B


def _setup(n, T, V, D, grad_dtype, opt, **kw):
    from paper_2604_24708_b200.arena import StackedArena
    from paper_2604_24708_b200.vocab import TiedTable
    gen = torch.Generator(device="cuda").manual_seed(0)
    arena = StackedArena([V * D, 3 * D], [0, 0], n, opt, B.HDET_DTYPE_F32 if grad_dtype == torch.float32 else B.HDET_DTYPE_BF16)
    arena.param.normal_(0, 0.3, generator=gen)
    h = B.hdet_create(B.hdet_config(n_replicas=n, n_groups=1, optimizer=opt, grad_dtype=arena.grad_dtype, beta1=0.9, beta2=0.999, eps=1e-8,
                                    alpha_lr=0.2, sync_interval=2, fuse_converge=1), arena.descriptors())
    B.hdet_set_schedule(h, B.make_schedule(B.HDET_SCHED_CONSTANT, 100, [1e-2]))
    table = TiedTable(arena, 0, V, D, T, scale=0.5, scores=True, **kw)
    ids = torch.randint(0, V, (n, T + 1), generator=gen, device="cuda", dtype=torch.int32)
    ids[:, -3:] = -1
    out = {k: torch.zeros((n, T), device="cuda") for k in ("logprob", "entropy", "lse")}
    return arena, h, table, ids, out, gen


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_against_64_bits(dtype):
    """Gradients, norms and the parameters after a clipped step of plain SGD."""
    n, T, V, D, beta = 3, 200, 1000, 64, 0.05
    arena, h, table, ids, out, gen = _setup(n, T, V, D, dtype, B.HDET_OPT_SGD)
    hidden, d_hidden = torch.empty((n, T, D), dtype=torch.bfloat16, device="cuda"), torch.empty((n, T, D), dtype=dtype, device="cuda")
    advantage = torch.randn((n, T), generator=gen, device="cuda") / T
    norms, losses = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    start = arena.param.double()
    table.embed(ids[:, :T], hidden)
    y = ids[:, 1:].contiguous()
    table.scores(hidden, y, **out)
    # the loss: - sum of advantage x log probability - beta x mean entropy
    table.scores_grad(hidden, y, out["lse"], d_hidden, logprob=out["logprob"], entropy=out["entropy"], d_logprob=-advantage,
                      d_entropy=torch.full((n, T), -beta / T, device="cuda"))
    table.embed_grad(ids[:, :T], d_hidden)
    stream = torch.cuda.current_stream().cuda_stream
    B.hdet_grad_norm(h, norms, stream=stream)
    limit = float(norms.median())
    clipped = torch.zeros(n, device="cuda")
    B.hdet_set_clip(h, limit, clipped)
    B.hdet_step_device(h, losses, stream)
    torch.cuda.synchronize()
    assert torch.equal(norms, clipped)
    # the two gradients of the table, in 64 bits from the values that the calls were given
    tol = 2.0 ** -15 if dtype == torch.float32 else 3 * 2.0 ** -8           # bf16: G, the hidden states' gradient and the sum are rounded
    st = B.hdet_get_state(h)
    for r in range(n):
        w = table.weight[r].double().requires_grad_()
        hid = hidden[r].double().requires_grad_()
        keep = (y[r] >= 0).nonzero()[:, 0]
        lp = torch.log_softmax(hid[keep] @ w.t(), 1)
        loss = -(advantage[r][keep].double() * lp[torch.arange(len(keep)), y[r][keep].long()]).sum() + beta / T * (lp.exp() * lp).sum()
        loss.backward()
        want = w.grad.clone()
        some = (ids[r, :T] >= 0).nonzero()[:, 0]
        want.index_add_(0, ids[r, :T][some].long(), 0.5 * hid.grad[some])
        got = table.grad[r].double()
        assert float((got - want).norm()) <= tol * float(want.norm())
        assert abs(float(norms[r]) - float(want.norm())) <= tol * float(want.norm())
        factor = min(1.0, limit / float(norms[r]))
        moved = (arena.param[r].double() - start[r])[:V * D].view(V, D)
        # a step of fp32 of the parameters, and the gradient's
        assert ((moved + st.lr[0][r] * factor * got).abs() <= 2.0 ** -23 * start[r][:V * D].view(V, D).abs() + 1e-6 * moved.abs() + 1e-12).all()
    B.hdet_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_captured_into_one_graph_are_the_steps(dtype):
    n, T, V, D = 2, 130, 700, 72

    def build():
        arena, h, table, ids, out, gen = _setup(n, T, V, D, dtype, B.HDET_OPT_ADAMW, n_top=4)
        hidden, d_hidden = torch.empty((n, T, D), dtype=torch.bfloat16, device="cuda"), torch.empty((n, T, D), dtype=dtype, device="cuda")
        a, b = torch.randn((n, T), generator=gen, device="cuda") / T, torch.full((n, T), -0.1 / T, device="cuda")
        top, top_lp = torch.zeros((n, T, 4), dtype=torch.int32, device="cuda"), torch.zeros((n, T, 4), device="cuda")
        norms, losses, y = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), ids[:, 1:].contiguous()
        B.hdet_set_clip(h, 1e-3, norms)

        def step():
            table.embed(ids[:, :T], hidden)
            table.scores(hidden, y, top_ids=top, top_logprob=top_lp, **out)
            torch.sum(out["logprob"], 1, out=losses)
            table.scores_grad(hidden, y, out["lse"], d_hidden, logprob=out["logprob"], entropy=out["entropy"], d_logprob=a, d_entropy=b)
            table.embed_grad(ids[:, :T], d_hidden)
            B.hdet_step_device(h, losses, torch.cuda.current_stream().cuda_stream)
            table.refresh()
        return arena, h, step, norms, top, top_lp
    eager, captured = build(), build()
    for _ in range(6):
        eager[2]()
    for _ in range(2):                   # a round of two: the state is on the device
        captured[2]()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(2):
            captured[2]()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(eager[3:], captured[3:]):
        assert torch.equal(x, y)
    assert torch.equal(eager[0].param, captured[0].param) and torch.isfinite(eager[0].param).all()
    graph.reset()
    for e in (eager, captured):
        B.hdet_destroy(e[1])


@pytest.mark.gpu
def test_the_table_takes_shorter_batches_and_fewer_alternatives():
    n, T, V, D = 3, 400, 1000, 64
    arena, h, table, ids, out, gen = _setup(n, T, V, D, torch.bfloat16, B.HDET_OPT_ADAMW, n_top=20, piece_bytes=1_000_000)
    with pytest.raises(ValueError):
        table.scores(torch.zeros((n, T, D), device="cuda").bfloat16(), None, top_ids=torch.zeros((n, T, 21), dtype=torch.int32, device="cuda"))
    for t in (400, 399, 200, 192, 64, 5, 2, 1):
        hidden = torch.randn((n, t, D), generator=gen, device="cuda").bfloat16()
        y = ids[:, :t].contiguous()
        for k in (0, 1, 12, 13, 20):
            res = {name: torch.zeros((n, t), device="cuda") for name in out}
            top = torch.zeros((n, t, k), dtype=torch.int32, device="cuda") if k else None
            table.scores(hidden, y, top_ids=top, **res)
            if k:
                z = hidden.double() @ table.weight.double().transpose(1, 2)
                best = torch.sort(z, dim=-1, descending=True, stable=True).indices[..., :k].int()
                assert torch.equal(top, torch.where((y >= 0)[..., None], best, -1))
        d_hidden = torch.empty_like(hidden)
        table.scores_grad(hidden, y, res["lse"], d_hidden, logprob=res["logprob"], d_logprob=torch.ones((n, t), device="cuda"))
        assert torch.isfinite(d_hidden).all() and torch.isfinite(table.grad).all()
    B.hdet_destroy(h)


def test_the_table_says_what_it_was_not_built_for():
    from paper_2604_24708_b200.vocab import TiedTable
    table = TiedTable.__new__(TiedTable)
    table.n_top = -1
    with pytest.raises(ValueError):
        table.scores(None, None)
    with pytest.raises(ValueError):
        table.scores_grad(None, None, None, None)
