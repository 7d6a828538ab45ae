"""The vocabulary ends as they are used together: lookup, loss, both gradients into the arena, device-resident update."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2604_24708_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DT = {B.HDET_DTYPE_F32: torch.float32, B.HDET_DTYPE_BF16: torch.bfloat16}


class _Model:
    """N replicas of: rows of wte -> multiplied by a vector g -> logits against wte.  Tensors: wte, g (and one that nothing
    touches, between them, to see that it stays)."""

    def __init__(self, n, T, V, D, grad_dtype, sync=2, use_mean=False):
        from paper_2604_24708_b200.arena import StackedArena
        from paper_2604_24708_b200.vocab import TiedTable
        self.n, self.T, self.V, self.D = n, T, V, D
        gen = torch.Generator(device="cuda").manual_seed(1)
        self.arena = StackedArena([V * D, 11, D], [0, 1, 1], n, B.HDET_OPT_ADAMW, grad_dtype, bf16_copy=use_mean)
        start = torch.randn(self.arena.p_pad, generator=gen, device="cuda") * 0.2
        self.arena.param.copy_(start.expand(n, -1))
        self.g = self.arena.param_view(2, (D,))
        self.g.fill_(1.0)
        if use_mean:
            self.arena.param_bf16.copy_(self.arena.param[0])
        cfg = B.hdet_config(n_replicas=n, n_groups=2, optimizer=B.HDET_OPT_ADAMW, grad_dtype=grad_dtype, beta1=0.9, beta2=0.99, eps=1e-8,
                            alpha_lr=0.25, sync_interval=sync, fuse_converge=1, seed=3)
        self.h = B.hdet_create(cfg, self.arena.descriptors())
        B.hdet_set_schedule(self.h, B.make_schedule(B.HDET_SCHED_CONSTANT, 100, [2e-2, 1e-2]))
        self.table = TiedTable(self.arena, 0, V, D, T, scale=2.0, use_mean=use_mean)
        dev = dict(device="cuda")
        self.rows = torch.empty((n, T, D), dtype=torch.bfloat16, **dev)
        self.hidden, self.d_hidden, self.d_rows = (torch.empty_like(self.rows) for _ in range(3))
        self.losses = torch.empty(n, dtype=torch.float64, **dev)
        self.ids = torch.empty((n, T + 1), dtype=torch.int32, **dev)
        self.g_grad = self.arena.grad_view(2, (D,))

    def batch(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.ids.copy_(torch.randint(0, self.V, self.ids.shape, generator=gen, device="cuda", dtype=torch.int32))
        self.ids[:, -self.T // 4:] = -1             # the end of every sequence is padding

    def step(self):
        t = self.table
        t.embed(self.ids[:, :self.T], self.rows)
        torch.mul(self.rows, self.g[:, None].bfloat16(), out=self.hidden)
        t.loss(self.hidden, self.ids[:, 1:], self.losses, d_hidden=self.d_hidden)
        torch.mul(self.d_hidden, self.g[:, None].bfloat16(), out=self.d_rows)
        self.g_grad.copy_((self.d_hidden.float() * self.rows.float()).sum(1))
        t.embed_grad(self.ids[:, :self.T], self.d_rows)
        B.hdet_step_device(self.h, self.losses, torch.cuda.current_stream().cuda_stream)
        t.refresh()

    def close(self):
        torch.cuda.synchronize()
        B.hdet_destroy(self.h)


def _table_gradient(m):
    """The table's gradient of the step that `m` holds the inputs of, in 64 bits, and the sum of its terms' magnitudes."""
    total = torch.zeros((m.n, m.V, m.D), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    for r in range(m.n):
        x, y = m.ids[r, :m.T].long(), m.ids[r, 1:].long()
        w = (m.table.weight if m.table.use_mean else m.table.weight[r]).double()
        keep = y >= 0
        h = m.hidden[r][keep].double()
        p = torch.softmax(h @ w.t(), 1)
        p[torch.arange(len(h)), y[keep]] -= 1.0
        p /= keep.sum()
        total[r] = p.t() @ h
        size[r] = p.t().abs() @ h.abs()
        some = x >= 0
        rows = m.d_rows[r][some].double() * 2.0
        total[r].index_add_(0, x[some], rows)
        size[r].index_add_(0, x[some], rows.abs())
    return total, size


@pytest.mark.gpu
@pytest.mark.parametrize("grad_dtype", [B.HDET_DTYPE_F32, B.HDET_DTYPE_BF16])
@pytest.mark.parametrize("use_mean", [False, True])
def test_training_steps(grad_dtype, use_mean):
    m = _Model(3, 96, 400, 40, grad_dtype, sync=1 if use_mean else 2, use_mean=use_mean)
    untouched = m.arena.grad_view(1, (11,)).clone()
    for i in range(4):
        m.batch(i)
        before = m.arena.param.clone()
        m.step()
        torch.cuda.synchronize()
        # the step refreshed the copy; what the loss read is the copy of the parameters before it
        if use_mean:
            weight_now, m.table.weight = m.table.weight, before[0, :m.V * m.D].view(m.V, m.D).bfloat16()
        else:
            weight_now, m.table.weight = m.table.weight, before[:, :m.V * m.D].view(m.n, m.V, m.D).bfloat16()
        ref, size = _table_gradient(m)
        m.table.weight = weight_now
        got = m.table.grad.double()
        # the softmax's gradient as operand (2^-8, or 2^-16 as a pair), twice the output's rounding (loss, then lookup), and
        # fp32 sums and exponentials
        half = torch.finfo(DT[grad_dtype]).eps / 2
        tol = size * ((2.0 ** -8 if grad_dtype == B.HDET_DTYPE_BF16 else 2.0 ** -16) + 2 * half + 512 * 2.0 ** -23)
        assert ((got - ref).abs() <= tol).all()
        assert torch.equal(m.arena.grad_view(1, (11,)), untouched)
        assert torch.isfinite(m.losses).all()
        assert (m.arena.param_view(0, (m.V, m.D)) != before[:, :m.V * m.D].view(m.n, m.V, m.D)).any()
    st = B.hdet_get_state(m.h)
    assert st.step == 4 and st.device_status == 0
    m.close()


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(2, 64, 300, 64), (2, 200, 700, 72)], ids=str)
def test_a_captured_round_gives_the_same_bits(size):
    n, T, V, D = size
    batches = range(2)

    def run(captured):
        m = _Model(n, T, V, D, B.HDET_DTYPE_BF16, sync=2)
        for k in batches:                            # the first round directly
            m.batch(k)
            m.step()
        torch.cuda.synchronize()
        if captured:
            side = torch.cuda.Stream()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                m.step()
                m.step()
            for k in range(2):
                m.batch(5 + k)
                graph.replay()
        else:
            for k in range(2):
                m.batch(5 + k)
                m.step()
                m.step()
        torch.cuda.synchronize()
        out = m.arena.param.clone(), m.losses.clone()
        m.close()
        return out
    (pa, la), (pb, lb) = run(False), run(True)
    assert torch.equal(pa, pb) and torch.equal(la, lb)


FIRST = r"""
import torch
from paper_2604_24708_b200 import binding as B
h, w = torch.randn(2, 200, 64, device="cuda").bfloat16(), torch.randn(2, 300, 64, device="cuda").bfloat16()
y = torch.randint(0, 300, (2, 200), device="cuda", dtype=torch.int32)
out = dict(loss=torch.empty(2, device="cuda"), d_hidden=torch.empty_like(h), d_weight=torch.empty_like(w))
ws = torch.empty(B.hdet_token_loss_workspace(h, w, y, d_hidden=out["d_hidden"], d_weight=out["d_weight"]), dtype=torch.uint8, device="cuda")
es = torch.empty(B.hdet_embed_grad_workspace(y, h, w), dtype=torch.uint8, device="cuda")
rows, table = torch.empty_like(h), torch.empty_like(w)
def call():
    s = torch.cuda.current_stream().cuda_stream
    B.hdet_embed(y, w, rows, stream=s)
    B.hdet_embed_grad(y, h, table, es, stream=s)
    B.hdet_token_loss(h, w, y, workspace=ws, stream=s, **out)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    call()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (rows, table, *out.values())]
call()
assert all(torch.equal(a, b) for a, b in zip(got, (rows, table, *out.values())))
print("same bits")
"""


@pytest.mark.gpu
def test_the_first_calls_of_a_process_can_be_captured():
    res = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "same bits" in res.stdout, res.stdout + res.stderr


def test_the_table_checks_its_tensor():
    from paper_2604_24708_b200.vocab import TiedTable

    class Arena:
        numels, shared_grad = [12], False
    with pytest.raises(ValueError):
        TiedTable(Arena(), 0, 5, 3, 4)
    Arena.shared_grad = True
    with pytest.raises(ValueError):
        TiedTable(Arena(), 0, 4, 3, 4)


@pytest.mark.gpu
def test_a_table_takes_shorter_batches():
    """Batches of up to n_tokens, with the loss alone, and with gradients of the hidden states in either type."""
    from paper_2604_24708_b200.arena import StackedArena
    from paper_2604_24708_b200.vocab import TiedTable
    n, T, V, D = 3, 400, 1000, 64
    arena = StackedArena([V * D], [0], n, B.HDET_OPT_ADAMW, B.HDET_DTYPE_BF16)
    arena.param.normal_(0, 0.3)
    table = TiedTable(arena, 0, V, D, T, piece_bytes=1_000_000)
    for t in (400, 399, 300, 200, 192, 130, 64, 5, 4, 1):
        ids = torch.randint(0, V, (n, t + 1), device="cuda", dtype=torch.int32)
        hidden = torch.randn((n, t, D), device="cuda").bfloat16()
        losses, again = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        for dt in (None, torch.bfloat16, torch.float32):
            d_hidden = None if dt is None else torch.empty((n, t, D), dtype=dt, device="cuda")
            table.loss(hidden, ids[:, 1:], losses, d_hidden=d_hidden)
            if dt is None:
                continue
            apart, grad = torch.empty_like(d_hidden), torch.empty_like(table.grad)
            ws = torch.empty(B.hdet_token_loss_workspace(hidden, table.weight, ids[:, 1:], d_hidden=apart, d_weight=grad, piece_bytes=1_000_000),
                             dtype=torch.uint8, device="cuda")
            B.hdet_token_loss(hidden, table.weight, ids[:, 1:], again, ws, d_hidden=apart, d_weight=grad, piece_bytes=1_000_000,
                              stream=torch.cuda.current_stream().cuda_stream)
            assert torch.equal(losses, again) and torch.equal(apart, d_hidden) and torch.equal(grad, table.grad)
            table.embed_grad(ids[:, :t], d_hidden)
