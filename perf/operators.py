"""Cases for the vocabulary ends of the replicated decoder: embedding lookup, its gradient, and the token loss.

HDET keeps N replicas of a model on one GPU.  Around the update sit the two places where a decoder meets its
vocabulary, both on the tied table ``wte``:

* ``embed``       rows of the table for the tokens of every replica, times a scale;
* ``embed_grad``  the table's gradient, each row the sum of its tokens' gradients;
* ``loss``        softmax cross entropy of hidden states against the table: one mean per replica (what the
                  auto-LR controller reads) and one value per token;
* ``loss_grad``   the same with the gradients of hidden states and table;
* ``tied``        ``loss_grad`` followed by ``embed_grad`` added into the same table gradient.

A token or target outside 0 .. V-1 is padding: it has no row, no loss and no gradient.
Shapes: tokens, targets [R, T]; table, weight [R, V, D] ([V, D] when all replicas share it); hidden [R, T, D].
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_VOCAB = 50257          # the vocabulary of this repository's decoder lists


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one sequence, as when a model is sampled: latency
        dict(name="embed_one_token", op="embed", R=1, T=1, V=_VOCAB, D=768, table="f32", out="bf16", shared=False),
        # a training batch of eight replicas, each with its own fp32 master table (the 1.3 B list)
        dict(name="embed_replicas", op="embed", R=8, T=4096, V=_VOCAB, D=2048, table="f32", out="bf16", shared=False),
        # one averaged bf16 table for all replicas, odd sizes, fp32 activations
        dict(name="embed_shared_odd", op="embed", R=5, T=777, V=4099, D=1001, table="bf16", out="f32", shared=True),
        # a small ragged model with fp32 gradients
        dict(name="embed_grad_small", op="embed_grad", R=1, T=96, V=1000, D=72, grad="f32", table="f32"),
        # sixteen replicas of the 125 M list
        dict(name="embed_grad_125m", op="embed_grad", R=16, T=1024, V=_VOCAB, D=768, grad="bf16", table="bf16"),
        # eight replicas of the 1.3 B list, long batches
        dict(name="embed_grad_1p3b", op="embed_grad", R=8, T=8192, V=_VOCAB, D=2048, grad="bf16", table="bf16"),
        # the loss of one token: latency, bound by reading the table
        dict(name="loss_one_token", op="loss", R=1, T=1, V=_VOCAB, D=768, shared=False),
        # evaluation of eight replicas' hidden states against the averaged table (350 M list)
        dict(name="loss_eval_350m", op="loss", R=8, T=2048, V=_VOCAB, D=1024, shared=True),
        # a small ragged model with fp32 gradients
        dict(name="loss_grad_small", op="loss_grad", R=3, T=129, V=4099, D=520, grad="f32", shared=False),
        # a training step of sixteen replicas of the 125 M list
        dict(name="loss_grad_125m", op="loss_grad", R=16, T=1024, V=_VOCAB, D=768, grad="bf16", shared=False),
        # a training step of eight replicas of the 1.3 B list
        dict(name="loss_grad_1p3b", op="loss_grad", R=8, T=2048, V=_VOCAB, D=2048, grad="bf16", shared=False),
        # both ends of the tied table, gradients kept in fp32
        dict(name="tied_f32", op="tied", R=4, T=1024, V=_VOCAB, D=768, grad="f32", shared=False),
    ]


_TABLE_MAX = 8 * _VOCAB * 2048          # elements of the largest listed table
_ROWS_MAX = 8 * 8192 * 2048             # elements of the largest listed batch of rows
_LOGITS_MAX = 8 * 2048 * _VOCAB         # logits of the largest listed loss
_LOSS_MAX = _LOGITS_MAX * 2048


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "loss", "loss_grad", "tied"])
    while True:
        R, T = rng.randint(1, 16), _log_int(rng, 1, 8192)
        V, D = _log_int(rng, 64, 60000), _log_int(rng, 8, 2048)
        if rng.random() < 0.5:
            D = max(8, D // 64 * 64)
        if R * V * D > _TABLE_MAX or R * T * D > _ROWS_MAX:
            continue
        if op in ("loss", "loss_grad", "tied") and (R * T * V > _LOGITS_MAX or R * T * V * D > _LOSS_MAX / 4):
            continue
        break
    c = dict(op=op, R=R, T=T, V=V, D=D)
    if op == "embed":
        c.update(table=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]), shared=rng.random() < 0.3)
    elif op == "embed_grad":
        c.update(grad=rng.choice(["f32", "bf16"]), table=rng.choice(["f32", "bf16"]))
    elif op == "loss":
        c.update(shared=rng.random() < 0.3)
    elif op == "loss_grad":
        c.update(grad=rng.choice(["bf16", "bf16", "f32"]), shared=rng.random() < 0.3)
    else:
        c.update(grad="f32", shared=False)
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _ids(gen, R, T, V, pad):
    """Tokens whose frequencies fall like 1 / rank, as words' do; the end of every longer sequence is padding."""
    u = torch.rand((R, T), generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1).int()
    if T > 8:
        length = T - (torch.rand((R, 1), generator=gen, device="cuda") * 0.2 * T).long()
        ids = torch.where(torch.arange(T, device="cuda") < length, ids, pad)
    return ids.contiguous()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 17)
    R, T, V, D, op = c["R"], c["T"], c["V"], c["D"], c["op"]
    s = dict(case=c, scale=math.sqrt(D))
    if op in ("embed", "embed_grad", "tied"):
        s["tokens"] = _ids(gen, R, T, V, -1)
    if op == "embed":
        shape = (V, D) if c["shared"] else (R, V, D)
        s["table"] = (torch.randn(shape, generator=gen, device="cuda") * 0.02).to(_DT[c["table"]])
        s["out"] = torch.empty((R, T, D), device="cuda", dtype=_DT[c["out"]])
    if op in ("embed_grad", "tied"):
        gd = c["grad"] if op == "embed_grad" else "bf16"
        s["d_out"] = (torch.randn((R, T, D), generator=gen, device="cuda") * 1e-3).to(_DT[gd])
    if op == "embed_grad":
        s["d_table"] = torch.empty((R, V, D), device="cuda", dtype=_DT[c["table"]])
    if op in ("loss", "loss_grad", "tied"):
        shape = (V, D) if c["shared"] else (R, V, D)
        s["weight"] = (torch.randn(shape, generator=gen, device="cuda") * 0.02).bfloat16()
        s["targets"] = _ids(gen, R, T, V, -100)
        # hidden states of a model that has learnt something: each leans towards its target's row by some amount
        at = s["targets"].long().clamp(min=0)
        rows = s["weight"][at] if c["shared"] else torch.stack([s["weight"][r][at[r]] for r in range(R)])
        lean = torch.rand((R, T, 1), generator=gen, device="cuda") * (200.0 / math.sqrt(D))
        s["hidden"] = (torch.randn((R, T, D), generator=gen, device="cuda") + lean * rows.float()).bfloat16()
        s["loss"] = torch.empty((R,), device="cuda", dtype=torch.float32)
        s["token_loss"] = torch.empty((R, T), device="cuda", dtype=torch.float32)
    if op in ("loss_grad", "tied"):
        s["d_hidden"] = torch.empty((R, T, D), device="cuda", dtype=_DT[c["grad"]])
        s["d_weight"] = torch.empty((R, V, D), device="cuda", dtype=_DT[c["grad"]])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _embed_plain(s):
    tok, table, V = s["tokens"].long(), s["table"], s["case"]["V"]
    some = (tok >= 0) & (tok < V)
    at = torch.where(some, tok, 0)
    if table.dim() == 2:
        rows = table[at]
    else:
        rows = table[torch.arange(tok.shape[0], device="cuda")[:, None], at]
    return torch.where(some[..., None], rows.float() * s["scale"], 0.0).to(s["out"].dtype)


def _embed_grad_plain(s, R, V, D):
    tok = s["tokens"].long()
    some = (tok >= 0) & (tok < V)
    at = torch.where(some, tok, 0) + V * torch.arange(R, device="cuda")[:, None]
    g = torch.where(some[..., None], s["d_out"].float() * s["scale"], 0.0)
    total = torch.zeros((R * V, D), device="cuda", dtype=torch.float32)
    total.index_add_(0, at.reshape(-1), g.reshape(-1, D))
    return total.view(R, V, D)


def _loss_plain(s, grads):
    y, V = s["targets"].long(), s["case"]["V"]
    some = (y >= 0) & (y < V)
    at = torch.where(some, y, 0)[..., None]
    count = some.sum(1).clamp(min=1).float()
    h, w = s["hidden"].float(), s["weight"].float()
    e = torch.matmul(h, w.transpose(-1, -2))
    picked = torch.gather(e, 2, at)[..., 0]
    top = e.amax(-1, keepdim=True)
    e.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    each = torch.where(some, torch.log(total[..., 0]) + top[..., 0] - picked, 0.0)
    found = {"loss": each.sum(1) / count, "token_loss": each}
    if not grads:
        return found, None
    e.div_(total)
    e.scatter_add_(2, at, torch.full_like(total, -1.0))
    e.mul_((some.float() / count[:, None])[..., None])
    found["d_hidden"] = torch.matmul(e, w).to(s["d_hidden"].dtype)
    return found, torch.matmul(e.transpose(1, 2), torch.where(some[..., None], h, 0.0))


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "embed":
        return {"out": _embed_plain(s)}
    if op == "embed_grad":
        return {"d_table": _embed_grad_plain(s, c["R"], c["V"], c["D"]).to(s["d_table"].dtype)}
    found, d_weight = _loss_plain(s, op != "loss")
    if op == "loss_grad":
        found["d_weight"] = d_weight.to(s["d_weight"].dtype)
    elif op == "tied":
        found["d_weight"] = d_weight.add_(_embed_grad_plain(s, c["R"], c["V"], c["D"])).to(s["d_weight"].dtype)
    return found


# ------------------------------------------------------------------------------------------------ the framework's calls
def _workspace(s, name, need):
    """A workspace that the program keeps beside its inputs and gives to every call."""
    if name not in s:
        s[name] = torch.empty(max(16, need()), device="cuda", dtype=torch.uint8)
    return s[name]


def _run_own(s):
    from paper_2604_24708_b200 import binding as B

    op, stream = s["case"]["op"], torch.cuda.current_stream().cuda_stream
    if op == "embed":
        B.hdet_embed(s["tokens"], s["table"], s["out"], scale=s["scale"], stream=stream)
        return {"out": s["out"]}
    found = {}
    if op in ("loss", "loss_grad", "tied"):
        dh, dw = s.get("d_hidden"), s.get("d_weight")
        ws = _workspace(s, "loss_ws", lambda: B.hdet_token_loss_workspace(s["hidden"], s["weight"], s["targets"], d_hidden=dh, d_weight=dw))
        B.hdet_token_loss(s["hidden"], s["weight"], s["targets"], s["loss"], ws, token_loss=s["token_loss"], d_hidden=dh, d_weight=dw,
                          stream=stream)
        found.update(loss=s["loss"], token_loss=s["token_loss"])
        if dh is not None:
            found.update(d_hidden=dh, d_weight=dw)
    if op in ("embed_grad", "tied"):
        into = s["d_table"] if op == "embed_grad" else s["d_weight"]
        ws = _workspace(s, "embed_ws", lambda: B.hdet_embed_grad_workspace(s["tokens"], s["d_out"], into))
        B.hdet_embed_grad(s["tokens"], s["d_out"], into, ws, scale=s["scale"], accumulate=op == "tied", stream=stream)
        found["d_table" if op == "embed_grad" else "d_weight"] = into
    return found


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    c = case
    R, T, V, D, op = c["R"], c["T"], c["V"], c["D"], c["op"]
    size = {"f32": 4, "bf16": 2}
    b = f = 0.0
    if op == "embed":
        b += 4 * R * T + min(R * T, (1 if c["shared"] else R) * min(T * R, V)) * D * size[c["table"]] + R * T * D * size[c["out"]]
        f += R * T * D
    if op == "embed_grad":
        b += 4 * R * T + R * T * D * size[c["grad"]] + R * V * D * size[c["table"]]
        f += 2 * R * T * D
    if op == "tied":                                   # the table's gradient is counted once, below
        b += 4 * R * T + R * T * D * 2
        f += 2 * R * T * D
    if op in ("loss", "loss_grad", "tied"):
        b += R * T * D * 2 + (1 if c["shared"] else R) * V * D * 2 + 4 * R * T + 4 * R * T + 4 * R
        f += 2.0 * R * T * V * D
    if op in ("loss_grad", "tied"):
        b += (R * T * D + R * V * D) * size[c["grad"]]
        f += 4.0 * R * T * V * D
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------------------------ 64 bits
def _table_sums(s, R, V, D):
    """Sums of the tokens' gradients by row, in 64 bits, one replica at a time: a product with the tokens' indicator matrix
    would be dense, so rows are added at their places."""
    full = torch.zeros((R, V, D), device="cuda", dtype=torch.float64)
    for r in range(R):
        t = s["tokens"][r].long()
        keep = torch.nonzero((t >= 0) & (t < V))[:, 0]
        full[r].index_put_((t[keep],), s["d_out"][r][keep].double() * s["scale"], accumulate=True)
    return full


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    R, V, D, op = c["R"], c["V"], c["D"], c["op"]
    if op == "embed":
        out = torch.zeros(s["out"].shape, device="cuda", dtype=torch.float64)
        for r in range(R):
            t = s["tokens"][r].long()
            keep = torch.nonzero((t >= 0) & (t < V))[:, 0]
            table = s["table"] if c["shared"] else s["table"][r]
            out[r, keep] = table[t[keep]].double() * s["scale"]
        return {"out": out}
    if op == "embed_grad":
        return {"d_table": _table_sums(s, R, V, D)}
    losses, each, dh = [], torch.zeros(s["targets"].shape, device="cuda", dtype=torch.float64), None
    dw = None
    if op != "loss":
        dh = torch.zeros(s["hidden"].shape, device="cuda", dtype=torch.float64)
        dw = _table_sums(s, R, V, D) if op == "tied" else torch.zeros((R, V, D), device="cuda", dtype=torch.float64)
    for r in range(R):
        y = s["targets"][r].long()
        keep = torch.nonzero((y >= 0) & (y < V))[:, 0]
        y = y[keep]
        w = (s["weight"] if c["shared"] else s["weight"][r]).double()
        h = s["hidden"][r][keep].double()
        z = h @ w.t()
        norm = torch.logsumexp(z, 1)
        each[r, keep] = norm - z[torch.arange(len(y), device="cuda"), y]
        losses.append(each[r].sum() / max(1, len(y)))
        if dh is not None and len(y):
            p = torch.exp(z.sub_(norm[:, None]))
            p[torch.arange(len(y), device="cuda"), y] -= 1.0
            p /= len(y)
            dh[r, keep] = p @ w
            dw[r] += p.t() @ h
    found = {"loss": torch.stack(losses), "token_loss": each}
    if dh is not None:
        found.update(d_hidden=dh, d_weight=dw)
    return found
