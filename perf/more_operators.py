"""Cases for what a training loop of replicas does around its loss and before its update.

Beside the tied table's lookup and mean loss, a decoder's tokens are asked for more than a mean, and gradients are
measured before the update takes them:

* ``scores``       of every token's hidden state against the table: the log probability of the given token, the entropy of
                   the distribution, its normaliser (log sum exp) and the best alternatives with their log probabilities;
* ``scores_grad``  gradients of hidden states and table for given gradients of log probabilities and entropies;
* ``norm``         every replica's global gradient norm over a list of tensors;
* ``clip_step``    the optimizer's update with gradients clipped to a largest norm, replica by replica.

A given token outside 0 .. V-1 is padding: its values are 0, its alternatives -1, and it has no gradient.  Alternatives are
ordered by their logits, equal ones by their ids.
Shapes: given tokens [R, T]; table [R, V, D] ([V, D] when all replicas share it); hidden [R, T, D]; parameters, moments and
gradients [R, P] with the tensors of the list at multiples of ``align`` elements.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_VOCAB = 50257          # the vocabulary of this repository's decoder lists
_MARGIN = 16            # candidates behind the wanted ones whose order is looked at in 64 bits
_ALPHA, _RATE, _DECAY, _B1, _B2, _EPS = 1.0 / 9.0, 3e-4, 0.01, 0.9, 0.999, 1e-8


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one sequence, as when a model is sampled and asked for its best alternatives: latency
        dict(name="scores_one_token", op="scores", R=1, T=1, V=_VOCAB, D=768, top=20, given=False, shared=False),
        # the next tokens of a batch of sequences
        dict(name="scores_batch", op="scores", R=1, T=48, V=_VOCAB, D=1024, top=8, given=False, shared=False),
        # log probabilities and entropies of a small ragged model's tokens, with alternatives
        dict(name="scores_ragged", op="scores", R=3, T=777, V=4099, D=520, top=5, given=True, shared=False),
        # evaluation of eight replicas' tokens against the averaged table (350 M list)
        dict(name="scores_eval_350m", op="scores", R=8, T=2048, V=_VOCAB, D=1024, top=8, given=True, shared=True),
        # a small ragged model with fp32 gradients
        dict(name="scores_grad_small", op="scores_grad", R=3, T=129, V=4099, D=520, grad="f32", shared=False),
        # a training step on weighted tokens with an entropy term, sixteen replicas of the 125 M list
        dict(name="scores_grad_125m", op="scores_grad", R=16, T=1024, V=_VOCAB, D=768, grad="bf16", shared=False),
        # the same for eight replicas of the 1.3 B list
        dict(name="scores_grad_1p3b", op="scores_grad", R=8, T=2048, V=_VOCAB, D=2048, grad="bf16", shared=False),
        # a few small tensors that start at any element: latency
        dict(name="norm_small", op="norm", R=2, layers=0, width=300, vocab=0, align=1, grad="f32", mean=False),
        # four replicas of the 350 M list
        dict(name="norm_350m", op="norm", R=4, layers=24, width=1024, vocab=_VOCAB, align=8, grad="bf16", mean=False),
        # the norm of the replicas' mean gradient, fp32 (125 M list)
        dict(name="norm_mean_125m", op="norm", R=4, layers=12, width=768, vocab=_VOCAB, align=8, grad="f32", mean=True),
        # a small model whose tensors start at any element, plain SGD
        dict(name="clip_step_small", op="clip_step", R=3, layers=1, width=129, vocab=999, align=1, grad="f32", mean=False, opt="sgd",
             converge=False),
        # eight replicas of the 125 M list, averaged after the update
        dict(name="clip_step_125m", op="clip_step", R=8, layers=12, width=768, vocab=_VOCAB, align=8, grad="bf16", mean=False, opt="adamw",
             converge=True),
    ]


_TABLE_MAX = 8 * _VOCAB * 2048          # elements of the largest listed table
_LOGITS_MAX = 8 * 2048 * _VOCAB         # logits of the largest listed batch
_WORK_MAX = _LOGITS_MAX * 2048
_LIST_MAX = 8 * 124_439_808             # parameters of the largest listed update


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scores", "scores", "scores_grad", "norm", "clip_step"])
    if op in ("scores", "scores_grad"):
        while True:
            R, T = rng.randint(1, 16), _log_int(rng, 1, 8192)
            V, D = _log_int(rng, 64, 60000), _log_int(rng, 8, 2048)
            if rng.random() < 0.5:
                D = max(8, D // 64 * 64)
            if R * V * D <= _TABLE_MAX and R * T * V <= _LOGITS_MAX and R * T * V * D <= _WORK_MAX / 4 and R * T <= 16384:
                break
        c = dict(op=op, R=R, T=T, V=V, D=D, shared=rng.random() < 0.3)
        if op == "scores":
            c.update(top=rng.choice([0, 1, rng.randint(2, 20)]), given=rng.random() < 0.7)
        else:
            c.update(grad=rng.choice(["bf16", "bf16", "f32"]))
        return c
    while True:
        c = dict(op=op, R=rng.randint(1, 16), layers=rng.randint(0, 24), width=_log_int(rng, 24, 1280), vocab=_log_int(rng, 100, _VOCAB),
                 align=rng.choice([1, 4, 8, 8]), grad=rng.choice(["f32", "bf16"]), mean=rng.random() < 0.3)
        if c["R"] * sum(_numels(c)) <= _LIST_MAX:
            break
    if op == "clip_step":
        c.update(opt=rng.choice(["adamw", "adamw", "sgd"]), converge=rng.random() < 0.5)
    return c


def _numels(c):
    """Tensor sizes of a decoder with a tied table (12 a layer and four); without layers, a few odd ones."""
    d, v = c["width"], c["vocab"]
    if not c["layers"]:
        return [d, 1, 3 * d + 1, d * d, 7, d * 7]
    layer = [d, d, d * 3 * d, 3 * d, d * d, d, d, d, d * 4 * d, 4 * d, 4 * d * d, d]
    return [v * d, 1024 * d] + layer * c["layers"] + [d, d]


def _layout(c):
    """Elements of one replica, and the tensors' (offset, size)."""
    places, at = [], 0
    for n in _numels(c):
        places.append((at, n))
        at += -(-n // c["align"]) * c["align"]
    return at, places


# ------------------------------------------------------------------------------------------------ inputs
def _ids(gen, R, T, V, pad):
    """Tokens whose frequencies fall like 1 / rank, as words' do; the end of every longer sequence is padding."""
    u = torch.rand((R, T), generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1).int()
    if T > 8:
        length = T - (torch.rand((R, 1), generator=gen, device="cuda") * 0.2 * T).long()
        ids = torch.where(torch.arange(T, device="cuda") < length, ids, pad)
    return ids.contiguous()


def _prepare_tokens(c, gen, s):
    R, T, V, D = c["R"], c["T"], c["V"], c["D"]
    some = lambda dt, *more: torch.zeros((R, T) + more, device="cuda", dtype=dt)  # noqa: E731
    s["weight"] = (torch.randn((V, D) if c["shared"] else (R, V, D), generator=gen, device="cuda") * 0.02).bfloat16()
    ids = _ids(gen, R, T, V, -100)
    # hidden states of a model that has learnt something: each leans towards its token's row by some amount
    at = ids.long().clamp(min=0)
    rows = s["weight"][at] if c["shared"] else torch.stack([s["weight"][r][at[r]] for r in range(R)])
    lean = torch.rand((R, T, 1), generator=gen, device="cuda") * (200.0 / math.sqrt(D))
    s["hidden"] = (torch.randn((R, T, D), generator=gen, device="cuda") + lean * rows.float()).bfloat16()
    given = c["op"] == "scores_grad" or c["given"]
    s["targets"] = ids if given else None
    s["logprob"] = some(torch.float32) if given else None
    s["entropy"], s["lse"] = some(torch.float32), some(torch.float32)
    if c["op"] == "scores":
        top = min(c["top"], V)
        s["top_ids"] = some(torch.int32, top) if top else None
        s["top_logprob"] = some(torch.float32, top) if top else None
        return
    # what the forward call left, and the gradients that the rest of the loss sends back: an advantage for every token's log
    # probability and a bonus for its entropy
    for r in range(R):
        z = torch.matmul(s["hidden"][r].float(), (s["weight"] if c["shared"] else s["weight"][r]).float().t())
        lse = torch.logsumexp(z, 1)
        z.sub_(lse[:, None])
        found = (lse, -(z.exp() * z).sum(1), torch.gather(z, 1, at[r][:, None])[:, 0])
        for name, value in zip(("lse", "entropy", "logprob"), found):
            s[name][r] = torch.where(ids[r] >= 0, value, 0.0)
    s["d_logprob"] = torch.randn((R, T), generator=gen, device="cuda") / T
    s["d_entropy"] = torch.rand((R, T), generator=gen, device="cuda") * (0.1 / T)
    s["d_hidden"] = torch.empty((R, T, D), device="cuda", dtype=_DT[c["grad"]])
    s["d_weight"] = torch.empty((R, V, D), device="cuda", dtype=_DT[c["grad"]])


def _prepare_list(c, gen, s):
    R = c["R"]
    P, s["places"] = _layout(c)
    # gradients of replicas that differ in size: norms on both sides of the largest allowed one
    size = torch.exp(torch.rand((R, 1), generator=gen, device="cuda") * 2.4 - 1.2) / math.sqrt(P)
    s["grad"] = torch.empty((R, P), device="cuda", dtype=_DT[c["grad"]])
    s["param"] = torch.empty((R, P), device="cuda", dtype=torch.float32)
    adam = c["op"] == "clip_step" and c["opt"] == "adamw"
    if adam:
        s["exp_avg"], s["exp_avg_sq"] = torch.empty_like(s["param"]), torch.empty_like(s["param"])
    for r in range(R):
        s["grad"][r] = torch.randn(P, generator=gen, device="cuda") * size[r]
        if c["op"] == "clip_step":
            s["param"][r] = torch.randn(P, generator=gen, device="cuda") * 0.02
        if adam:
            s["exp_avg"][r] = torch.randn(P, generator=gen, device="cuda") * size[r] * 0.3
            s["exp_avg_sq"][r] = (torch.randn(P, generator=gen, device="cuda") * size[r]).square_()
    for (at, n), (end, _) in zip(s["places"], s["places"][1:] + [(P, 0)]):
        for name in ("grad", "param", "exp_avg", "exp_avg_sq"):
            if name in s:
                s[name][:, at + n:end] = 0
    s["norms"] = torch.zeros((R,), device="cuda", dtype=torch.float32)
    s["max_norm"], s["t"] = 0.75, 0


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)
    s = dict(case=case)
    if case["op"] in ("scores", "scores_grad"):
        _prepare_tokens(case, gen, s)
    else:
        _prepare_list(case, gen, s)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _rows_of(weight, ids):
    """[R, T, C, D]: the table's rows of ids [R, T, C]."""
    if weight.dim() == 2:
        return weight[ids]
    return weight[torch.arange(ids.shape[0], device="cuda")[:, None, None], ids]


def _scores_plain(s):
    h, w, V = s["hidden"], s["weight"], s["case"]["V"]
    z = torch.matmul(h.float(), w.float().transpose(-1, -2))
    best = z.amax(-1, keepdim=True)
    e = torch.exp(z - best)
    total = e.sum(-1, keepdim=True)
    lse = (best + torch.log(total))[..., 0]
    found = {"lse": lse, "entropy": torch.log(total)[..., 0] - (e.mul_(z - best).sum(-1) / total[..., 0])}
    some = torch.ones_like(lse, dtype=torch.bool)
    if s["targets"] is not None:
        y = s["targets"].long()
        some = (y >= 0) & (y < V)
        found["logprob"] = torch.gather(z, 2, torch.where(some, y, 0)[..., None])[..., 0] - lse
    found = {k: torch.where(some, v, 0.0) for k, v in found.items()}
    if s["top_ids"] is not None:
        n = s["top_ids"].shape[-1]
        ids = torch.topk(z, min(V, n + _MARGIN), dim=-1).indices.sort(-1).values
        exactly = (_rows_of(w, ids).double() * h.double()[:, :, None]).sum(-1)      # in 64 bits: values next to one another
        ids = torch.gather(ids, 2, torch.sort(exactly, dim=-1, descending=True, stable=True).indices[..., :n])
        found["top_ids"] = torch.where(some[..., None], ids, -1).int()
        found["top_logprob"] = torch.where(some[..., None], torch.gather(z, 2, ids) - lse[..., None], 0.0)
    return found


def _scores_grad_plain(s):
    h, w, V = s["hidden"].float(), s["weight"].float(), s["case"]["V"]
    y = s["targets"].long()
    some = (y >= 0) & (y < V)
    a, b = torch.where(some, s["d_logprob"], 0.0)[..., None], torch.where(some, s["d_entropy"], 0.0)[..., None]
    z = torch.matmul(h, w.transpose(-1, -2))
    z.sub_(torch.where(some, s["lse"], 1e30)[..., None])              # the logarithms of the probabilities
    g = torch.exp(z)
    z.add_(s["entropy"][..., None]).mul_(b).add_(a)
    g.mul_(z).neg_()
    del z
    g.scatter_add_(2, torch.where(some, y, 0)[..., None], a)
    g.masked_fill_(~some[..., None], 0.0)
    return {"d_hidden": torch.matmul(g, w).to(s["d_hidden"].dtype),
            "d_weight": torch.matmul(g.transpose(1, 2), torch.where(some[..., None], h, 0.0)).to(s["d_weight"].dtype)}


def _gradients(s):
    g = s["grad"].float()
    return g.mean(0, keepdim=True) if s["case"]["mean"] else g


def _norms_plain(s, g):
    return g.square().sum(1, dtype=torch.float64).sqrt().expand(s["norms"].shape)


def _rates(R):
    half = (R - 1) / 2.0
    return _RATE * (1.0 + _ALPHA * (torch.arange(R, dtype=torch.float64) - half) / max(half, 0.5))


def _clip_step_plain(s):
    c, p = s["case"], s["param"]
    s["t"] += 1
    g = _gradients(s)
    norms = _norms_plain(s, g)
    clip = torch.where(norms > s["max_norm"], s["max_norm"] / norms, 1.0).float()[:, None]
    rate = _rates(c["R"]).to(torch.float32).cuda()[:, None]
    if c["mean"]:
        g = g.expand(p.shape)
    g = g * clip
    if c["opt"] == "sgd":
        p.sub_(rate * (g + _DECAY * p))
    else:
        m, v = s["exp_avg"], s["exp_avg_sq"]
        m.add_((g - m).mul_(1.0 - _B1))
        v.add_(g.square_().sub_(v).mul_(1.0 - _B2))
        del g
        step = (v.sqrt().mul_(1.0 / math.sqrt(1.0 - _B2 ** s["t"])).add_(_EPS)).reciprocal_().mul_(m)
        p.sub_(p * (rate * _DECAY)).sub_(step.mul_(rate / (1.0 - _B1 ** s["t"])))
    if c["converge"]:
        p.copy_(p.mean(0, keepdim=True).expand(p.shape))
    return norms.float()


def _state(s):
    return {k: s[k] for k in ("param", "exp_avg", "exp_avg_sq") if k in s}


def _run_plain(s):
    op = s["case"]["op"]
    if op == "scores":
        return _scores_plain(s)
    if op == "scores_grad":
        return _scores_grad_plain(s)
    if op == "norm":
        return {"norms": _norms_plain(s, _gradients(s)).float()}
    return dict(_state(s), norms=_clip_step_plain(s))


# ------------------------------------------------------------------------------------------------ the framework's calls
def _workspace(s, need):
    """A workspace that the program keeps beside its inputs and gives to every call."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(16, need()), device="cuda", dtype=torch.uint8)
    return s["workspace"]


class _Handle:
    """The update's handle for a state's tensors, made once and kept."""

    def __init__(self, B, s):
        c, P = s["case"], s["param"].shape[1]
        self.B = B
        tensors = []
        for at, n in s["places"]:
            t = B.hdet_tensor(numel=n, param_stride=P, grad_stride=P, state_stride=P)
            t.param, t.grad = s["param"].data_ptr() + 4 * at, s["grad"].data_ptr() + s["grad"].element_size() * at
            if "exp_avg" in s:
                t.exp_avg, t.exp_avg_sq = s["exp_avg"].data_ptr() + 4 * at, s["exp_avg_sq"].data_ptr() + 4 * at
            tensors.append(t)
        adam = "exp_avg" in s
        self.h = B.hdet_create(B.hdet_config(
            n_replicas=c["R"], n_groups=1, optimizer=B.HDET_OPT_ADAMW if adam else B.HDET_OPT_SGD,
            grad_dtype=B.HDET_DTYPE_BF16 if c["grad"] == "bf16" else B.HDET_DTYPE_F32, beta1=_B1, beta2=_B2, eps=_EPS, alpha_lr=_ALPHA,
            sync_interval=1 if c.get("converge") else 1 << 40, fuse_converge=1, device=s["param"].device.index,
            grad_mode=B.HDET_GRAD_REPLICA_MEAN if c["mean"] else B.HDET_GRAD_AS_GIVEN), tensors)
        B.hdet_set_schedule(self.h, B.make_schedule(B.HDET_SCHED_CONSTANT, 1 << 40, [_RATE], weight_decay=[_DECAY]))
        if c["op"] == "clip_step":
            B.hdet_set_clip(self.h, s["max_norm"], s["norms"])

    def __del__(self):
        torch.cuda.synchronize()
        self.B.hdet_destroy(self.h)


def _run_own(s):
    from paper_2604_24708_b200 import binding as B

    op, stream = s["case"]["op"], torch.cuda.current_stream().cuda_stream
    if op == "scores":
        h, w, y, ids = s["hidden"], s["weight"], s["targets"], s["top_ids"]
        ws = _workspace(s, lambda: B.hdet_token_scores_workspace(h, w, y, n_top=0 if ids is None else ids.shape[-1]))
        B.hdet_token_scores(h, w, y, ws, logprob=s["logprob"], entropy=s["entropy"], lse=s["lse"], top_ids=ids, top_logprob=s["top_logprob"],
                            stream=stream)
        return {k: s[k] for k in ("logprob", "entropy", "lse", "top_ids", "top_logprob") if s[k] is not None}
    if op == "scores_grad":
        h, w, y, dh, dw = s["hidden"], s["weight"], s["targets"], s["d_hidden"], s["d_weight"]
        ws = _workspace(s, lambda: B.hdet_token_scores_grad_workspace(h, w, y, d_hidden=dh, d_weight=dw))
        B.hdet_token_scores_grad(h, w, y, ws, lse=s["lse"], logprob=s["logprob"], entropy=s["entropy"], d_logprob=s["d_logprob"],
                                 d_entropy=s["d_entropy"], d_hidden=dh, d_weight=dw, stream=stream)
        return {"d_hidden": dh, "d_weight": dw}
    if "handle" not in s:
        s["handle"] = _Handle(B, s)
    if op == "norm":
        B.hdet_grad_norm(s["handle"].h, s["norms"], stream=stream)
        return {"norms": s["norms"]}
    B.hdet_step(s["handle"].h, stream=stream)
    return dict(_state(s), norms=s["norms"])


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    c, size = case, {"f32": 4, "bf16": 2}
    R, op = c["R"], c["op"]
    if op in ("scores", "scores_grad"):
        T, V, D = c["T"], c["V"], c["D"]
        b = R * T * D * 2 + (1 if c["shared"] else R) * V * D * 2 + 4 * R * T * (3 if op == "scores" else 6)
        f = 2.0 * R * T * V * D
        if op == "scores":
            b += 8 * R * T * min(c["top"], V)
        else:
            b += (R * T * D + R * V * D) * size[c["grad"]]
            f *= 3
        return {"bytes": float(b), "flops": f}
    n = R * sum(_numels(c))
    if op == "norm":
        return {"bytes": float(n * size[c["grad"]] + 4 * R), "flops": 2.0 * n}
    each = size[c["grad"]] + (24 if c["opt"] == "adamw" else 8)
    return {"bytes": float(n * each + 4 * R), "flops": 16.0 * n}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_scores(c, s):
    R, V = c["R"], c["V"]
    n = 0 if s["top_ids"] is None else s["top_ids"].shape[-1]
    found = {k: [] for k in ("lse", "entropy", "top_logprob") + (("logprob",) if s["targets"] is not None else ())}
    ids = []
    for r in range(R):
        w = (s["weight"] if c["shared"] else s["weight"][r]).double()
        z = s["hidden"][r].double() @ w.t()
        some = torch.ones(len(z), device="cuda", dtype=torch.bool)
        if s["targets"] is not None:
            y = s["targets"][r].long()
            some = (y >= 0) & (y < V)
            found["logprob"].append(torch.where(some, torch.log_softmax(z, 1)[torch.arange(len(z), device="cuda"), y.clamp(0, V - 1)], 0.0))
        norm = torch.logsumexp(z, 1)
        found["lse"].append(torch.where(some, norm, 0.0))
        if n:
            value, at = torch.sort(z, dim=1, descending=True, stable=True)
            ids.append(torch.where(some[:, None], at[:, :n], -1).int())
            found["top_logprob"].append(torch.where(some[:, None], value[:, :n] - norm[:, None], 0.0))
        z.sub_(norm[:, None])
        found["entropy"].append(torch.where(some, -(torch.exp(z) * z).sum(1), 0.0))
    found = {k: torch.stack(v) for k, v in found.items() if v}
    if n:
        found["top_ids"] = torch.stack(ids)
    return found


def _exact_scores_grad(c, s):
    dh = torch.zeros(s["hidden"].shape, device="cuda", dtype=torch.float64)
    dw = torch.zeros(s["d_weight"].shape, device="cuda", dtype=torch.float64)
    for r in range(c["R"]):
        y = s["targets"][r].long()
        keep = torch.nonzero((y >= 0) & (y < c["V"]))[:, 0]
        if not len(keep):
            continue
        w = (s["weight"] if c["shared"] else s["weight"][r]).double()
        h = s["hidden"][r][keep].double()
        lp = torch.log_softmax(h @ w.t(), 1)
        p = torch.exp(lp)
        entropy = -(p * lp).sum(1, keepdim=True)
        g = -p * (s["d_entropy"][r][keep].double()[:, None] * (lp + entropy))
        g -= p * s["d_logprob"][r][keep].double()[:, None]
        g[torch.arange(len(keep), device="cuda"), y[keep]] += s["d_logprob"][r][keep].double()
        dh[r, keep] = g @ w
        dw[r] = g.t() @ h
    return {"d_hidden": dh, "d_weight": dw}


def _exact_list(c, s):
    R = c["R"]
    mean = s["grad"].double().mean(0) if c["mean"] else None
    grad = lambda r: mean if mean is not None else s["grad"][r].double()  # noqa: E731
    norms = torch.stack([grad(r).square().sum().sqrt() for r in range(R)])
    if c["op"] == "norm":
        return {"norms": norms}
    rates = _rates(R).tolist()
    found = {k: torch.empty(v.shape, device="cuda", dtype=torch.float64) for k, v in _state(s).items()}
    for r in range(R):
        g = grad(r) * min(1.0, s["max_norm"] / float(norms[r]))
        p = s["param"][r].double()
        if c["opt"] == "sgd":
            p -= rates[r] * (g + _DECAY * p)
        else:
            m = _B1 * s["exp_avg"][r].double() + (1 - _B1) * g
            v = _B2 * s["exp_avg_sq"][r].double() + (1 - _B2) * g * g
            p = p * (1 - rates[r] * _DECAY) - rates[r] * (m / (1 - _B1)) / (torch.sqrt(v / (1 - _B2)) + _EPS)
            found["exp_avg"][r], found["exp_avg_sq"][r] = m, v
        found["param"][r] = p
    if c["converge"]:
        found["param"] = found["param"].mean(0, keepdim=True).expand(R, -1)
    return dict(found, norms=norms)


def exact(case, seed):
    s = prepare(case, seed)
    return {"scores": _exact_scores, "scores_grad": _exact_scores_grad}.get(case["op"], _exact_list)(case, s)
