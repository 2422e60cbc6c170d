"""The operators at the two ends of a language model, as measurable cases.

What a training program calls between its tokens and the gradients that the optimizer step takes: the embedding of tokens with
its gradient, the layer norm in front of the head with its gradients, and the head itself -- the cross entropy over a large
vocabulary from the hidden states, in pieces of the vocabulary, with its gradients.  Batches, outputs and workspaces exist
before the call; a pass is the calls alone.  With `own` false the same operators are computed in elementary torch operations.

Sizes are those of the repository's own configurations (widths of 4096 and 8192 with vocabularies of 32,000 and 128,256;
the example's vocabulary of 4099 and width of 256) and generic ones around them.
"""
import math

import torch

own = False

DEV = "cuda:0"
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_EPS = 1e-5


def listed():
    return [
        # Scoring one token of a 7B-shaped model: the smallest call on a large head.
        dict(name="head-one", op="head", half="bf16", tokens=1, vocab=32000, width=4096, pad=0, masked=0.0, uneven=False,
             grad=False),
        # A step of the example's model with a loss scale: the launches decide.
        dict(name="head-tiny", op="head", half="fp16", tokens=37, vocab=4099, width=256, pad=0, masked=0.0, uneven=False,
             grad=True),
        # Scoring a batch on an odd vocabulary; rows that are not packed, a quarter of them prompts.
        dict(name="head-score-f16", op="head", half="fp16", tokens=777, vocab=50021, width=1000, pad=8, masked=0.25,
             uneven=True, grad=False),
        # A micro-batch of the 7B-shaped model.
        dict(name="head-32k", op="head", half="bf16", tokens=4096, vocab=32000, width=4096, pad=0, masked=0.0, uneven=False,
             grad=True),
        # One of the 70B-shaped model, the largest vocabulary and width; prompts and padding masked.
        dict(name="head-128k", op="head", half="bf16", tokens=4096, vocab=128256, width=8192, pad=0, masked=0.1,
             uneven=False, grad=True),
        # The token that a generating model has just chosen.
        dict(name="embed-one", op="embed", half="bf16", tokens=1, vocab=32000, width=4096, pad=0, scale=1.0),
        # A long context's tokens on the largest table, with the scaling by the root of the width.
        dict(name="embed-128k", op="embed", half="bf16", tokens=16384, vocab=128256, width=8192, pad=0, scale=90.5),
        # Gradient of an odd, small table in fp32 with rows that lie apart.
        dict(name="embed-grad-f32", op="embed_grad", half="fp32", tokens=3001, vocab=4099, width=257, pad=3, scale=16.0,
             add=False),
        # Gradient of the 7B-shaped model's tied table, added to what the head has left there.
        dict(name="embed-grad-32k", op="embed_grad", half="bf16", tokens=16384, vocab=32000, width=4096, pad=0, scale=1.0,
             add=True),
        # One generated token's norm.
        dict(name="norm-one", op="norm", half="bf16", rows=1, width=4096, pad=0, bias=True, grad=False),
        # Forward and backward, odd sizes in fp32, rows apart, no bias.
        dict(name="norm-odd-f32", op="norm", half="fp32", rows=3001, width=1003, pad=5, bias=False, grad=True),
        # Forward and backward on a long context of the 70B-shaped width.
        dict(name="norm-8k", op="norm", half="bf16", rows=16384, width=8192, pad=0, bias=True, grad=True),
    ]


def draw(rng):
    """One more case: heads of 1 to 4096 tokens on vocabularies of 1000 to 128,256 and widths of 64 to 8192; embeddings of 1 to
    16,384 tokens on the same tables; norms of 1 to 16,384 rows of 16 to 8192."""
    log = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))  # noqa: E731
    op = rng.choice(("head", "head", "embed", "embed_grad", "norm"))
    if op == "head":
        width = log(64, 8192)
        if rng.random() < 0.6:  # most models' widths are
            width = max(64, width // 64 * 64)
        return dict(op=op, half=rng.choice(("bf16", "bf16", "fp16")), tokens=log(1, 4096), vocab=log(1000, 128256), width=width,
                    pad=rng.choice((0, 0, 1, 8)), masked=rng.choice((0.0, 0.1, 0.5)), uneven=rng.random() < 0.3,
                    grad=rng.random() < 0.7)
    half = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if op == "norm":
        return dict(op=op, half=half, rows=log(1, 16384), width=log(16, 8192), pad=rng.choice((0, 0, 3, 8)),
                    bias=rng.random() < 0.7, grad=rng.random() < 0.7)
    width = log(16, 8192 if half != "fp32" else 4096)
    if rng.random() < 0.6:
        width = max(16, width // 16 * 16)
    case = dict(op=op, half=half, tokens=log(1, 16384), vocab=log(1000, 128256), width=width, pad=rng.choice((0, 0, 1, 8)),
                scale=rng.choice((1.0, round(math.sqrt(width), 3))))
    if op == "embed_grad":
        case["add"] = rng.random() < 0.5
        case["vocab"] = max(1000, min(case["vocab"], int(1.6e8 / width)))
    return case


class _State:
    pass


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(n, width, pad, dtype, gen, std=1.0):
    """n rows of normal values, `pad` elements of other values between them."""
    return torch.empty(n, width + pad, dtype=dtype, device=DEV).normal_(0, std, generator=gen)[:, :width]


def _empty(n, width, pad, dtype):
    return torch.zeros(n, width + pad, dtype=dtype, device=DEV)[:, :width]


def _loss_scale(case):
    return 1024.0 if case["half"] == "fp16" else 1.0


def _token_ids(n, vocab, gen):
    """Frequent and rare tokens as in text (the k-th most frequent about 1/k as often as the first), spread over the table."""
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    rank = (u * math.log(vocab)).exp().long().sub_(1).clamp_(0, vocab - 1)
    step = next(k for k in range(7919, 7919 + vocab) if math.gcd(k, vocab) == 1)
    return rank * step % vocab


def _head_inputs(case, seed):
    gen, s = _gen(seed), _State()
    n, v, w, t = case["tokens"], case["vocab"], case["width"], _TYPES[case["half"]]
    s.weight = _rows(v, w, case["pad"], t, gen, 0.02)
    s.targets = _token_ids(n, v, gen)
    # hidden states that lean towards their targets, some more than others
    lean = torch.rand(n, generator=gen, device=DEV).mul_(12.0 / (4e-4 * w))
    s.hidden = _empty(n, w, case["pad"], t)
    s.hidden.copy_(torch.randn(n, w, generator=gen, device=DEV) + lean[:, None] * s.weight[s.targets].float())
    off = int(case["masked"] * n)
    s.weights = torch.full((n,), 1.0 / max(1, n - off), device=DEV)
    if case["uneven"]:
        s.weights.mul_(torch.rand(n, generator=gen, device=DEV).add_(0.5))
    s.weights[torch.randperm(n, generator=gen, device=DEV)[:off]] = 0.0
    return s


def prepare(case, seed):
    if own:
        from paper_2512_03644_amd import binding as ff
    op, t = case["op"], _TYPES[case["half"]]
    if op == "head":
        s = _head_inputs(case, seed)
        s.case, s.op, s.loss_scale = case, op, _loss_scale(case)
        s.logp = torch.zeros(case["tokens"], device=DEV)
        s.dhidden = s.dweight = None
        if case["grad"]:
            s.dhidden = torch.zeros(case["tokens"], case["width"], dtype=t, device=DEV)
            s.dweight = torch.zeros(case["vocab"], case["width"], dtype=t, device=DEV)
        if own:
            s.stats = ff.HeadStats(DEV)
            s.workspace = ff.alloc_head_workspace(
                ff.head_batch(s.hidden, s.weight, s.targets, s.weights, s.loss_scale), DEV, grad=case["grad"])
        return s
    s, gen = _State(), _gen(seed)
    s.case, s.op = case, op
    if op == "norm":
        n, w = case["rows"], case["width"]
        s.x = _rows(n, w, case["pad"], t, gen, 1.5)
        # a few features that are much larger than the others, as in the residual stream
        s.x[:, torch.randint(0, w, (max(1, w // 500),), generator=gen, device=DEV)] += 20.0
        s.weight = torch.randn(w, generator=gen, device=DEV).mul_(0.1).add_(1.0).to(t)
        s.bias = torch.randn(w, generator=gen, device=DEV).mul_(0.1).to(t) if case["bias"] else None
        s.y = torch.zeros(n, w, dtype=t, device=DEV)
        s.mean, s.rstd = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        if case["grad"]:
            s.dy = _rows(n, w, case["pad"], t, gen, 1e-2)
            s.dx = torch.zeros(n, w, dtype=t, device=DEV)
            s.dweight = torch.zeros(w, dtype=t, device=DEV)
            s.dbias = torch.zeros(w, dtype=t, device=DEV) if case["bias"] else None
            if own:
                s.workspace = ff.alloc_norm_workspace(n, w, DEV)
        return s
    n, v, w = case["tokens"], case["vocab"], case["width"]
    s.ids = _token_ids(n, v, gen)
    s.ids[torch.rand(n, generator=gen, device=DEV) < (0.05 if n > 1 else 0.0)] = -1  # padding
    if op == "embed":
        s.table = _rows(v, w, case["pad"], t, gen, 0.02)
        s.out = torch.zeros(n, w, dtype=t, device=DEV)
        return s
    s.dout = _rows(n, w, case["pad"], t, gen, 1e-3 * _loss_scale(case))
    s.dtable = _empty(v, w, case["pad"], t)
    if case["add"]:
        s.dtable.normal_(0, 1e-3 * _loss_scale(case), generator=gen)
    if own:
        s.workspace = ff.alloc_embed_workspace(n, v, w, DEV)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2512_03644_amd import binding as ff
    case = s.case
    if s.op == "head":
        batch = ff.head_batch(s.hidden, s.weight, s.targets, s.weights, s.loss_scale)
        ff.ff_head_loss(batch, s.logp, s.stats, s.workspace, s.dhidden, s.dweight)
        out = {"loss": s.stats.loss, "logp": s.logp, "n_tokens": s.stats.n_tokens}
        if case["grad"]:
            out.update(dhidden=s.dhidden, dweight=s.dweight)
        return out
    if s.op == "embed":
        ff.ff_embed(s.table, s.ids, s.out, case["scale"])
        return {"out": s.out}
    if s.op == "embed_grad":
        ff.ff_embed_grad(s.dout, s.ids, s.dtable, s.workspace, case["scale"], add=case["add"])
        return {"dtable": s.dtable}
    ff.ff_layer_norm(s.x, s.weight, s.bias, s.y, s.mean, s.rstd, _EPS)
    out = {"y": s.y, "mean": s.mean, "rstd": s.rstd}
    if case["grad"]:
        ff.ff_layer_norm_grad(s.x, s.weight, s.mean, s.rstd, s.dy, s.dx, s.dweight, s.dbias, s.workspace)
        out.update(dx=s.dx, dweight=s.dweight)
        if s.dbias is not None:
            out["dbias"] = s.dbias
    return out


# ---- plain forms -------------------------------------------------------------------------------

def _plain_head(s):
    """Products and exponentials in 32 bits; sums over the vocabulary and what hangs on them in 64."""
    w = s.weights.double()
    used = w != 0
    z = s.hidden.float() @ s.weight.float().t()
    y = s.targets[:, None]
    m = z.amax(1, keepdim=True)
    picked = (z.gather(1, y) - m)[:, 0].double()
    e = z.sub_(m).exp_()
    total = e.sum(1, dtype=torch.float64)
    logp = picked - total.log()
    zero = torch.zeros_like(logp)
    out = {"loss": -torch.where(used, w * logp, zero).sum().float(), "logp": torch.where(used, logp, zero).float(),
           "n_tokens": used.sum()}
    if s.dhidden is not None:
        c = w * s.loss_scale
        g = e.mul_((c / total).float()[:, None]).scatter_(1, y, (c * torch.expm1(logp)).float()[:, None])
        out["dhidden"] = (g @ s.weight.float()).to(s.hidden.dtype)
        out["dweight"] = (g.t() @ s.hidden.float()).to(s.hidden.dtype)
    return out


def _plain_norm(s):
    x = s.x.float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = (x.square().mean(1) + _EPS).rsqrt()
    x = x * rstd[:, None]
    wide = s.weight.float()
    y = x * wide
    if s.bias is not None:
        y = y + s.bias.float()
    out = {"y": y.to(s.x.dtype), "mean": mean, "rstd": rstd}
    if s.case["grad"]:
        dy = s.dy.float()
        g = dy * wide
        dx = g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True)
        out["dx"] = (dx * rstd[:, None]).to(s.x.dtype)
        out["dweight"] = (dy * x).sum(0).to(s.x.dtype)
        if s.bias is not None:
            out["dbias"] = dy.sum(0).to(s.x.dtype)
    return out


def _run_plain(s):
    case = s.case
    if s.op == "head":
        return _plain_head(s)
    if s.op == "norm":
        return _plain_norm(s)
    inside = s.ids >= 0
    at = torch.where(inside, s.ids, 0)
    if s.op == "embed":
        s.out.copy_(torch.where(inside[:, None], s.table[at].float() * case["scale"], 0.0))
        return {"out": s.out}
    rows = torch.where(inside[:, None], s.dout.float() * case["scale"], 0.0)
    wide = s.dtable.float() if case["add"] else torch.zeros(s.dtable.shape, device=DEV)
    s.dtable.copy_(wide.index_add_(0, at, rows))
    return {"dtable": s.dtable}


# ---- what is known about a case ------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once.  The head's products: one for the logits and, with gradients, one
    for each of them; masked tokens take none.  Of an embedding's table only the rows that tokens ask for are counted,
    as if no two asked for the same; a gradient that is not added to anything is written whole."""
    item = 4 if case["half"] == "fp32" else 2
    if case["op"] == "head":
        n, v, w = case["tokens"], case["vocab"], case["width"]
        used = n - int(case["masked"] * n)
        moved = item * (v * w + used * w) + 16 * n
        if case["grad"]:
            moved += item * (v * w + n * w)
        return {"bytes": moved, "flops": (6 if case["grad"] else 2) * used * v * w}
    if case["op"] == "norm":
        n, w = case["rows"], case["width"]
        return {"bytes": item * n * w * (5 if case["grad"] else 2) + 16 * n + 4 * item * w,
                "flops": (19 if case["grad"] else 7) * n * w}
    n, v, w = case["tokens"], case["vocab"], case["width"]
    if case["op"] == "embed":
        return {"bytes": 2 * item * n * w + 8 * n, "flops": n * w}
    rows = min(n, v)
    return {"bytes": item * w * (n + (2 * rows if case["add"] else v)) + 8 * n, "flops": 2 * n * w}


def exact(case, seed):
    """The definitions in float64 from the same inputs."""
    global own
    if case["op"] == "head":
        return _exact_head(case, seed)
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "embed":
        out = torch.zeros(s.out.shape, dtype=torch.float64, device=DEV)
        for k in range(0, s.ids.numel(), 4096):
            ids = s.ids[k:k + 4096]
            on = (ids >= 0).nonzero()[:, 0]
            out[k + on] = s.table.index_select(0, ids[on]).double() * case["scale"]
        return {"out": out}
    order = torch.argsort(s.ids, stable=True)
    ids, counts = torch.unique_consecutive(s.ids[order], return_counts=True)
    sums = s.dout[order].double()
    # a run's sum is the difference of the running sums at its ends, within blocks of columns
    total = torch.cat([torch.zeros(1, sums.shape[1], dtype=torch.float64, device=DEV), sums.cumsum(0)])
    ends = counts.cumsum(0)
    runs = (total[ends] - total[ends - counts]) * case["scale"]
    out = s.dtable.double() if case["add"] else torch.zeros(s.dtable.shape, dtype=torch.float64, device=DEV)
    real = ids >= 0
    out[ids[real]] += runs[real]
    return {"dtable": out}


def _exact_head(case, seed):
    s = _head_inputs(case, seed)
    n, v = case["tokens"], case["vocab"]
    table = s.weight.double()
    loss, logps = 0.0, []
    dhidden, dweight = [], torch.zeros(table.shape, dtype=torch.float64, device=DEV) if case["grad"] else None
    for a in range(0, n, 1024):
        part = slice(a, a + 1024)
        h, y, w = s.hidden[part].double(), s.targets[part], s.weights[part].double()
        probs = torch.log_softmax(h @ table.t(), dim=1)
        row = torch.arange(y.numel(), device=DEV)
        logp = probs[row, y] * (w != 0)
        loss -= float((w * logp).sum())
        logps.append(logp)
        if case["grad"]:
            g = probs.exp_()
            g[row, y] = torch.expm1(logp)
            g *= (w * _loss_scale(case))[:, None]
            dhidden.append(g @ table)
            dweight += g.t() @ h
    out = {"loss": torch.tensor(loss, dtype=torch.float64), "logp": torch.cat(logps), "n_tokens": None}
    if case["grad"]:
        out.update(dhidden=torch.cat(dhidden), dweight=dweight)
    return out


def _exact_norm(s):
    case, parts = s.case, {k: [] for k in ("y", "mean", "rstd", "dx")}
    n, w = s.x.shape
    weight = s.weight.double()
    dweight, dbias = (torch.zeros(w, dtype=torch.float64, device=DEV) for _ in range(2))
    for a in range(0, n, 2048):
        x = s.x[a:a + 2048].double()
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        rstd = 1.0 / (var + _EPS).sqrt()
        normed = (x - mean) * rstd
        parts["y"].append(torch.addcmul(s.bias.double() if case["bias"] else torch.zeros_like(weight), normed, weight))
        parts["mean"].append(mean[:, 0])
        parts["rstd"].append(rstd[:, 0])
        if case["grad"]:
            dy = s.dy[a:a + 2048].double()
            dweight += torch.einsum("ij,ij->j", dy, normed)
            dbias += dy.sum(0)
            g = dy * weight
            inner = (g * normed).sum(1, keepdim=True)
            parts["dx"].append((w * g - g.sum(1, keepdim=True) - normed * inner) * rstd / w)
    out = {k: torch.cat(v) for k, v in parts.items() if v}
    if case["grad"]:
        out["dweight"] = dweight
        if case["bias"]:
            out["dbias"] = dbias
    return out
