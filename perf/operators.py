"""The operators around the optimizer step, as measurable cases.

What a training program calls between its model's output and the next snapshot: the policy loss
with its gradient, the norm of all gradients, their clipping, and the clipped AdamW step that writes
the snapshot in the same pass.  Plans, lists, buffers and inputs exist before the call; a pass is
the calls alone.  With `own` false the same operators are computed in elementary torch operations.

Sizes are those of the repository's own configurations (workloads.py: a small model's 64
parameters, one worker's share of a 7B- and of a 70B-shaped model, ragged lists whose tensors begin
anywhere, vocabularies of 32,000 and 128,256) and generic ones around them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
KiB, MiB = 1 << 10, 1 << 20
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

_7B = dict(layout="llama", layers=32, hidden=4096, ffn=11008, kv=4096, vocab=32000, dp=8)
_TINY = dict(layout="uniform", n=64, lo=1024, hi=65536)
_RAGGED = dict(layout="lognormal", mu=9.0, sigma=2.0)


def listed():
    return [
        # The gradients of a small model (or of a test job), 4 MB: the launch and one round of loads decide.
        dict(name="norm-tiny", op="norm", half="bf16", scale=1.0, **_TINY),
        # The gradients of one worker of the 8-way data-parallel 7B job, 1.7 GB.
        dict(name="norm-7b8", op="norm", half="bf16", scale=1.0, **_7B),
        # A flat buffer's 20,000 ragged gradients in two formats, most of them short, off every line.
        dict(name="norm-ragged", op="norm", half="mixed", scale=1.0, n=20000, **_RAGGED),
        # Clipping for an optimizer of the program's own: fp32 gradients of the small model ...
        dict(name="clip-tiny-f32", op="clip", half="fp32", scale=1.0, **_TINY),
        # ... and the 7B worker's.
        dict(name="clip-7b8", op="clip", half="bf16", scale=1.0, **_7B),
        # The small model's step: norm, clipped update and snapshot; first step of a run.
        dict(name="step-tiny", op="step", half="bf16", scale=1.0, step=1, chained=False,
             chunk=1 * MiB, **_TINY),
        # fp16 training with a loss scale on ragged parameter groups.
        dict(name="step-f16-ragged", op="step", half="fp16", scale=1024.0, step=40, chained=False,
             chunk=4 * MiB, n=2000, **_RAGGED),
        # The 7B worker's step with its state in the two alternating snapshots.
        dict(name="step-7b8-chained", op="step", half="bf16", scale=1.0, step=1000, chained=True,
             chunk=4 * MiB, **_7B),
        # One token: the smallest call on a vocabulary of 32,000.
        dict(name="policy-one", op="policy", half="bf16", tokens=1, vocab=32000, pad=0, beta=0.05,
             masked=0.0, grad=True),
        # Scoring alone, fp32 logits of an odd vocabulary in rows that are not packed.
        dict(name="policy-score-f32", op="policy", half="fp32", tokens=777, vocab=50021, pad=3,
             beta=0.0, masked=0.0, grad=False),
        # A micro-batch on a vocabulary of 32,000 with a reference policy; prompts and padding masked.
        dict(name="policy-32k", op="policy", half="bf16", tokens=4096, vocab=32000, pad=0, beta=0.05,
             masked=0.25, grad=True),
        # The 70B-shaped model's vocabulary: the largest rows, 1.05 GB of logits.
        dict(name="policy-128k", op="policy", half="bf16", tokens=4096, vocab=128256, pad=0,
             beta=0.05, masked=0.1, grad=True),
    ]


def draw(rng):
    """One more case: any operator; 1 MB to 1 GB of gradients in 1 to 10,000 tensors, 3 MB to 6 GB
    of state, 1 to 4096 tokens on vocabularies of 1000 to 130,000."""
    op = rng.choice(("norm", "clip", "step", "policy"))
    log = lambda lo, hi: math.exp(rng.uniform(math.log(lo), math.log(hi)))  # noqa: E731
    if op == "policy":
        vocab = int(log(1000, 130000))
        tokens = max(1, min(4096, int(log(1, 4096)), int(4e8 / vocab)))
        return dict(op=op, half=rng.choice(("bf16", "bf16", "fp16", "fp32")), tokens=tokens,
                    vocab=vocab, pad=rng.choice((0, 0, 1, 8)), beta=rng.choice((0.0, 0.05)),
                    masked=rng.choice((0.0, 0.1, 0.5)), grad=rng.random() < 0.75)
    c = dict(op=op)
    if op == "step":
        c["half"] = rng.choice(("bf16", "bf16", "fp16"))
        total = log(3e6, 6e9) / 14
        n = int(log(1, 2000))
        c.update(step=rng.choice((1, 10, 1000)), chained=rng.random() < 0.5,
                 chunk=1 << rng.randint(18, 23))
    else:
        c["half"] = rng.choice(("bf16", "bf16", "fp16", "fp32", "mixed"))
        total = log(1e6, 1e9) / 4
        n = int(log(1, 10000))
    c["scale"] = 1024.0 if c["half"] == "fp16" else 1.0
    n = max(1, min(n, int(total / 64)))
    mean = total / n
    if rng.random() < 0.5:
        c.update(layout="uniform", n=n, lo=max(1, int(0.25 * mean)),
                 hi=max(2, int(1.75 * mean)) + rng.randint(0, 15))
    else:
        sigma = rng.choice((1.0, 1.5, 2.0))
        c.update(layout="lognormal", n=n, sigma=sigma, mu=round(math.log(mean) - sigma * sigma / 2, 3))
    return c


# ---- layouts -----------------------------------------------------------------------------------

def _numels(case):
    """Element counts; they belong to the case, not to the seed."""
    if case["layout"] == "llama":
        h, f, kv, v, dp = (case[k] for k in ("hidden", "ffn", "kv", "vocab", "dp"))
        block = [h * h, h * kv, h * kv, h * h, h * f, h * f, f * h]
        return [x // dp for x in [v * h] + block * case["layers"] + [v * h]]
    rng = np.random.default_rng(case["n"])
    if case["layout"] == "uniform":
        return [int(x) for x in rng.integers(case["lo"], case["hi"], size=case["n"], endpoint=True)]
    most = 4 * MiB if case["n"] > 64 else 64 * MiB
    return [int(x) for x in np.clip(np.floor(rng.lognormal(case["mu"], case["sigma"], case["n"])),
                                    1, most)]


def _items(case, n):
    """Bytes per element of every gradient."""
    if case["half"] == "mixed":
        return [int(x) for x in np.where(np.random.default_rng(n + 1).random(n) < 0.5, 2, 4)]
    return [4 if case["half"] == "fp32" else 2] * n


def _carve(numels, items, ragged, salt, gen, std, types):
    """One allocation per element size, filled with normal values, and a tensor in it for every entry of
    numels: on 512-byte boundaries as an allocator places them or, ragged, at any multiple of the
    element size with gaps between, as a flat buffer holds them."""
    rng = np.random.default_rng(salt)
    gaps, mis = rng.integers(0, 5, len(numels)), rng.integers(0, 16, len(numels))
    pos, off = {s: 0 for s in types}, []
    for k, (n, s) in enumerate(zip(numels, items)):
        if ragged:
            at = (pos[s] + 15) // 16 * 16 + 16 * int(gaps[k]) + int(mis[k]) // s * s
        else:
            at = (pos[s] + 511) // 512 * 512
        off.append(at // s)
        pos[s] = at + n * s
    flat = {}
    for s, t in types.items():
        f = torch.empty(pos[s] // s + 16, dtype=t, device=DEV)
        flat[s] = f.normal_(0, std, generator=gen)
    return flat, [flat[s][o:o + n] for o, n, s in zip(off, numels, items)]


class _State:
    pass


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


_STD = 1e-3  # of a gradient's elements


def _grads(case, gen):
    ns = _numels(case)
    items = _items(case, len(ns))
    half = torch.bfloat16 if case["half"] == "mixed" else _TYPES[case["half"]]
    types = {s: torch.float32 if s == 4 else half for s in sorted(set(items))}
    return _carve(ns, items, case["layout"] == "lognormal", 25, gen, _STD * case["scale"], types)


def _max_norm(case):
    """Somewhat less than the norm of such gradients is about: clipping is at work."""
    return 0.6 * _STD * math.sqrt(sum(_numels(case)))


def _hparams(case):
    return dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=case["step"])


def _model_state(case, gen):
    """(flat allocations by name, [w16, master, m, v] of every group)."""
    ns = _numels(case)
    ragged = case["layout"] == "lognormal"
    flats, lists = {}, {}
    for salt, (name, std, item) in enumerate((("w16", 0.02, 2), ("master", 0.02, 4), ("m", 1e-3, 4),
                                              ("v", 1e-3, 4))):
        t = _TYPES[case["half"]] if item == 2 else torch.float32
        flat, lists[name] = _carve(ns, [item] * len(ns), ragged, 21 + salt, gen, std, {item: t})
        flats[name] = flat[item]
    flats["v"].square_()
    return flats, [[lists[name][k] for name in ("w16", "master", "m", "v")] for k in range(len(ns))]


def _payload(case):
    return 14 * sum(_numels(case))


# ---- inputs of the policy loss -------------------------------------------------------------------

_CLIP_LOW, _CLIP_HIGH = 0.2, 0.28


def _policy_inputs(case, seed):
    gen = _gen(seed)
    n, v = case["tokens"], case["vocab"]
    s = _State()
    rows = torch.empty(n, v + case["pad"], dtype=_TYPES[case["half"]], device=DEV)
    rows.normal_(0, 2.0, generator=gen)
    s.logits = rows[:, :v]
    s.targets = torch.randint(0, v, (n,), generator=gen, device=DEV)
    every = torch.arange(n, device=DEV)
    # tokens that the policy chose: likelier than most
    s.logits[every, s.targets] += torch.rand(n, generator=gen, device=DEV).mul_(12.0).to(rows.dtype)
    # every fourth row: a third of the vocabulary is ruled out
    keep = s.logits[every, s.targets].clone()
    lo = v // 3
    s.logits[3::4, lo:2 * lo] = -math.inf
    s.logits[every, s.targets] = keep
    n_off = int(case["masked"] * n)
    weights = torch.full((n,), 1.0 / max(1, n - n_off), device=DEV)
    weights[torch.randperm(n, generator=gen, device=DEV)[:n_off]] = 0.0
    s.weights = weights
    s.advantages = torch.randn(n, generator=gen, device=DEV)
    # the log-probabilities of the policy that made the tokens, and of the reference
    logp = torch.empty(n, dtype=torch.float64, device=DEV)
    for a in range(0, n, 1024):
        z = s.logits[a:a + 1024].float()
        m = z.amax(1, keepdim=True)
        lse = (z - m).exp_().sum(1, dtype=torch.float64).log() + m[:, 0].double()
        logp[a:a + 1024] = z.gather(1, s.targets[a:a + 1024, None])[:, 0].double() - lse
    ratio = torch.randn(n, generator=gen, device=DEV).double().mul_(0.2)
    # (whether a ratio within rounding of a border is clipped is nobody's to say)
    for border in (math.log(1 - _CLIP_LOW), math.log(1 + _CLIP_HIGH)):
        ratio = torch.where((ratio - border).abs() < 1e-4, ratio + 5e-4, ratio)
    s.old_logp = (logp - ratio).float()
    s.ref_logp = None
    if case["beta"]:
        s.ref_logp = (logp - 0.3 * torch.randn(n, generator=gen, device=DEV).double()).float()
    return s


def _loss_scale(case):
    return 1024.0 if case["half"] == "fp16" else 1.0


# ---- state -------------------------------------------------------------------------------------

def prepare(case, seed):
    if own:
        from paper_2512_03644_amd import binding as ff
    op = case["op"]
    if op == "policy":
        s = _policy_inputs(case, seed)
        s.case, s.op, n = case, op, case["tokens"]
        s.beta, s.loss_scale, s.dlogits = case["beta"], _loss_scale(case), None
        if case["grad"]:
            s.dlogits = torch.empty(n, case["vocab"], dtype=s.logits.dtype, device=DEV)
        s.logp = torch.empty(n, device=DEV)
        s.token_loss = torch.empty(n, device=DEV)
        if own:
            s.stats = ff.PolicyStats(DEV)
            s.workspace = ff.alloc_policy_workspace(n, case["vocab"], DEV)
        return s
    s = _State()
    s.case, s.op, gen = case, op, _gen(seed)
    flat, s.grads = _grads(case, gen)
    s.flat_grads = list(flat.values())
    s.max_norm, s.inv_scale = _max_norm(case), 1.0 / case["scale"]
    if own:
        s.list = ff.ff_grad_list(s.grads)
        s.stats, s.workspace = ff.GradStats(DEV), ff.alloc_grad_workspace(s.list, DEV)
    if op == "clip":  # the norm is known by now
        if own:
            ff.ff_grad_norm(s.list, s.stats, s.workspace, s.max_norm, s.inv_scale)
        else:
            s.factor, s.skip = _plain_norm(s)[2:]
            s.places = [_places(flat, s.grads) for flat in s.flat_grads]
    if op == "step":
        s.flats, groups = _model_state(case, gen)
        s.hp, s.chunk = _hparams(case), case["chunk"]
        s.tensors = [t for g in groups for t in g]
        n_chunks = -(-_payload(case) // s.chunk)
        s.chunks = torch.empty(n_chunks * s.chunk, dtype=torch.uint8, device=DEV)
        s.crcs = torch.empty(n_chunks, dtype=torch.int32, device=DEV)
        s.prev = None
        if case["chained"]:  # the snapshot of the step before this one
            s.prev = torch.zeros_like(s.chunks)
            _write_stream(s.tensors, s.prev)
        if own:
            kinds = [ff.FF_KIND_W16, ff.FF_KIND_MASTER, ff.FF_KIND_M, ff.FF_KIND_V] * len(groups)
            s.plan = ff.ff_snapshot_plan(s.tensors, s.chunk, 0, kinds, [k // 4 for k in range(len(kinds))])
        else:
            s.crc_tables = _crc_tables(s.chunk)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _step_outputs(s, norm):
    out = {"chunks": s.chunks.view(torch.int64), "crcs": s.crcs, "w16": s.flats["w16"], "norm": norm}
    if s.prev is None:
        out.update(master=s.flats["master"], m=s.flats["m"], v=s.flats["v"])
    return out


def _run_own(s):
    from paper_2512_03644_amd import binding as ff
    if s.op == "norm":
        ff.ff_grad_norm(s.list, s.stats, s.workspace, s.max_norm, s.inv_scale)
        return {"norm": s.stats.norm, "factor": s.stats.scale, "n_nonfinite": s.stats.n_nonfinite}
    if s.op == "clip":
        ff.ff_grad_clip(s.list, s.stats)
        return {"grads": s.flat_grads}
    if s.op == "step":
        ff.ff_grad_norm(s.list, s.stats, s.workspace, s.max_norm, s.inv_scale)
        ff.ff_adam_step_clipped(s.plan, s.grads, s.hp, s.stats, s.chunks, s.crcs, s.prev)
        return _step_outputs(s, s.stats.norm)
    batch = ff.policy_batch(s.logits, s.targets, s.old_logp, s.advantages, s.weights, s.ref_logp,
                            _CLIP_LOW, _CLIP_HIGH, s.beta, s.loss_scale)
    ff.ff_policy_loss(batch, s.logp, s.token_loss, s.stats, s.workspace, s.dlogits)
    out = {"loss": s.stats.loss, "kl": s.stats.kl, "logp": s.logp, "token_loss": s.token_loss,
           "n_tokens": s.stats.n_tokens, "n_clipped": s.stats.n_clipped}
    if s.dlogits is not None:
        out["dlogits"] = s.dlogits
    return out


# ---- plain forms -------------------------------------------------------------------------------

def _of_one_type(tensors):
    types = sorted({t.dtype for t in tensors}, key=str)
    return [torch.cat([t for t in tensors if t.dtype == k]) for k in types]


def _plain_norm(s):
    """norm, non-finite elements, what a gradient is multiplied by, whether the update is left out.
    Squares and their sum in 64 bits: a 16-bit element's square passes 32-bit floats at either end."""
    lists = _of_one_type(s.grads)
    total = torch.stack([g.double().square_().sum() for g in lists]).sum()
    bad = torch.stack([(~torch.isfinite(g)).sum() for g in lists]).sum()
    norm = total.sqrt() * s.inv_scale
    factor = torch.where(norm > s.max_norm, s.max_norm / norm, torch.ones_like(norm)) * s.inv_scale
    return norm, bad, factor.float(), bad > 0


def _places(flat, tensors):
    """Which elements of an allocation are its tensors' (the others lie in gaps)."""
    at = [((t.data_ptr() - flat.data_ptr()) // flat.element_size(), t.numel()) for t in tensors if t.dtype == flat.dtype]
    begin = torch.tensor([a for a, _ in at], device=DEV)
    end = torch.tensor([a + n for a, n in at], device=DEV)
    edges = torch.zeros(flat.numel(), dtype=torch.int8, device=DEV)
    edges[begin] += 1
    edges[end] -= 1
    return torch.cumsum(edges, 0, dtype=torch.int32) > 0


def _plain_clip(flat, inside, s):
    wide = flat.float()
    return flat.copy_(torch.where(inside & ~s.skip, wide * s.factor, wide))


def _write_stream(tensors, buf):
    n = sum(t.numel() * t.element_size() for t in tensors)
    torch.cat([t.view(torch.uint8) for t in tensors], out=buf[:n])
    buf[n:] = 0


def _plain_step(s):
    """Every operation of the update rounded to 32 bits by itself, in the order in which the step
    states it, so that its bytes have one value; then the stream and its checksums."""
    norm, _, factor, skip = _plain_norm(s)
    h = {k: np.float32(x) for k, x in s.hp.items()}
    lr, b1, b2, wd = (float(h[k]) for k in ("lr", "beta1", "beta2", "weight_decay"))
    t = float(s.hp["step"])
    c = lambda x: torch.tensor(np.float32(x), device=DEV)  # noqa: E731
    decay, omb1, omb2 = c(1.0 - lr * wd), c(1.0 - b1), c(1.0 - b2)
    size, bc2s = c(lr / (1.0 - b1 ** t)), c(math.sqrt(1.0 - b2 ** t))
    fb1, fb2, eps = c(b1), c(b2), c(s.hp["eps"])
    if s.prev is None:
        p, m, v = (torch.cat(s.tensors[k::4]) for k in (1, 2, 3))
    else:
        parts = s.prev[:_payload(s.case)].split([x.numel() * x.element_size() for x in s.tensors])
        p, m, v = (torch.cat(parts[k::4]).view(torch.float32) for k in (1, 2, 3))
    g = torch.cat(s.grads).float() * factor
    m1 = fb1 * m + omb1 * g
    v1 = fb2 * v + (omb2 * g) * g
    p1 = p * decay - size * (m1 / (v1.sqrt() / bc2s + eps))
    new = [torch.where(skip, old, x) for old, x in ((p, p1), (m, m1), (v, v1))]
    counts = [x.numel() for x in s.grads]
    new = [x.split(counts) for x in (new[0].to(s.tensors[0].dtype), *new)]
    torch._foreach_copy_(s.tensors[0::4], list(new[0]))
    if s.prev is None:
        torch._foreach_copy_([x for k in (1, 2, 3) for x in s.tensors[k::4]], [x for k in (1, 2, 3) for x in new[k]])
    _write_stream([x for group in zip(*new) for x in group], s.chunks)
    _plain_crcs(s.chunks, s.chunk, s.crc_tables, s.crcs)
    return norm


def _crc_tables(chunk):
    """Tables of what 4, 8, 16 ... zero bytes make of a CRC32C register, by its halves, and the checksum of
    a chunk of zeros."""
    u = np.arange(65536, dtype=np.uint32)
    halves = [u.copy(), u << np.uint32(16)]
    for t in halves:
        for _ in range(32):
            t[:] = (t >> np.uint32(1)) ^ np.where(t & np.uint32(1), np.uint32(0x82F63B78), np.uint32(0))
    tables, n, zeros = [], 4, np.array([0xFFFFFFFF], dtype=np.uint32)
    while n < chunk:
        tables.append(halves)
        lo, hi = halves
        step = lambda x: lo[x & 0xFFFF] ^ hi[x >> 16]  # noqa: E731
        halves = [step(lo), step(hi)]
        n *= 2
    tables.append(halves)
    zeros = tables[-1][0][zeros & 0xFFFF] ^ tables[-1][1][zeros >> 16]
    on_gpu = lambda t: torch.from_numpy(t.view(np.int32)).to(DEV)  # noqa: E731
    return [[on_gpu(t) for t in pair] for pair in tables], int(zeros.view(np.int32)[0])


def _plain_crcs(buf, chunk, tables, out):
    """CRC32C of every chunk: the registers of single words, joined in pairs up to the chunk."""
    levels, zeros = tables
    per = max(1, (256 * MiB) // chunk)
    for a in range(0, out.numel(), per):
        x = buf[a * chunk:(a + per) * chunk].view(torch.int32)
        shift = lambda x, t: t[0][(x & 0xFFFF).long()] ^ t[1][((x >> 16) & 0xFFFF).long()]  # noqa: E731
        x = shift(x, levels[0])
        for t in levels[:-1]:
            x = x.view(-1, 2)
            x = shift(x[:, 0], t) ^ x[:, 1]
        out[a:a + per] = ~(x.view(-1) ^ zeros)


def _plain_policy(s):
    """Sums over the vocabulary in 32 bits; what hangs on a token's log-probability, with the clipping's
    borders, in 64."""
    z = s.logits.to(torch.float32, copy=True)  # made the exponentials below
    w, adv = s.weights.double(), s.advantages.double()
    inside = (s.targets >= 0) & (s.targets < z.shape[1])
    y = torch.where(inside, s.targets, 0)[:, None]
    m = z.amax(1, keepdim=True)
    used = (w != 0) & inside & (m[:, 0] != -math.inf)
    picked = (z.gather(1, y) - m)[:, 0].double()
    e = z.sub_(m).exp_()
    total = e.sum(1, dtype=torch.float64)
    logp = picked - total.log()
    r = (logp - s.old_logp.double()).exp()
    kept, cut = r * adv, r.clamp(1 - _CLIP_LOW, 1 + _CLIP_HIGH) * adv
    clipped = (cut < kept) & used
    zero = torch.zeros_like(r)
    token, slope, kl = -torch.minimum(kept, cut), torch.where(clipped, zero, -kept), zero
    if s.ref_logp is not None:
        d = s.ref_logp.double() - logp
        kl = d.exp() - d - 1
        if s.beta:
            token, slope = token + s.beta * kl, slope + s.beta * (1 - d.exp())
    loss = torch.where(used, w * token, zero).sum()
    kl = torch.where(used, w * kl, zero).sum()
    out = {"loss": loss.float(), "kl": kl.float(), "logp": torch.where(used, logp, zero).float(),
           "token_loss": torch.where(used, token, zero).float(), "n_tokens": used.sum(), "n_clipped": clipped.sum()}
    if s.dlogits is not None:
        c = torch.where(used, w * slope * s.loss_scale, zero)
        g = e.mul_((-c / total).float()[:, None]).scatter_(1, y, (c * -torch.expm1(logp)).float()[:, None])
        out["dlogits"] = torch.where(used[:, None], g, 0.0).to(s.logits.dtype)
    return out


def _run_plain(s):
    if s.op == "norm":
        norm, bad, factor, _ = _plain_norm(s)
        return {"norm": norm, "factor": factor, "n_nonfinite": bad}
    if s.op == "clip":
        return {"grads": [_plain_clip(flat, own_places, s) for flat, own_places in zip(s.flat_grads, s.places)]}
    if s.op == "step":
        return _step_outputs(s, _plain_step(s))
    return _plain_policy(s)


# ---- what is known about a case ------------------------------------------------------------------

def work(case):
    """Every input byte read once, every output byte written once; rows of masked tokens are not
    read.  The checksum is counted as no work; an update is about 25 operations per element."""
    if case["op"] == "policy":
        n, v, item = case["tokens"], case["vocab"], 4 if case["half"] == "fp32" else 2
        read = n - int(case["masked"] * n)
        return {"bytes": item * v * (read + (n if case["grad"] else 0)) + 32 * n,
                "flops": (9 if case["grad"] else 4) * read * v}
    ns = _numels(case)
    held = sum(n * s for n, s in zip(ns, _items(case, len(ns))))
    if case["op"] == "norm":
        return {"bytes": held, "flops": 2 * sum(ns)}
    if case["op"] == "clip":
        return {"bytes": 2 * held, "flops": sum(ns)}
    return {"bytes": (30 if case["chained"] else 42) * sum(ns), "flops": 27 * sum(ns)}


def exact(case, seed):
    """The definitions in float64 from the same inputs; None for what is bytes."""
    global own
    if case["op"] == "policy":
        return _exact_policy(case, seed)
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    sums = [math.fsum(float(x) for x in torch.stack([torch.dot(p, p) for p in g.double().split(1 << 24)]))
            for g in s.grads]
    norm = math.sqrt(math.fsum(sums)) / case["scale"]
    factor = min(1.0, s.max_norm / norm) / case["scale"]
    wide = lambda x: torch.tensor(x, dtype=torch.float64)  # noqa: E731
    if case["op"] == "norm":
        return {"norm": wide(norm), "factor": wide(factor), "n_nonfinite": None}
    if case["op"] == "clip":
        out = []
        for flat in s.flat_grads:
            x, base, item = flat.double(), flat.data_ptr(), flat.element_size()
            for g in s.grads:
                at = (g.data_ptr() - base) // item
                if g.dtype == flat.dtype and 0 <= at < flat.numel():
                    x[at:at + g.numel()] *= factor
            out.append(x)
        return {"grads": out}
    h = {k: (float(np.float32(x)) if k != "step" else x) for k, x in s.hp.items()}
    bc1, bc2 = 1.0 - h["beta1"] ** h["step"], 1.0 - h["beta2"] ** h["step"]
    names = ("w16",) if case["chained"] else ("w16", "master", "m", "v")
    out = {name: s.flats[name].double() for name in names}
    for k, grad in enumerate(s.grads):
        old = dict(zip(("w16", "master", "m", "v"), s.tensors[4 * k:4 * k + 4]))
        g = grad.double() * factor
        new = {"m": old["m"].double().lerp(g, 1.0 - h["beta1"]), "v": old["v"].double().lerp(g * g, 1.0 - h["beta2"])}
        rate = (new["m"] / bc1) / ((new["v"] / bc2).sqrt() + h["eps"])
        new["master"] = old["master"].double() - h["lr"] * (h["weight_decay"] * old["master"].double() + rate)
        new["w16"] = new["master"]
        for name in names:
            at = (old[name].data_ptr() - s.flats[name].data_ptr()) // old[name].element_size()
            out[name][at:at + grad.numel()] = new[name]
    out.update(chunks=None, crcs=None, norm=wide(norm))
    return out


def _exact_policy(case, seed):
    s = _policy_inputs(case, seed)
    n, v = s.logits.shape
    out = {k: [] for k in ("logp", "token_loss", "dlogits")}
    loss = kl_sum = 0.0
    for a in range(0, n, max(1, int(1e8 / v))):
        part = slice(a, a + max(1, int(1e8 / v)))
        probs = torch.log_softmax(s.logits[part].double(), dim=1)
        y, w = s.targets[part], s.weights[part].double()
        row = torch.arange(y.numel(), device=DEV)
        logp = probs[row, y]
        change = logp - s.old_logp[part].double()
        gain = s.advantages[part].double()
        low, high = math.log1p(-_CLIP_LOW), math.log1p(_CLIP_HIGH)
        # the smaller of the two products is the clipped one above the upper border where the gain is
        # positive, and below the lower border where it is negative
        flat = ((gain > 0) & (change > high)) | ((gain < 0) & (change < low))
        token = -gain * torch.where(flat, change.clamp(low, high), change).exp()
        slope = torch.where(flat, 0.0, -gain * change.exp())
        if s.ref_logp is not None:
            up = logp - s.ref_logp[part].double()
            kl = torch.expm1(-up) + up
            token, slope = token + case["beta"] * kl, slope - case["beta"] * torch.expm1(-up)
            kl_sum += float((w * kl).sum())
        loss += float((w * token).sum())
        on = w != 0
        out["logp"].append(logp * on)
        out["token_loss"].append(token * on)
        if case["grad"]:
            g = -probs.exp_()
            g[row, y] = -torch.expm1(logp)
            out["dlogits"].append(g.mul_((w * slope * _loss_scale(case))[:, None]))
    got = {k: torch.cat(x) for k, x in out.items() if x}
    wide = lambda x: torch.tensor(x, dtype=torch.float64)  # noqa: E731
    got.update(loss=wide(loss), kl=wide(kl_sum), n_tokens=None, n_clipped=None)
    return got
