"""The calls between loss and step on the GPU against plain forms on the CPU (trainref.py): gradient norm, clipping,
the clipped step with its snapshot, and the policy loss with its gradient.

Tolerances.  A rounding is off by at most half a step: U32 = 2^-24, U64 = 2^-53 of the value.  The norm: squares are exact
in 64 bits, a lane adds no more than a few hundred of them one after the other.  The policy loss: a thread's
sum of V/256 + 64 additions at most, each term exp(z - m) off by 2 U32 of itself for the instruction and 2 U32 of |z - m| log2(e) in
its argument."""
import math

import numpy as np
import pytest
import torch

import trainref
from paper_2512_03644_amd import binding as ff
from paper_2512_03644_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")
U32, U64 = 2.0 ** -24, 2.0 ** -53
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def _tensors(spec, seed, std=1.0, pad=0):
    """Normal values; spec: (elements, type) each, carved out `pad` elements behind 16 bytes, elements around them 7.0."""
    g = torch.Generator().manual_seed(seed)
    out, arenas = [], []
    for n, t in spec:
        arena = torch.full((n + 48,), 7.0, dtype=t)
        arena[16 + pad:16 + pad + n] = (torch.randn(n, generator=g) * std).to(t)
        arenas.append(arena.to(DEV))
        out.append(arenas[-1][16 + pad:16 + pad + n])
    return out, arenas


def _norm(tensors, max_norm=INF, inv=1.0, grads=None, stream=None):
    lst = ff.ff_grad_list(tensors)
    stats, ws = ff.GradStats(DEV), ff.alloc_grad_workspace(lst, DEV)
    stats.words.fill_(-3.0)
    ff.ff_grad_norm(lst, stats, ws, max_norm, inv, grads, stream)
    torch.cuda.synchronize()
    return lst, stats, ws


def _check_norm(stats, tensors, max_norm, inv):
    sumsq, bad = trainref.sum_of_squares(tensors)
    assert int(stats.n_nonfinite) == bad and int(stats.skip) == (1 if bad else 0)
    if bad:
        assert float(stats.scale) == 0.0 and not math.isfinite(float(stats.norm))
        return
    norm = math.sqrt(sumsq) * inv
    assert float(stats.sumsq) == pytest.approx(sumsq, rel=1000 * U64, abs=0)
    assert float(stats.norm) == pytest.approx(norm, rel=510 * U64, abs=0)
    assert float(stats.scale) == pytest.approx(trainref.factor(norm, inv, max_norm), rel=U32 * 1.001, abs=0)


SIZES = [[1], [1, 1, 1], [0, 5, 0], [7, 8, 9, 15, 16, 17], [4095, 4096, 4097, 8192, 8193], [2047, 2048, 2049],
         [70001, 3, 257, 0, 100000], [1 << 20]]


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("pad", [0, 1, 3])
def test_norm_over_sizes_and_alignments(sizes, dtype, pad):
    ts, _ = _tensors([(n, dtype) for n in sizes], 5, 0.5, pad)
    for max_norm, inv in ((INF, 1.0), (0.25, 1.0 / 1024), (1e6, 0.5)):
        _, stats, _ = _norm(ts, max_norm, inv)
        _check_norm(stats, ts, max_norm, inv)


def test_norm_of_nothing():
    for ts in ([], [torch.zeros(0, device=DEV)]):
        _, stats, _ = _norm(ts, 1.0, 0.25)
        assert float(stats.norm) == 0.0 and float(stats.scale) == 0.25 and int(stats.skip) == 0
    _, stats, _ = _norm([torch.zeros(100, device=DEV)], 1.0)
    assert float(stats.norm) == 0.0 and float(stats.scale) == 1.0


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_no_finite_element_overflows_or_vanishes(dtype):
    big, small = torch.finfo(dtype).max, 2.0 ** -133 if dtype == BF16 else 2.0 ** -149
    for x in (big, small, 2.0 ** -126):
        ts = [torch.full((3000,), x, dtype=dtype, device=DEV)]
        _, stats, _ = _norm(ts)
        _check_norm(stats, ts, INF, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_elements_that_are_not_finite_are_counted(dtype, bad):
    ts, _ = _tensors([(20011, dtype), (3, dtype), (5000, dtype)], 8)
    for where in ([(0, 0)], [(0, 20010), (1, 1)], [(0, 4096), (0, 4097), (2, 4999), (1, 2), (0, 12345)]):
        cp = [t.clone() for t in ts]
        for k, i in where:
            cp[k][i] = bad
        _, stats, _ = _norm(cp, 1.0)
        _check_norm(stats, cp, 1.0, 1.0)


def test_norm_of_mixed_formats_in_several_launches_and_with_addresses_of_the_call():
    rng = np.random.default_rng(3)
    spec = [(int(n), (BF16, F16, F32)[k % 3]) for k, n in enumerate(rng.integers(0, 3000, size=4500))]
    ts, _ = _tensors(spec, 9, 1.0, 1)
    lst, stats, ws = _norm(ts, 10.0)
    _check_norm(stats, ts, 10.0, 1.0)
    first = stats.words.clone()
    others = [t.clone() for t in ts]  # the same values elsewhere
    ff.ff_grad_norm(lst, stats, ws, 10.0, 1.0, others)
    torch.cuda.synchronize()
    _check_norm(stats, ts, 10.0, 1.0)
    for _ in range(3):  # the same bits every time, and the workspace is as it was
        stats.words.fill_(-1.0)
        ff.ff_grad_norm(lst, stats, ws, 10.0)
        torch.cuda.synchronize()
        assert torch.equal(stats.words.view(torch.int64), first.view(torch.int64))


def test_norms_of_several_workers_join():
    parts = [_tensors([(5000 + 100 * k, BF16)], 20 + k)[0] for k in range(5)]
    each = ff.GradStats(DEV, 5)
    for k, ts in enumerate(parts):
        _, stats, _ = _norm(ts)
        each.words[k] = stats.words[0]
    total = ff.GradStats(DEV)
    everything = [t for ts in parts for t in ts]
    ff.ff_grad_norm_join(each, total, 3.0, 0.5)
    _check_norm(total, everything, 3.0, 0.5)
    ff.ff_grad_norm_join(each, each, 3.0, 0.5)  # into one of the parts
    assert torch.equal(each.words[0].view(torch.int64), total.words[0].view(torch.int64))
    bad = parts[3][0].clone()
    bad[17] = NAN
    _, stats, _ = _norm([bad])
    each.words[3] = stats.words[0]
    ff.ff_grad_norm_join(each, total, 3.0, 0.5)
    assert int(total.skip) == 1 and int(total.n_nonfinite) == 1 and float(total.scale) == 0.0


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("pad", [0, 1])
def test_clip_is_one_rounded_product(sizes, dtype, pad):
    ts, arenas = _tensors([(n, dtype) for n in sizes], 6, 3.0, pad)
    before = [t.clone() for t in ts]
    lst, stats, _ = _norm(ts, 0.7, 0.125)
    ff.ff_grad_clip(lst, stats)
    torch.cuda.synchronize()
    for t, b in zip(ts, before):
        assert torch.equal(t.cpu(), trainref.clipped(b, float(stats.scale)))
    for (n, _), a in zip([(n, 0) for n in sizes], arenas):  # nothing beside them
        assert (a[:16 + pad] == 7).all() and (a[16 + pad + n:] == 7).all()


def test_clip_leaves_alone_what_is_not_to_be_clipped():
    ts, _ = _tensors([(5000, BF16), (300, F32)], 7)
    ts[0][:4] = torch.tensor([NAN, INF, -INF, -0.0], dtype=BF16)
    bits = [t.clone().view(torch.int16) for t in ts]
    lst, stats, _ = _norm(ts, 0.01)
    assert int(stats.skip) == 1
    ff.ff_grad_clip(lst, stats)
    assert all(torch.equal(t.view(torch.int16), b) for t, b in zip(ts, bits))
    ts[0][:4] = 0
    bits = [t.clone().view(torch.int16) for t in ts]
    lst, stats, _ = _norm(ts, 1e9)
    assert float(stats.scale) == 1.0
    ff.ff_grad_clip(lst, stats)
    assert all(torch.equal(t.view(torch.int16), b) for t, b in zip(ts, bits))


def test_clip_of_many_tensors_with_addresses_of_the_call():
    rng = np.random.default_rng(4)
    spec = [(int(n), (BF16, F16, F32)[k % 3]) for k, n in enumerate(rng.integers(0, 600, size=4200))]
    ts, _ = _tensors(spec, 10)
    lst, stats, _ = _norm(ts, 1.0)
    others = [t.clone() for t in ts]
    ff.ff_grad_clip(lst, stats, others)
    torch.cuda.synchronize()
    for t, o in zip(ts, others):
        assert torch.equal(o.cpu(), trainref.clipped(t, float(stats.scale)))


# ---- clipped step --------------------------------------------------------------------------------

HP = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=3)


def _shard(numels, half, scale, seed=11, chunk=1 << 14):
    return wl.param_shard("s", numels, chunk, seed, DEV, with_grads=True, half=half, loss_scale=scale)


def _expect(shard, grads, hp, scale, skip, oracle):
    segs, new = [], []
    for q, g in zip(shard.params, grads):
        w, p, m, v = trainref.step(q.w16, q.master, q.m, q.v, g, hp, scale, skip)
        new.append((w, p, m, v))
        segs += [w.view(torch.int16).numpy(), p, m, v]
    buf, crcs = oracle.pack(segs, shard.chunk_bytes, threads=4)
    return new, buf, crcs


def _same(t, x):
    a = t.detach().cpu().contiguous()
    b = x if isinstance(x, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(x))
    return torch.equal(a.view(torch.int16), b.contiguous().view(torch.int16))


NUMELS = [[1], [5000, 70001, 257], [3, 1, 8191, 8192, 8193, 2, 16385], [40000] * 70]


@pytest.mark.parametrize("half", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("numels", NUMELS, ids=lambda n: "%dx%d" % (len(n), n[0]))
@pytest.mark.parametrize("chained", [False, True], ids=["inplace", "chained"])
@pytest.mark.parametrize("skip", [False, True], ids=["update", "skip"])
@pytest.mark.parametrize("side", [False, True], ids=["default", "sidestream"])
def test_clipped_step_and_its_snapshot(numels, half, chained, skip, side, oracle):
    loss_scale = 1024.0 if half == F16 else 1.0
    shard = _shard(numels, half, loss_scale)
    plan = ff.plan_for_shard(shard)
    chunks, crcs, bad, n_bad = ff.alloc_outputs(plan, DEV)
    chunks.fill_(0xA5)
    prev = None
    grads = [q.grad for q in shard.params]
    if skip:
        grads[-1][0] = INF
        shard.params[0].master[0] = NAN
    lst = ff.ff_grad_list(grads)
    stats, ws = ff.GradStats(DEV), ff.alloc_grad_workspace(lst, DEV)
    host = [[t.clone() for t in (q.w16, q.master, q.m, q.v)] for q in shard.params]
    if chained:
        prev, prev_crcs, _, _ = ff.alloc_outputs(plan, DEV)
        ff.ff_pack(plan, prev, prev_crcs)
        torch.cuda.synchronize()
        for q in shard.params:
            for t in (q.w16, q.master, q.m, q.v):
                t.view(torch.uint8).fill_(0x5A)
    s = torch.cuda.Stream() if side else None
    torch.cuda.synchronize()
    ff.ff_grad_norm(lst, stats, ws, 1e-4, 1 / loss_scale, stream=s)
    ff.ff_adam_step_clipped(plan, grads, HP, stats, chunks, crcs, prev, stream=s)
    torch.cuda.synchronize()
    assert int(stats.skip) == int(skip)
    if not skip:
        assert float(stats.scale) < 1 / loss_scale or sum(numels) == 1
    old = wl.Shard("old", shard.chunk_bytes, [], [wl.ParamGroup(*h) for h in host])
    new, buf, want = _expect(old, grads, HP, float(stats.scale), skip, oracle)
    assert np.array_equal(chunks.cpu().numpy(), buf)
    assert np.array_equal(crcs.cpu().numpy().view(np.uint32), want)
    for q, n in zip(shard.params, new):
        assert _same(q.w16, n[0])
        for t, x in zip((q.master, q.m, q.v), n[1:]):
            if chained:
                assert bool((t.view(torch.uint8) == 0x5A).all())
            else:
                assert _same(t, x)


@pytest.mark.parametrize("step", [1, 333, 100000])
def test_clipped_step_is_the_unclipped_one_where_nothing_is_clipped(step, oracle):
    hp = dict(HP, step=step)
    for half, scale in ((BF16, 1.0), (F16, 512.0)):
        shard = _shard([5000, 70001, 257], half, scale)
        plan = ff.plan_for_shard(shard)
        a, ca, _, _ = ff.alloc_outputs(plan, DEV)
        b, cb, _, _ = ff.alloc_outputs(plan, DEV)
        prev, cp, _, _ = ff.alloc_outputs(plan, DEV)
        grads = [q.grad for q in shard.params]
        lst, stats, _ = _norm(grads, INF, 1 / scale)
        ff.ff_pack(plan, prev, cp)
        ff.ff_adam_step_chained(plan, grads, hp, prev, a, ca, 1 / scale)
        ff.ff_adam_step_clipped(plan, grads, hp, stats, b, cb, prev)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and torch.equal(ca, cb)


def test_clipped_step_follows_the_formula_in_64_bits():
    # five rounded operations to m' and v', about ten to p': the step itself is lr * (at most about 1/sqrt(1 - b2)) large
    shard = _shard([30001, 511], BF16, 1.0)
    plan = ff.plan_for_shard(shard)
    grads = [q.grad for q in shard.params]
    lst, stats, _ = _norm(grads, 0.05)
    old = [[t.clone().cpu().double().numpy() for t in (q.master, q.m, q.v)] for q in shard.params]
    chunks, crcs, _, _ = ff.alloc_outputs(plan, DEV)
    ff.ff_adam_step_clipped(plan, grads, HP, stats, chunks, crcs)
    torch.cuda.synchronize()
    hp = {k: float(np.float32(x)) if k != "step" else x for k, x in HP.items()}
    sumsq, _ = trainref.sum_of_squares(grads)
    scale = trainref.factor(math.sqrt(sumsq), 1.0, 0.05)
    for q, o, g in zip(shard.params, old, grads):
        gg = g.cpu().double().numpy() * scale
        p, m, v = trainref.step64(*o, gg, hp)
        got = [t.cpu().double().numpy() for t in (q.master, q.m, q.v)]
        size_m = np.abs(0.9 * o[1]) + np.abs(0.1 * gg)
        assert (np.abs(got[1] - m) <= 8 * U32 * size_m).all()
        assert (np.abs(got[2] - v) <= 10 * U32 * np.abs(v) + 1e-44).all()
        rate = hp["lr"] * (size_m / (1 - hp["beta1"] ** 3)) / (np.sqrt(v / (1 - hp["beta2"] ** 3)) + hp["eps"])
        assert (np.abs(got[0] - p) <= 3 * U32 * np.abs(o[0]) + 24 * U32 * rate).all()


# ---- policy loss ---------------------------------------------------------------------------------

def _policy_inputs(n, v, dtype, seed, pad=0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    rows = torch.full((n, v + pad), 9.0)
    rows[:, :v] = torch.randn(n, v, generator=g) * spread
    y = torch.randint(0, v, (n,), generator=g)
    z = rows[:, :v]
    z[torch.arange(n), y] += 6 * torch.rand(n, generator=g)
    rows = rows.to(dtype)
    z = rows[:, :v]
    logp = z.double().log_softmax(1)[torch.arange(n), y]
    change = torch.randn(n, generator=g).double() * 0.25
    for border in (math.log(0.8), math.log(1.3)):  # rounding decides next to a border
        change = torch.where((change - border).abs() < 1e-3, change + 4e-3, change)
    old = (logp - change).float()
    ref = (logp + 0.4 * torch.randn(n, generator=g).double()).float()
    adv = torch.randn(n, generator=g)
    w = torch.rand(n, generator=g) + 0.5
    return rows, y, old, ref, adv, w


def _run_policy(rows, v, y, old, adv, w, ref, beta, loss_scale=1.0, grad=True, in_place=False, grad_pad=0, low=0.2, high=0.3,
                stream=None):
    rows = rows.to(DEV).clone()
    z = rows[:, :v]
    n = z.shape[0]
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    tensors = [dev(t) for t in (y, old, adv, w, ref)]
    batch = ff.policy_batch(z, *tensors, low, high, beta, loss_scale)
    logp, token = (torch.full((n,), -7.0, device=DEV) for _ in range(2))
    stats, ws = ff.PolicyStats(DEV), ff.alloc_policy_workspace(n, v, DEV)
    stats.words.fill_(-1)
    out = rows if in_place else torch.full((n, v + grad_pad), 5.0, dtype=rows.dtype, device=DEV)
    torch.cuda.synchronize()
    ff.ff_policy_loss(batch, logp, token, stats, ws, out[:, :v] if grad else None, stream)
    torch.cuda.synchronize()
    return dict(logp=logp.cpu(), token_loss=token.cpu(), loss=float(stats.loss), kl=float(stats.kl),
                n_tokens=int(stats.n_tokens), n_clipped=int(stats.n_clipped), n_invalid=int(stats.n_invalid),
                dlogits=out[:, :v].cpu() if grad else None, beside=out[:, v:].cpu())


def _check_policy(got, rows, v, y, old, adv, w, ref, beta, loss_scale=1.0, low=0.2, high=0.3):
    z = rows[:, :v]
    want = trainref.policy(z, y, old, adv, w, ref, low, high, beta, loss_scale)
    assert [got[k] for k in ("n_tokens", "n_clipped", "n_invalid")] == [want[k] for k in ("n_tokens", "n_clipped", "n_invalid")]
    zz = z.double()
    m = zz.masked_fill(zz == -INF, -1e30).amax(1, keepdim=True)
    far = torch.where(zz == -INF, 0.0, m - zz)
    # of the sum: additions, and the terms' own errors weighted by what they add
    mean_far = (torch.where(zz == -INF, 0.0, zz.softmax(1)) * far).sum(1).nan_to_num()
    total = U32 * (v / 256 + 64 + 2 + 3 * mean_far)
    used = want["used"]
    err = torch.where(used, total + U32 * want["logp"].abs(), 0.0)
    assert ((got["logp"].double() - want["logp"]).abs() <= err).all()
    # d token / d logp is the slope, which changes by no more than its parts do
    err = torch.where(used, total * want["size"] * 1.01 + U32 * (want["token_loss"].abs() + 4), 0.0)
    assert ((got["token_loss"].double() - want["token_loss"]).abs() <= err + 1e-30).all()
    ww = w.abs().double()
    slack = float((ww * (err + 2 * U32)).sum())
    assert abs(got["loss"] - want["loss"]) <= slack + U32 * abs(want["loss"])
    kl_err = 0.0 if ref is None else float((ww * used * (total * (1 + (ref.double() - want["logp"]).exp())) + 1e-12).sum())
    assert abs(got["kl"] - want["kl"]) <= kl_err * 1.01 + U32 * abs(want["kl"])
    if got["dlogits"] is None:
        return
    g, x = got["dlogits"].double(), want["dlogits"]
    fi = torch.finfo(rows.dtype)
    shape = x.abs() * (fi.eps / 2 * 1.01 + U32 * (8 + 4 * far) + 2 * total[:, None])
    # the slope's own error comes from its parts, which may cancel; and what is below the format's smallest steps
    probs = torch.where(used[:, None], zz.softmax(1), 0.0)
    hot = torch.zeros_like(probs)
    inside = (y >= 0) & (y < v)
    hot[torch.arange(len(y))[inside], y[inside]] = 1.0
    parts = (want["coef"] * (total + 8 * U32))[:, None] * torch.maximum(probs, hot * (1 - probs))
    floor = fi.smallest_normal * fi.eps / 2 if rows.dtype == F16 else 2.0 ** -126
    assert ((g - x).abs() <= shape + parts * 1.01 + floor).all(), float((g - x).abs().max())


VOCABS = [1, 2, 7, 8, 9, 63, 511, 2047, 2048, 4099, 16384, 32000, 50021]


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("v", VOCABS)
def test_policy_over_vocabularies(v, dtype):
    n = 5
    for pad, beta in ((0, 0.05), (3, 0.0)):
        rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, v + pad, pad)
        y[0], y[1] = 0, v - 1
        r = ref if beta else None
        scale = 256.0 if dtype == F16 else 1.0
        got = _run_policy(rows, v, y, old, adv, w, r, beta, scale, grad_pad=pad)
        _check_policy(got, rows, v, y, old, adv, w, r, beta, scale)
        assert (got["beside"] == 5).all()


@pytest.mark.parametrize("n,v", [(1, 32000), (1, 1000), (2, 128256), (3, 130001), (64, 3001), (777, 1003), (300, 20000)])
def test_policy_over_token_counts(n, v):
    rows, y, old, ref, adv, w = _policy_inputs(n, v, BF16, n)
    w[1::3] = 0
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1)
    _check_policy(got, rows, v, y, old, adv, w, ref, 0.1)
    alone = _run_policy(rows, v, y, old, adv, w, ref, 0.1, grad=False)
    for k in ("logp", "token_loss"):
        assert torch.equal(alone[k], got[k])
    assert alone["loss"] == got["loss"] and alone["kl"] == got["kl"]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,v,pad", [(40, 4099, 0), (40, 4099, 5), (3, 32000, 0)])
def test_policy_gradient_in_place_of_the_logits(n, v, pad, dtype):
    rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, 31, pad)
    w[5:9] = 0
    apart = _run_policy(rows, v, y, old, adv, w, ref, 0.1)
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1, in_place=True)
    assert torch.equal(got["dlogits"], apart["dlogits"]) and torch.equal(got["logp"], apart["logp"])
    assert (got["beside"] == 9).all()


# one workgroup to a row, or several; tokens counted one by one, or joined by a kernel of their own; rows that registers hold whole, or
# in part, or that have more parts than are joined
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,slots", [(64, 4097), (65, 4097), (64, 256), (65, 257), (300, 1025), (257, 4097), (2, 8193), (70, 16385),
                                     (1, 65535), (1, 65537)])
@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "inplace"])
def test_policy_on_both_sides_of_every_rule(n, slots, dtype, in_place):
    items = 4 if dtype == F32 else 8
    v = slots * items + 3
    rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, slots, 1)
    y[0] = v - 1
    y[-1] = (slots - 1) * items
    w[n // 2] = 0 if n > 2 else w[n // 2]
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1, in_place=in_place)
    _check_policy(got, rows, v, y, old, adv, w, ref, 0.1)
    assert (got["beside"] == 9).all() or not in_place


@pytest.mark.parametrize("n,slots,dtype,in_place", [
    (257, 8193, BF16, True), (257, 14336, F32, False), (257, 14337, BF16, False), (300, 16033, F16, True), (258, 20480, F32, True),
    (257, 20481, F32, False), (513, 2049, F32, True), (513, 4096, F16, True), (1025, 3072, BF16, False), (1025, 3073, BF16, True),
    (512, 2050, F16, False)], ids=lambda x: str(x).replace("torch.", ""))
def test_policy_of_many_long_rows(n, slots, dtype, in_place):
    """Rows in registers and LDS, whole and with an end that is read again, and those too long for it."""
    items = 4 if dtype == F32 else 8
    v = slots * items + 1
    rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, slots, 1)
    for k, at in enumerate((0, 511, 512, 8 * 512 - 1, 8 * 512, slots - 1)):  # targets at the borders of what is held where
        y[k] = min(slots - 1, at) * items + k % items
    y[6] = v - 1
    w[7] = 0
    rows[8, :v] = -INF
    rows[9, 5:v - 5] = -INF
    y[9] = 2
    moved = [0, 1, 2, 3, 4, 5, 6, 9]
    logp = rows[moved, :v].double().log_softmax(1).gather(1, y[moved, None])[:, 0]
    old[moved], ref[moved] = (logp - 0.1).float(), (logp + 0.2).float()
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1, in_place=in_place)
    _check_policy(got, rows, v, y, old, adv, w, ref, 0.1)
    assert (got["beside"] == 9).all() or not in_place


def test_policy_workspace_serves_call_after_call():
    """Counted tokens leave the count as they found it: calls of several sizes on one workspace, back to back."""
    v = 2000
    ws = ff.alloc_policy_workspace(64, 40000, DEV)
    calls = []
    for k, (n, vocab) in enumerate(((64, v), (1, 40000), (7, v), (64, 36000), (3, 40000), (64, v))):
        rows, y, old, ref, adv, w = _policy_inputs(n, vocab, BF16, 100 + k)
        t = [x.to(DEV) for x in (rows, y, old, adv, w, ref)]
        stats, logp, token = ff.PolicyStats(DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        calls.append((ff.policy_batch(*t, beta=0.1), logp, token, stats, t, trainref.policy(rows, y, old, adv, w, ref, 0.2, 0.2, 0.1)))
    torch.cuda.synchronize()
    for _ in range(3):
        for batch, logp, token, stats, _, _ in calls:
            ff.ff_policy_loss(batch, logp, token, stats, ws)
    torch.cuda.synchronize()
    for _, _, _, stats, _, want in calls:
        assert int(stats.n_tokens) == want["n_tokens"] and float(stats.loss) == pytest.approx(want["loss"], rel=1e-4)
        assert float(stats.kl) == pytest.approx(want["kl"], rel=1e-4)
    assert int(ws[:64].max()) == 0


def test_policy_rows_that_leave_nothing_targets_outside_and_masked_rows():
    n, v = 24, 3001
    rows, y, old, ref, adv, w = _policy_inputs(n, v, BF16, 77)
    rows[0] = -INF                      # nothing is left
    y[1], y[2], y[3] = -1, v, -100      # outside
    w[4] = w[5] = 0
    rows[4] = NAN                       # masked: not looked at
    y[5] = 1 << 40
    keep = rows[6, y[6]].clone()
    rows[6] = -INF                      # one candidate
    rows[6, y[6]] = keep
    rows[7, : v // 2] = -INF
    rows[7, y[7]] = 1.0
    rows[8] = torch.finfo(BF16).min     # the type's lowest value everywhere
    rows[9, 5] = torch.finfo(BF16).max
    y[9] = 5
    rows[10] = -INF
    w[10] = 0                           # masked and nothing left
    logp = rows.double().log_softmax(1)
    for k in (6, 7, 8, 9):
        old[k] = float(logp[k, y[k]]) + 0.1
        ref[k] = float(logp[k, y[k]]) - 0.1
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1)
    _check_policy(got, torch.where(torch.isnan(rows), torch.zeros_like(rows), rows), v, y, old, adv, w, ref, 0.1)
    assert got["n_invalid"] == 4
    for k in (0, 1, 2, 3, 4, 5, 10):
        assert (got["dlogits"][k] == 0).all() and got["logp"][k] == 0 and got["token_loss"][k] == 0
    assert torch.isfinite(got["dlogits"]).all()


@pytest.mark.parametrize("n", [2, 63, 64, 65, 127, 129, 4095, 4096, 20000])
def test_policy_tokens_are_joined_whatever_their_number(n):
    """Counted in one group or in 64 of unequal sizes; the same bits every time, on a workspace that other sizes use in between."""
    v = 40
    ws = ff.alloc_policy_workspace(20000, v, DEV)
    rows, y, old, ref, adv, w = _policy_inputs(n, v, F32, n)
    w[::3] = 0
    y[1] = v  # outside
    want = trainref.policy(rows, y, old, adv, w, ref, 0.2, 0.2, 0.1)
    other, t = ([x.to(DEV) for x in given] for given in (
        [x for x in _policy_inputs(70, v, F32, 1)], (rows, y, old, ref, adv, w)))
    calls = []
    for z, yy, o, r, a, ww in (t, other):
        logp, token = (torch.empty(z.shape[0], device=DEV) for _ in range(2))
        calls.append((ff.policy_batch(z, yy, o, a, ww, r, 0.2, 0.2, 0.1), logp, token, ff.PolicyStats(DEV)))
    seen = set()
    for _ in range(4):
        for batch, logp, token, stats in calls:
            ff.ff_policy_loss(batch, logp, token, stats, ws)
        seen.add(tuple(calls[0][3].words.tolist()))
    assert len(seen) == 1
    stats = calls[0][3]
    assert [int(stats.n_tokens), int(stats.n_clipped), int(stats.n_invalid)] == [want[k] for k in ("n_tokens", "n_clipped", "n_invalid")]
    # the sums add the tokens' own losses in 64 bits: what is out is the tokens' rounding to 32, and that of the result
    token, ww = calls[0][2].double().cpu(), w.double()
    size = float((ww * token.abs()).sum())
    assert abs(float(stats.loss) - float((ww * token).sum())) <= U32 * (1.01 * size + abs(float(stats.loss)))


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("n,v", [(6, 3001), (2, 64000)])
def test_policy_rows_with_a_nan_or_infinity_say_so(bad, n, v):
    rows, y, old, ref, adv, w = _policy_inputs(n, v, BF16, 78)
    rows[1, v - 1] = bad
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1)
    assert math.isnan(got["logp"][1]) and math.isnan(got["loss"]) and torch.isnan(got["dlogits"][1]).all()
    others = [k for k in range(n) if k != 1]
    assert torch.isfinite(got["dlogits"][others]).all() and got["n_tokens"] == n
    rows[1] = -INF
    rows[1, 7] = NAN
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1)
    assert math.isnan(got["logp"][1]) and torch.isnan(got["dlogits"][1]).all()


def test_policy_target_that_is_ruled_out():
    rows, y, old, ref, adv, w = _policy_inputs(3, 501, F32, 79)
    rows[1, y[1]] = -INF
    adv[1] = 1.0
    got = _run_policy(rows, 501, y, old, adv, w, None, 0.0)
    assert got["logp"][1] == -INF and got["token_loss"][1] == 0 and (got["dlogits"][1] == 0).all()
    got = _run_policy(rows, 501, y, old, adv, w, ref, 0.1)
    assert got["token_loss"][1] == INF and got["kl"] == INF


def test_policy_of_no_tokens():
    z = torch.zeros(0, 100, dtype=BF16, device=DEV)
    e, i = torch.zeros(0, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV)
    stats = ff.PolicyStats(DEV)
    stats.words.fill_(-1)
    ff.ff_policy_loss(ff.policy_batch(z, i, e, e, e), e, e, stats, ff.alloc_policy_workspace(0, 100, DEV))
    assert torch.equal(stats.words.cpu(), torch.zeros(4, dtype=torch.int64))


def test_policy_gradient_against_differences():
    n, v, h = 6, 37, 1e-6
    rows, y, old, ref, adv, w = _policy_inputs(n, v, F32, 5)
    args = (y, old, adv, w, ref, 0.2, 0.3, 0.1, 8.0)
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1, 8.0)["dlogits"].double()
    z = rows.double()
    for t in range(n):
        for j in list(range(0, v, 5)) + [int(y[t])]:
            up, down = z.clone(), z.clone()
            up[t, j] += h
            down[t, j] -= h
            diff = 8.0 * (trainref.policy(up, *args)["loss"] - trainref.policy(down, *args)["loss"]) / (2 * h)
            # (the difference itself: h^2 of third derivatives, and 64-bit roundings of the loss over h)
            assert abs(diff - float(got[t, j])) <= 1e-4 * (1 + abs(diff)) * 0.1 + 1e-7


# ---- streams, graphs, everything together ----------------------------------------------------------

def test_calls_on_another_stream_and_in_a_graph(oracle):
    """norm -> clip, and loss -> norm -> clipped step, captured and replayed with eager work between the replays."""
    n, v = 33, 4001
    rows, y, old, ref, adv, w = _policy_inputs(n, v, BF16, 41)
    z = rows.to(DEV)
    y, old, ref, adv, w = (t.to(DEV) for t in (y, old, ref, adv, w))
    shard = _shard([5000, 70001], BF16, 1.0)
    plan = ff.plan_for_shard(shard)
    prev, prev_crcs, _, _ = ff.alloc_outputs(plan, DEV)
    ff.ff_pack(plan, prev, prev_crcs)
    chunks, crcs, _, _ = ff.alloc_outputs(plan, DEV)
    grads = [q.grad for q in shard.params]
    dz = torch.empty_like(z)
    logp, token = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    pstats, pws = ff.PolicyStats(DEV), ff.alloc_policy_workspace(n, v, DEV)
    everything = ff.ff_grad_list(grads + [dz])
    stats, ws = ff.GradStats(DEV), ff.alloc_grad_workspace(everything, DEV)
    clips, cstats = ff.ff_grad_list([dz]), ff.GradStats(DEV)
    cws = ff.alloc_grad_workspace(clips, DEV)
    batch = ff.policy_batch(z, y, old, adv, w, ref, beta=0.1)

    def iteration(stream=None):
        ff.ff_policy_loss(batch, logp, token, pstats, pws, dz, stream)
        ff.ff_grad_norm(everything, stats, ws, 0.02, stream=stream)
        ff.ff_grad_norm(clips, cstats, cws, 0.01, stream=stream)
        ff.ff_grad_clip(clips, cstats, stream=stream)
        ff.ff_adam_step_clipped(plan, grads, HP, stats, chunks, crcs, prev, stream)

    outputs = [logp, token, pstats.words, dz, stats.words, cstats.words, chunks, crcs] + [q.w16 for q in shard.params]

    def bits():
        return [t.clone().view(torch.uint8) for t in outputs]

    def spoil():
        for t in outputs:
            t.view(torch.uint8).fill_(0x33)

    iteration()
    torch.cuda.synchronize()
    first = bits()
    _check_norm(stats, grads + [_unclipped(batch, dz)], 0.02, 1.0)
    s = torch.cuda.Stream()
    spoil()
    torch.cuda.synchronize()
    iteration(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, bits()))
    graph = torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph.capture_begin()
        iteration(s)
        graph.capture_end()
    torch.cuda.synchronize()
    for k in range(4):
        spoil()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, bits())), k
        spoil()
        iteration()  # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, bits())), k


@pytest.mark.parametrize("n,v", [(130, 1000), (300, 70001), (600, 20000)])
def test_policy_of_many_tokens_in_a_graph(n, v):
    """Tokens counted in groups, rows partly in LDS: replayed with eager calls on the same workspace between the replays."""
    rows, y, old, ref, adv, w = (t.to(DEV) for t in _policy_inputs(n, v, BF16, n))
    batch = ff.policy_batch(rows, y, old, adv, w, ref, beta=0.1)
    logp, token, dz = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty_like(rows)
    stats, ws = ff.PolicyStats(DEV), ff.alloc_policy_workspace(n, v, DEV)
    outputs = [logp, token, dz, stats.words]

    def call(stream=None):
        ff.ff_policy_loss(batch, logp, token, stats, ws, dz, stream)

    def bits():
        torch.cuda.synchronize()
        got = [t.clone().view(torch.uint8) for t in outputs]
        for t in outputs:
            t.view(torch.uint8).fill_(0x33)
        return got

    call()
    first = bits()
    assert int(first[3].view(torch.int64)[1]) == n
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph.capture_begin()
        call(s)
        graph.capture_end()
    torch.cuda.synchronize()
    for k in range(3):
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(first, bits())), k
        call()
        assert all(torch.equal(a, b) for a, b in zip(first, bits())), k


def _unclipped(batch, dz):
    out = torch.empty_like(dz)
    n, v = dz.shape
    logp, token = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ff.ff_policy_loss(batch, logp, token, ff.PolicyStats(DEV), ff.alloc_policy_workspace(n, v, DEV), out)
    torch.cuda.synchronize()
    return out


def test_offsets_beyond_32_bits():
    """A gradient of more than 4 GiB, and rows of logits that lie 4 GiB apart."""
    n = (1 << 30) + 4099  # fp32
    t = torch.zeros(n, device=DEV)
    places = [0, 1, (1 << 29) + 5, (1 << 30) - 1, 1 << 30, (1 << 30) + 7, n - 1]
    for k, i in enumerate(places):
        t[i] = k + 1.0
    lst, stats, _ = _norm([t, torch.ones(3, device=DEV)], 2.0)
    want = math.sqrt(sum((k + 1) ** 2 for k in range(len(places))) + 3)
    assert float(stats.norm) == pytest.approx(want, rel=1e-12)
    ff.ff_grad_clip(lst, stats)
    for k, i in enumerate(places):
        assert float(t[i]) == float(np.float32(k + 1) * np.float32(float(stats.scale)))
    assert int((t != 0).sum()) == len(places)
    del t, lst
    v, stride = 3001, 1 << 31  # bf16 rows
    rows, y, old, ref, adv, w = _policy_inputs(3, v, BF16, 90)
    far = torch.empty(2 * stride + v, dtype=BF16, device=DEV)
    z = far.as_strided((3, v), (stride, 1))
    z.copy_(rows.to(DEV))
    dev = [x.to(DEV) for x in (y, old, adv, w, ref)]
    logp, token, stats = torch.empty(3, device=DEV), torch.empty(3, device=DEV), ff.PolicyStats(DEV)
    ff.ff_policy_loss(ff.policy_batch(z, *dev, 0.2, 0.3, 0.1), logp, token, stats, ff.alloc_policy_workspace(3, v, DEV), z)
    near = _run_policy(rows, v, y, old, adv, w, ref, 0.1)
    assert torch.equal(z.cpu(), near["dlogits"]) and torch.equal(logp.cpu(), near["logp"])


def test_join_of_many_workers_is_in_rank_order():
    n = 200
    g = torch.Generator().manual_seed(2)
    values = torch.randn(n, generator=g).double().exp()
    parts, total = ff.GradStats(DEV, n), ff.GradStats(DEV)
    parts.words[:, 0] = values.to(DEV)
    ff.ff_grad_norm_join(parts, total)
    want = 0.0
    for x in values.tolist():
        want += x
    assert float(total.sumsq) == want and float(total.norm) == math.sqrt(want) and float(total.scale) == 1.0


@pytest.mark.parametrize("skip", [False, True], ids=["update", "skip"])
@pytest.mark.parametrize("chained", [False, True], ids=["inplace", "chained"])
def test_clipped_step_copies_tensors_that_are_not_trained(chained, skip, oracle):
    shard = _shard([5000, 257], BF16, 1.0)
    g = torch.Generator().manual_seed(4)
    raw = [torch.randn(n, generator=g).to(DEV) for n in (1, 3001, 20000)]
    segs = [raw[0]] + shard.segments[:4] + [raw[1]] + shard.segments[4:] + [raw[2]]
    four = [ff.FF_KIND_W16, ff.FF_KIND_MASTER, ff.FF_KIND_M, ff.FF_KIND_V]
    kinds = [ff.FF_KIND_RAW] + four + [ff.FF_KIND_RAW] + four + [ff.FF_KIND_RAW]
    plan = ff.ff_snapshot_plan(segs, 1 << 14, 0, kinds, [0] + [0] * 4 + [0] + [1] * 4 + [0])
    chunks, crcs, _, _ = ff.alloc_outputs(plan, DEV)
    prev = None
    if chained:
        prev, prev_crcs, _, _ = ff.alloc_outputs(plan, DEV)
        ff.ff_pack(plan, prev, prev_crcs)
    grads = [q.grad for q in shard.params]
    if skip:
        grads[0][77] = NAN
    lst, stats, _ = _norm(grads, 1e-3)
    old = [[t.clone() for t in (q.w16, q.master, q.m, q.v)] for q in shard.params]
    ff.ff_adam_step_clipped(plan, grads, HP, stats, chunks, crcs, prev)
    torch.cuda.synchronize()
    new = [trainref.step(*o, gr, HP, float(stats.scale), skip) for o, gr in zip(old, grads)]
    flat = [[n[0].view(torch.int16).numpy(), *n[1:]] for n in new]
    r = [t.cpu().numpy() for t in raw]
    buf, want = oracle.pack([r[0], *flat[0], r[1], *flat[1], r[2]], 1 << 14, threads=2)
    assert np.array_equal(chunks.cpu().numpy(), buf)
    assert np.array_equal(crcs.cpu().numpy().view(np.uint32), want)


@pytest.mark.parametrize("half", [BF16, F16], ids=["bf16", "fp16"])
def test_example_learns_and_its_snapshot_is_taken_over(half):
    """The example's program: its loss falls, its gradients are clipped, and the newcomer has the trained weights."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_training.py")
    spec = importlib.util.spec_from_file_location("policy_training", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms, trained, taken_over = example.train(20, half, report=lambda s: None)
    assert losses[-1] < losses[0] - 0.02 and all(math.isfinite(x) for x in losses + norms)
    assert norms[0] > example.MAX_NORM
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(trained, taken_over))


@pytest.mark.parametrize("most", [65, 200, 512])
def test_policy_workspace_of_a_large_batch_serves_the_last_small_one(most):
    """A program's workspace is that of its largest batch; an epoch ends with fewer tokens, whose rows are split."""
    v = 40003
    size = ff.alloc_policy_workspace(most, v, "cpu").nbytes
    arena = torch.zeros(size + (1 << 16), dtype=torch.uint8, device=DEV)
    arena[size:] = 0xA7
    ws = arena[:size]
    for n in (60, most, 64, 3):
        rows, y, old, ref, adv, w = _policy_inputs(n, v, BF16, n)
        t = [x.to(DEV) for x in (rows, y, old, adv, w, ref)]
        logp, token, dz = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty_like(t[0])
        stats = ff.PolicyStats(DEV)
        ff.ff_policy_loss(ff.policy_batch(*t, 0.2, 0.3, 0.1), logp, token, stats, ws, dz)
        torch.cuda.synchronize()
        got = dict(logp=logp.cpu(), token_loss=token.cpu(), loss=float(stats.loss), kl=float(stats.kl), n_tokens=int(stats.n_tokens),
                   n_clipped=int(stats.n_clipped), n_invalid=int(stats.n_invalid), dlogits=dz.cpu())
        _check_policy(got, rows, v, y, old, adv, w, ref, 0.1)
        assert bool((arena[size:] == 0xA7).all())


def test_policy_of_more_tokens_than_one_launch_has_work_items_for():
    """A wavefront to a row: 67,108,863 rows fill the 32 bits that a launch's work items are counted in."""
    n, v = (1 << 26) + 6, 8
    g = torch.Generator(device=DEV).manual_seed(6)
    z = torch.empty(n, v, dtype=BF16, device=DEV).normal_(0, 2.0, generator=g)
    y = torch.randint(0, v, (n,), generator=g, device=DEV)
    old, adv = torch.full((n,), -2.0, device=DEV), torch.empty(n, device=DEV).normal_(generator=g)
    w = torch.full((n,), 1.0 / n, device=DEV)
    w[5::9] = 0
    logp, token, dz = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV), torch.full_like(z, 7.0)
    stats, ws = ff.PolicyStats(DEV), ff.alloc_policy_workspace(n, v, DEV)
    for _ in range(2):  # counters are left as they were
        ff.ff_policy_loss(ff.policy_batch(z, y, old, adv, w, None, 0.2, 0.3), logp, token, stats, ws, dz, None)
    torch.cuda.synchronize()
    assert int(stats.n_tokens) == int((w != 0).sum()) and int(stats.n_invalid) == 0
    loss = size = 0.0
    for a in range(0, n, 1 << 24):
        part = slice(a, a + (1 << 24))
        want = torch.log_softmax(z[part].double(), 1).gather(1, y[part, None])[:, 0] * (w[part] != 0)
        # eight terms, 2 U32 of each and 3 of its distance, at most 20 here; the result's rounding
        assert bool(((logp[part].double() - want).abs() <= 128 * U32 + U32 * want.abs()).all())
        counted = (w[part].double() * token[part].double())
        loss, size = loss + float(counted.sum()), size + float(counted.abs().sum())
    assert abs(float(stats.loss) - loss) <= U32 * (1.01 * size + abs(loss))
    border = (1 << 26) - 1
    for a in (0, border - 20, n - 20):
        part = slice(a, min(n, a + 40))
        small = [t[part].cpu() for t in (z, y, old, adv, w)]
        want = trainref.policy(*small, None, 0.2, 0.3)
        assert torch.equal(want["used"], small[4] != 0)
        assert torch.allclose(token[part].cpu().double(), want["token_loss"], rtol=200 * U32, atol=0)
        assert torch.allclose(dz[part].cpu().double(), want["dlogits"], rtol=2.0 ** -7, atol=2.0 ** -126)


@pytest.mark.parametrize("n", [2048, 2049, 4500, 10000])
def test_norm_has_the_same_bits_wherever_its_addresses_come_from(n):
    """Lists whose addresses fit a launch's arguments, and longer ones."""
    rng = np.random.default_rng(n)
    ts, _ = _tensors([(int(k), (BF16, F16, F32)[i % 3]) for i, k in enumerate(rng.integers(0, 3000, size=n))], n, 1.0, 1)
    lst, stats, ws = _norm(ts, 10.0)
    _check_norm(stats, ts, 10.0, 1.0)
    first = stats.words.clone()
    others = [t.clone() for t in ts]
    for grads in (others, ts, None, others):
        stats.words.fill_(-1.0)
        ff.ff_grad_norm(lst, stats, ws, 10.0, grads=grads)
        torch.cuda.synchronize()
        assert torch.equal(stats.words.view(torch.int64), first.view(torch.int64))
    others[n // 2] = torch.full_like(others[n // 2], 3.0)
    ff.ff_grad_norm(lst, stats, ws, 10.0, grads=others)
    torch.cuda.synchronize()
    _check_norm(stats, others, 10.0, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,v", [(5, 1003), (5, 40003), (300, 16011)])
@pytest.mark.parametrize("far", [60.0, 100.0, 200.0, 400.0])
def test_policy_slopes_beyond_32_bits(n, v, dtype, far):
    """A token that the policy had all but ruled out, or the reference had not: the slope passes the largest float, its products with small
    probabilities do not, and what is ruled out stays without a gradient."""
    rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, 17)
    y[:2] = 3
    rows[:2, v // 2:] = -INF
    rows[:2, 5:v // 3] = torch.linspace(-300.0, 0.0, v // 3 - 5).to(dtype)
    logp = rows.double().log_softmax(1).gather(1, y[:, None])[:, 0]
    old[0], ref[0] = float(logp[0] - far), float(logp[0])  # a ratio of exp(far), and a loss
    old[1], ref[1] = float(logp[1]), float(logp[1] + far)  # the KL term's slope
    adv[:2] = -1.0
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1)
    want = trainref.policy(rows, y, old, adv, w, ref, 0.2, 0.3, 0.1)
    g, x = got["dlogits"].double(), want["dlogits"]
    assert not torch.isnan(g).any() and bool((g[:2, v // 2:] == 0).all())
    # the slope follows the log-probability (v / 256 + 66 U32, and 4 U32 of what is added to it); the exponents of factor and distance
    # (up to 600 and 300) in 24 bits, a few roundings each; then the result's own
    fi = torch.finfo(dtype)
    floor = fi.smallest_normal * fi.eps / 2 if dtype == F16 else 2.0 ** -126
    err = x.abs() * (fi.eps / 2 + (v / 256 + 66 + 4 * far + 4 * 900) * U32) * 1.02 + floor
    most = float(fi.max)
    over = x.abs() > most * 1.01
    assert bool((torch.isinf(g[over]) & (torch.sign(g[over]) == torch.sign(x[over]))).all())
    close = (x.abs() < most * 0.99)
    assert bool(((g - x).abs() <= err)[close].all())
    assert far == 400 or int((close[:2] & (x[:2] != 0)).sum()) > 0
