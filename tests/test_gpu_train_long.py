"""The clipped step where it has other kernels than on the smallest lists: over more than 80 MiB, through the image in LDS, without a
tally, in several launches, in every room for the gradients' addresses; bytes against the plain form on the CPU (trainref.py)."""
import math

import numpy as np
import pytest
import torch

import trainref
from paper_2512_03644_amd import binding as ff
from paper_2512_03644_amd import workloads as wl
from test_gpu_step_blocks import EDGES, SHORT_STEP
from test_gpu_train import BF16, DEV, F16, HP, INF, NAN, _check_norm, _same

pytestmark = pytest.mark.gpu

# every edge 69 times (two launches, no tally), a large parameter among the edges behind cuts of several kinds (with a tally and, from
# 2560 workgroups on, without), all on the lines, and one chunk
LONG = [(EDGES * 69, 1 << 15), (EDGES + [6000001, 4096 * 3 + 512, 150001], 1 << 15), (EDGES + [6000001, 4096 * 3 + 512, 150001], 1 << 22),
        (EDGES + [10500001, 4096 * 3 + 512, 150001], 1 << 17), ([1 << 20] * 6 + [262144], 1 << 20), (EDGES, 1 << 27)]


def _clipped_and_compare(oracle, numels, chunk, half, chained, skip, raw=(), stream=None, max_norm=None):
    """raw: (how many segments of the parameters are in front of it, tensor) each."""
    loss_scale = 1024.0 if half == F16 else 1.0
    shard = wl.param_shard("s", numels, chunk, len(numels) + chunk, DEV, with_grads=True, half=half, loss_scale=loss_scale)
    four = [ff.FF_KIND_W16, ff.FF_KIND_MASTER, ff.FF_KIND_M, ff.FF_KIND_V]
    segs, kinds, ids, host_raw = list(shard.segments), four * len(numels), [k // 4 for k in range(4 * len(numels))], []
    for at, t in sorted(raw, key=lambda x: -x[0]):
        segs.insert(at, t)
        kinds.insert(at, ff.FF_KIND_RAW)
        ids.insert(at, 0)
    plan = ff.ff_snapshot_plan(segs, chunk, 0, kinds, ids)
    chunks, crcs, _, _ = ff.alloc_outputs(plan, DEV)
    chunks.fill_(0xA5)
    grads = [q.grad for q in shard.params]
    if skip:
        grads[len(grads) // 2][-1] = -INF
        shard.params[-1].master[0] = NAN
    lst = ff.ff_grad_list(grads)
    stats, ws = ff.GradStats(DEV), ff.alloc_grad_workspace(lst, DEV)
    old = [[t.clone() for t in (q.w16, q.master, q.m, q.v)] for q in shard.params]
    prev = None
    if chained:
        prev, prev_crcs, _, _ = ff.alloc_outputs(plan, DEV)
        ff.ff_pack(plan, prev, prev_crcs)
        torch.cuda.synchronize()
        for q in shard.params:
            for t in (q.w16, q.master, q.m, q.v):
                t.view(torch.uint8).fill_(0x5A)
    if max_norm is None:
        max_norm = 1e-4 * math.sqrt(sum(numels))
    torch.cuda.synchronize()
    ff.ff_grad_norm(lst, stats, ws, max_norm, 1 / loss_scale, stream=stream)
    ff.ff_adam_step_clipped(plan, grads, HP, stats, chunks, crcs, prev, stream=stream)
    torch.cuda.synchronize()
    _check_norm(stats, grads, max_norm, 1 / loss_scale)
    assert int(stats.skip) == int(skip) and (skip or float(stats.scale) < 1 / loss_scale)
    new = [trainref.step(*o, g, HP, float(stats.scale), skip) for o, g in zip(old, grads)]
    flat = [x for n in new for x in (n[0].view(torch.int16).numpy(), *n[1:])]
    for at, t in sorted(raw, key=lambda x: -x[0]):
        flat.insert(at, t.cpu().view(torch.int16).numpy())
    buf, want = oracle.pack(flat, chunk, threads=4)
    assert np.array_equal(chunks.cpu().numpy(), buf)
    assert np.array_equal(crcs.cpu().numpy().view(np.uint32), want)
    for q, n in zip(shard.params, new):
        assert _same(q.w16, n[0])
        for t, x in zip((q.master, q.m, q.v), n[1:]):
            assert bool((t.view(torch.uint8) == 0x5A).all()) if chained else _same(t, x)


@pytest.mark.parametrize("half", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("numels,chunk", LONG, ids=lambda x: "%dx" % len(x) if isinstance(x, list) else str(x))
@pytest.mark.parametrize("chained", [False, True], ids=["inplace", "chained"])
@pytest.mark.parametrize("skip", [False, True], ids=["update", "skip"])
def test_clipped_step_over_more_than_80_mib(numels, chunk, half, chained, skip, oracle):
    assert max(14 * sum(numels), chunk) > SHORT_STEP
    _clipped_and_compare(oracle, numels, chunk, half, chained, skip)


@pytest.mark.parametrize("half", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("chained", [False, True], ids=["inplace", "chained"])
def test_long_clipped_step_copies_tensors_that_are_not_trained(half, chained, oracle):
    g = torch.Generator().manual_seed(12)
    raw = [(5 * i, torch.randn(n, generator=g).to(BF16).to(DEV)) for i, n in enumerate([1, 7, 511, 4096, 16385 + 4096])]
    _clipped_and_compare(oracle, EDGES * 69, 1 << 15, half, chained, False, raw)
    _clipped_and_compare(oracle, EDGES, 1 << 27, half, chained, True, raw)


@pytest.mark.parametrize("chained", [False, True], ids=["inplace", "chained"])
def test_long_clipped_step_on_another_stream(chained, oracle):
    _clipped_and_compare(oracle, EDGES + [6000001, 4096 * 3 + 512, 150001], 1 << 22, BF16, chained, False, stream=torch.cuda.Stream())


# one room for the gradients' addresses, the next, a launch's end and further launches
@pytest.mark.parametrize("n", [64, 65, 384, 385, 2047, 2048, 2049, 4100])
@pytest.mark.parametrize("chained", [False, True], ids=["inplace", "chained"])
def test_clipped_step_of_so_many_groups(n, chained, oracle):
    numels = torch.randint(1, 40, (n,), generator=torch.Generator().manual_seed(n)).tolist()
    for half in (BF16, F16):
        _clipped_and_compare(oracle, numels, 1 << 14, half, chained, False)
    _clipped_and_compare(oracle, numels, 1 << 14, BF16, chained, True)
