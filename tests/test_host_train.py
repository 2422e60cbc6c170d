"""CPU-only checks of the calls between loss and step: what they refuse, and the sizes they report.  Every refusal
comes before any work on the device, so none of them needs one."""
import ctypes
import types
import weakref

import numpy as np
import pytest
import torch

from paper_2512_03644_amd import binding as ff

HOST = ff.FF_PLAN_HOST_ONLY
INF, NAN = float("inf"), float("nan")
A16 = 1 << 20  # an address that is aligned to everything and never used


def test_lists_count_elements_and_say_how_much_workspace_a_norm_takes():
    ts = [torch.zeros(n, dtype=t) for n, t in ((5, torch.bfloat16), (0, torch.float32), (100000, torch.float16),
                                                (3, torch.float32))]
    lst = ff.ff_grad_list(ts, HOST)
    assert lst.numel == 100008 and lst.workspace_bytes >= 16
    empty = ff.ff_grad_list([], HOST)
    assert empty.numel == 0 and empty.workspace_bytes >= 16
    many = ff.ff_grad_list([torch.zeros(3)] * 5000, HOST)  # several launches where every call brings its addresses
    assert many.numel == 15000 and many.workspace_bytes >= 16


def test_lists_refuse_what_is_no_gradient():
    L = ff.lib()
    out = ctypes.c_void_p()

    def status(field, value):
        segs = ff.make_segments([torch.zeros(8, dtype=torch.float32)])
        setattr(segs[0], field, value)
        rc = L.ff_grad_list_create(segs, 1, HOST, ctypes.byref(out))
        assert rc == ff.FF_OK or out.value is None
        if rc == ff.FF_OK:
            L.ff_grad_list_destroy(out)
        return rc

    assert status("dtype", 7) == ff.FF_ERR_INVALID and status("dtype", 0) == ff.FF_ERR_INVALID
    assert status("kind", ff.FF_KIND_M) == ff.FF_ERR_INVALID and status("reserved", 1) == ff.FF_ERR_INVALID
    assert status("nbytes", 30) == ff.FF_ERR_INVALID and status("ptr", A16 + 2) == ff.FF_ERR_INVALID
    assert status("ptr", None) == ff.FF_OK  # addresses may come with every call
    segs = ff.make_segments([torch.zeros(8)])
    assert L.ff_grad_list_create(segs, 1, HOST, None) == ff.FF_ERR_NULL
    assert L.ff_grad_list_create(None, 1, HOST, ctypes.byref(out)) == ff.FF_ERR_NULL
    assert L.ff_grad_list_create(segs, 1, HOST | 2, ctypes.byref(out)) == ff.FF_ERR_INVALID
    assert L.ff_grad_list_create(segs, 1 << 33, HOST, ctypes.byref(out)) == ff.FF_ERR_INVALID
    L.ff_grad_list_destroy(None)


def test_norm_and_clip_refuse_bad_arguments():
    L = ff.lib()
    lst = ff.ff_grad_list([torch.zeros(8), torch.zeros(0), torch.zeros(8, dtype=torch.bfloat16)], HOST)
    ok = (ctypes.c_uint64 * 3)(A16, 0, A16)

    def norm(handle=lst.handle, grads=ok, inv=1.0, most=1.0, ws=A16, stats=A16):
        return L.ff_grad_norm(handle, grads, inv, most, ws, stats, None)

    assert norm() == ff.FF_ERR_HOST_ONLY and norm(grads=None) == ff.FF_ERR_HOST_ONLY
    assert norm(most=INF) == ff.FF_ERR_HOST_ONLY
    assert norm(handle=None) == norm(ws=None) == norm(stats=None) == ff.FF_ERR_NULL
    for inv in (0.0, -1.0, INF, NAN, 1e300, 1e-300):
        assert norm(inv=inv) == ff.FF_ERR_INVALID
    for most in (0.0, -1.0, NAN):
        assert norm(most=most) == ff.FF_ERR_INVALID
    assert norm(ws=A16 + 8) == norm(stats=A16 + 4) == ff.FF_ERR_INVALID
    assert norm(grads=(ctypes.c_uint64 * 3)(A16, 0, 0)) == ff.FF_ERR_NULL
    assert norm(grads=(ctypes.c_uint64 * 3)(A16 + 2, 0, A16)) == ff.FF_ERR_INVALID   # fp32
    assert norm(grads=(ctypes.c_uint64 * 3)(A16, 1, A16 + 2)) == ff.FF_ERR_HOST_ONLY  # bf16; an empty one's is ignored
    assert norm(grads=(ctypes.c_uint64 * 3)(A16, 0, A16 + 1)) == ff.FF_ERR_INVALID
    assert L.ff_grad_clip(lst.handle, ok, A16, None) == ff.FF_ERR_HOST_ONLY
    assert L.ff_grad_clip(None, ok, A16, None) == L.ff_grad_clip(lst.handle, ok, None, None) == ff.FF_ERR_NULL
    assert L.ff_grad_clip(lst.handle, ok, A16 + 4, None) == ff.FF_ERR_INVALID
    segs = ff.make_segments([torch.zeros(8)])
    segs[0].ptr = None
    out = ctypes.c_void_p()
    assert L.ff_grad_list_create(segs, 1, HOST, ctypes.byref(out)) == ff.FF_OK
    assert norm(handle=out, grads=None) == L.ff_grad_clip(out, None, A16, None) == ff.FF_ERR_NULL
    L.ff_grad_list_destroy(out)

    def join(parts=A16, n=2, inv=1.0, most=1.0, stats=A16):
        return L.ff_grad_norm_join(parts, n, inv, most, stats, None)

    assert join(parts=None) == join(stats=None) == ff.FF_ERR_NULL
    for bad in (dict(n=0), dict(inv=0.0), dict(inv=NAN), dict(most=0.0), dict(most=NAN), dict(parts=A16 + 4),
                dict(stats=A16 + 4)):
        assert join(**bad) == ff.FF_ERR_INVALID, bad


def test_clipped_step_refuses_bad_arguments():
    L = ff.lib()
    t = [torch.zeros(64, dtype=torch.bfloat16)] + [torch.zeros(64) for _ in range(3)]
    plan = ff.ff_snapshot_plan(t, 1024, HOST, [1, 2, 3, 4], [0] * 4)
    hp = ff.ff_adam_hparams(3e-4, 0.9, 0.95, 1e-8, 0.1, 1)
    g = (ctypes.c_uint64 * 1)(A16)

    def step(handle=plan.handle, stats=A16):
        return L.ff_adam_step_clipped(handle, g, ctypes.byref(hp), stats, None, A16, A16, None)

    assert step() == ff.FF_ERR_HOST_ONLY
    assert step(handle=None) == step(stats=None) == ff.FF_ERR_NULL
    assert step(stats=A16 + 4) == ff.FF_ERR_INVALID


def _batch(**change):
    b = ff.ff_policy_batch(A16, 4, 100, 100, ff.FF_BF16, 0, A16, A16, A16, A16, A16, 0.2, 0.2, 0.1, 1.0)
    for k, v in change.items():
        setattr(b, k, v)
    return b


def test_policy_loss_refuses_bad_arguments():
    L = ff.lib()

    def loss(batch, logp=A16, token=A16, grad=None, stride=0, stats=A16, ws=A16):
        return L.ff_policy_loss(ctypes.byref(batch), logp, token, grad, stride, stats, ws, None)

    for name in ("logits", "targets", "old_logp", "advantages", "weights", "ref_logp"):
        assert loss(_batch(**{name: None})) == ff.FF_ERR_NULL, name
    for bad in (dict(logp=None), dict(token=None), dict(stats=None), dict(ws=None)):
        assert loss(_batch(), **bad) == ff.FF_ERR_NULL, bad
    assert L.ff_policy_loss(None, A16, A16, None, 0, A16, A16, None) == ff.FF_ERR_NULL
    for bad in (dict(dtype=0), dict(dtype=9), dict(reserved=1), dict(vocab=0), dict(vocab=1 << 31),
                dict(n_tokens=1 << 31), dict(row_stride=99), dict(logits=A16 + 1), dict(targets=A16 + 4),
                dict(old_logp=A16 + 2), dict(ref_logp=A16 + 2), dict(advantages=A16 + 1), dict(weights=A16 + 2),
                dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_low=NAN), dict(clip_high=-0.1),
                dict(clip_high=INF), dict(clip_high=NAN), dict(beta=-1.0), dict(beta=NAN), dict(beta=INF),
                dict(loss_scale=0.0), dict(loss_scale=INF), dict(loss_scale=NAN), dict(loss_scale=-1.0)):
        assert loss(_batch(**bad)) == ff.FF_ERR_INVALID, bad
    for bad in (dict(logp=A16 + 2), dict(token=A16 + 1), dict(stats=A16 + 4), dict(ws=A16 + 8),
                dict(grad=A16 + 1, stride=100), dict(grad=A16 + 64, stride=99), dict(grad=A16, stride=101)):
        assert loss(_batch(), **bad) == ff.FF_ERR_INVALID, bad


def test_binding_refuses_shapes_and_types():
    z, y = torch.zeros(4, 10, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    f = torch.zeros(4)
    ok = dict(logits=z, targets=y, old_logp=f, advantages=f, weights=f)
    b = ff.policy_batch(**ok)
    assert (b.n_tokens, b.vocab, b.row_stride, b.dtype) == (4, 10, 10, ff.FF_BF16)
    assert ff.policy_batch(**dict(ok, logits=torch.zeros(4, 16)[:, :10])).row_stride == 16
    for name, v in (("logits", z.t()), ("logits", z[0]), ("targets", y.int()), ("targets", y[:3]), ("old_logp", f.double()),
                    ("ref_logp", f[:2]), ("advantages", torch.zeros(8)[::2]), ("weights", torch.zeros(4, 1))):
        with pytest.raises(ValueError):
            ff.policy_batch(**dict(ok, **{name: v}))
    with pytest.raises(KeyError):
        ff.policy_batch(**dict(ok, logits=z.double()))
    for bad in (dict(logp=f.double()), dict(token_loss=f[:3]), dict(dlogits=z.float()), dict(dlogits=z[:3]),
                dict(dlogits=torch.zeros(10, 4, dtype=torch.bfloat16).t())):
        args = dict(dict(logp=f, token_loss=f, dlogits=None), **bad)
        with pytest.raises(ValueError):
            ff.ff_policy_loss(b, args["logp"], args["token_loss"], f, f, args["dlogits"])
    with pytest.raises(ValueError):
        ff.ff_grad_list([torch.zeros(4, 4).t()], HOST)


def test_binding_counts_gradients():
    lst = ff.ff_grad_list([torch.zeros(8), torch.zeros(3)], HOST)
    stats = ff.GradStats("cpu")
    with pytest.raises(ValueError):
        ff.ff_grad_norm(lst, stats, stats, grads=[torch.zeros(8)])
    with pytest.raises(ValueError):
        ff.ff_grad_clip(lst, stats, grads=[torch.zeros(8)] * 3)
    t = [torch.zeros(64, dtype=torch.bfloat16)] + [torch.zeros(64) for _ in range(3)]
    plan = ff.ff_snapshot_plan(t, 1024, HOST, [1, 2, 3, 4], [0] * 4)
    hp = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0, step=1)
    with pytest.raises(ValueError):
        ff.ff_adam_step_clipped(plan, [], hp, stats, t[1], t[1])


def test_binding_refuses_workspaces_that_are_too_small():
    lst = ff.ff_grad_list([torch.zeros(8), torch.zeros(3)], HOST)
    stats = ff.GradStats("cpu")
    with pytest.raises(ValueError):
        ff.ff_grad_norm(lst, stats, ff.alloc_grad_workspace(lst, "cpu")[:-1])
    with pytest.raises(ff.FFError):  # (a list without a device)
        ff.ff_grad_norm(lst, stats, ff.alloc_grad_workspace(lst, "cpu"), stream=types.SimpleNamespace(cuda_stream=0))
    for n, v in ((1, 8), (64, 300000), (65, 1000), (5000, 10)):
        rows = torch.zeros(n, v, dtype=torch.bfloat16)
        f = torch.zeros(n)
        b = ff.policy_batch(rows, torch.zeros(n, dtype=torch.int64), f, f, f)
        with pytest.raises(ValueError):
            ff.ff_policy_loss(b, f, f, ff.PolicyStats("cpu"), ff.alloc_policy_workspace(n, v, "cpu")[:-1])


def test_segments_are_filled_as_they_were():
    """Field by field, whatever the list: empty tensors have no address, kinds and groups as given."""
    ts = [torch.zeros(n, dtype=t) for n, t in ((5, torch.bfloat16), (0, torch.float32), (7, torch.float16), (3, torch.float32))]
    for kinds, ids in ((None, None), ([1, 0, 0, 2], [0, 0, 0xFFFFFFFF, 3])):
        segs = ff.make_segments(ts, kinds, ids)
        assert len(segs) == 4
        for k, (s, t) in enumerate(zip(segs, ts)):
            assert (s.ptr, s.nbytes) == (t.data_ptr() if t.numel() else None, t.numel() * t.element_size())
            assert s.dtype == {torch.bfloat16: ff.FF_BF16, torch.float16: ff.FF_F16, torch.float32: ff.FF_F32}[t.dtype]
            assert (s.kind, s.param_id, s.reserved) == (kinds[k] if kinds else 0, ids[k] if ids else 0, 0)
    none = ff.make_segments([])
    assert len(none) == 1 and (none[0].ptr, none[0].nbytes, none[0].dtype) == (None, 0, 0)
    with pytest.raises(ValueError, match="segment 1 "):
        ff.make_segments([ts[0], torch.zeros(4, 4).t()])


def test_a_policy_workspace_serves_every_smaller_call():
    """Sizes never fall with the tokens or the vocabulary: rows are split, and their parts stored, where there are few."""
    tokens = [0, 1, 2, 16, 63, 64, 65, 66, 100, 512, 4096, 1 << 20, (1 << 31) - 1]
    vocabs = [1, 8, 4096, 16384, 16385, 32000, 32769, 128256, 262144, 1 << 20, (1 << 31) - 1]
    sizes = [[ff.lib().ff_policy_workspace_bytes(n, v) for v in vocabs] for n in tokens]
    for row, more in zip(sizes, sizes[1:]):
        assert all(a <= b for a, b in zip(row, more))
    for row in sizes:
        assert row == sorted(row)


def test_a_policy_batch_keeps_its_tensors_alive():
    """Its addresses are read when the call comes: tensors that only the batch was given are not back with the allocator by then."""
    def make():
        z, y = torch.zeros(4, 10, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
        per_token = [torch.zeros(4) for _ in range(4)]
        return ff.policy_batch(z, y, *per_token), [weakref.ref(t) for t in (z, y, *per_token)]

    batch, kept = make()
    assert all(r() is not None for r in kept)
    assert {batch.logits, batch.targets, batch.old_logp, batch.advantages, batch.weights, batch.ref_logp} == {r().data_ptr() for r in kept}
    del batch
    assert all(r() is None for r in kept)


def test_lists_refuse_tensors_of_impossible_sizes():
    """Sizes that pass 64 bits when they are rounded up to items, and together."""
    L = ff.lib()
    out = ctypes.c_void_p()
    for dtype, sizes in ((ff.FF_F32, [2 ** 64 - 4]), (ff.FF_BF16, [2 ** 64 - 2]), (ff.FF_F32, [2 ** 64 - 8192]), (ff.FF_F32, [8, 2 ** 63]),
                         (ff.FF_F16, [2 ** 45]), (ff.FF_BF16, [2 ** 43, 2 ** 43 + 2])):
        segs = ff.make_segments([torch.zeros(2)] * len(sizes))
        for s, size in zip(segs, sizes):
            s.dtype, s.nbytes, s.ptr = dtype, size, A16
        assert L.ff_grad_list_create(segs, len(sizes), HOST, ctypes.byref(out)) == ff.FF_ERR_INVALID, sizes
        assert out.value is None


@pytest.mark.parametrize("kind", [int, np.uint8, np.int8, np.int32, np.uint32, np.int64, np.uint64, torch.tensor], ids=lambda k: k.__name__)
def test_segments_take_kinds_and_groups_of_any_integer_type(kind):
    """As they come out of an array: whatever has an index."""
    ts = [torch.zeros(4), torch.zeros(3, dtype=torch.bfloat16), torch.zeros(2)]
    kinds, ids = [1, 2, 4], [7, 0, 100]
    segs = ff.make_segments(ts, [kind(k) for k in kinds], [kind(k) for k in ids])
    assert [(s.dtype, s.kind, s.param_id, s.reserved) for s in segs] == [
        (ff.FF_F32, 1, 7, 0), (ff.FF_BF16, 2, 0, 0), (ff.FF_F32, 4, 100, 0)]
    if kind is not int:
        with pytest.raises(TypeError):
            ff.make_segments(ts, [1.0, 2.0, 3.0])
