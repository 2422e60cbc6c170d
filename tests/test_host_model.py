"""CPU-only checks of the operators at a model's two ends: what they refuse, the sizes they report, and the plain forms that
the GPU tests hold them to, against differences and closed forms."""
import ctypes
import math
import types
import weakref

import pytest
import torch

import modelref
from paper_2512_03644_amd import binding as ff

INF, NAN = float("inf"), float("nan")
A16 = 1 << 20  # an address that is aligned to everything and never used
BIG = 1 << 31
NOWHERE = types.SimpleNamespace(cuda_stream=0)
SHAPE = "is a |smaller"


def test_embedding_refuses_bad_arguments():
    L = ff.lib()

    def look(table=A16, vocab=10, width=8, stride=8, dtype=ff.FF_BF16, ids=A16, n=4, scale=1.0, out=3 * A16, out_stride=8):
        return L.ff_embed(table, vocab, width, stride, dtype, ids, n, scale, out, out_stride, None)

    def grad(dout=A16, stride=8, dtype=ff.FF_BF16, ids=A16, n=4, vocab=10, width=8, scale=1.0, dtable=3 * A16, out_stride=8, flags=0, ws=A16):
        return L.ff_embed_grad(dout, stride, dtype, ids, n, vocab, width, scale, dtable, out_stride, flags, ws, None)

    for f, names in ((look, ("table", "ids", "out")), (grad, ("dout", "ids", "dtable", "ws"))):
        for name in names:
            assert f(**{name: None}) == ff.FF_ERR_NULL, name
        for bad in (dict(dtype=0), dict(dtype=4), dict(vocab=0), dict(vocab=ff.FF_EMBED_MAX_VOCAB + 1), dict(width=0), dict(width=ff.FF_EMBED_MAX_WIDTH + 1, stride=1 << 30, out_stride=1 << 30),
                    dict(n=BIG), dict(stride=7), dict(out_stride=7), dict(stride=(1 << 40) + 1), dict(out_stride=1 << 60), dict(scale=INF), dict(scale=NAN),
                    {names[0]: A16 + 1}, {names[1]: A16 + 4}, {names[2]: A16 + 1}, {names[0]: 2 * A16, names[2]: 2 * A16}, {names[0]: A16 + 2, "dtype": ff.FF_F32}, {names[2]: A16 + 2, "dtype": ff.FF_F32}):
            assert f(**bad) == ff.FF_ERR_INVALID, bad
    assert grad(flags=2) == grad(ws=A16 + 8) == ff.FF_ERR_INVALID
    assert look(table=None, ids=None, out=None, n=0) == ff.FF_OK  # nothing to do
    assert grad(dout=None, ids=None, dtable=None, n=0, flags=ff.FF_GRAD_ADD) == ff.FF_OK
    assert grad(dout=None, ids=None, dtable=None, n=0) == ff.FF_ERR_NULL  # rows of zeros are wanted


def test_layer_norm_refuses_bad_arguments():
    L = ff.lib()

    def norm(x=A16, n=4, width=8, stride=8, dtype=ff.FF_BF16, weight=A16, bias=A16, eps=1e-5, out=2 * A16, out_stride=8, mean=A16, rstd=A16):
        return L.ff_layer_norm(x, n, width, stride, dtype, weight, bias, eps, out, out_stride, mean, rstd, None)

    def grad(x=A16, n=4, width=8, stride=8, dtype=ff.FF_BF16, weight=A16, mean=A16, rstd=A16, dy=3 * A16, dy_stride=8, out=2 * A16, out_stride=8, dw=4 * A16, db=5 * A16,
             ws=A16):
        return L.ff_layer_norm_grad(x, n, width, stride, dtype, weight, mean, rstd, dy, dy_stride, out, out_stride, dw, db, ws, None)

    for name in ("x", "weight", "out"):
        assert norm(**{name: None}) == grad(**{name: None}) == ff.FF_ERR_NULL, name
    for name in ("mean", "rstd", "dy", "ws"):
        assert grad(**{name: None}) == ff.FF_ERR_NULL, name
    wide = ff.FF_NORM_MAX_WIDTH + 1
    for bad in (dict(dtype=0), dict(dtype=9), dict(width=0), dict(width=wide, stride=wide, out_stride=wide), dict(n=BIG), dict(stride=7), dict(out_stride=7),
                dict(stride=1 << 60), dict(x=A16 + 1), dict(weight=A16 + 1), dict(out=A16 + 1), dict(mean=A16 + 2), dict(rstd=A16 + 1),
                dict(x=A16 + 2, dtype=ff.FF_F32)):
        assert norm(**bad) == ff.FF_ERR_INVALID, bad
        if "width" not in bad or bad["width"]:
            assert grad(**dict(bad, **({"dy_stride": wide} if bad.get("width") else {}))) == ff.FF_ERR_INVALID, bad
    for bad in (dict(eps=-1e-5), dict(eps=NAN), dict(eps=INF), dict(bias=A16 + 1), dict(out=A16, out_stride=16)):
        assert norm(**bad) == ff.FF_ERR_INVALID, bad
    for bad in (dict(dy_stride=7), dict(dy=A16 + 1), dict(dw=A16 + 1), dict(db=A16 + 1), dict(ws=A16 + 8), dict(out=3 * A16, out_stride=16),
                dict(out=A16, out_stride=16), dict(dw=A16), dict(db=A16)):
        assert grad(**bad) == ff.FF_ERR_INVALID, bad
    assert norm(x=None, out=None, n=0, mean=None, rstd=None) == ff.FF_OK


def _batch(**change):
    b = ff.ff_head_batch(A16, A16, 4, 100, 64, 64, 64, ff.FF_BF16, 0, A16, A16, 1.0, 0)
    for k, v in change.items():
        setattr(b, k, v)
    return b


def test_head_refuses_bad_arguments():
    L = ff.lib()

    def loss(batch, logp=A16, dh=None, dh_stride=0, dw=None, dw_stride=0, stats=A16, ws=A16):
        return L.ff_head_loss(ctypes.byref(batch), logp, dh, dh_stride, dw, dw_stride, stats, ws, None)

    for name in ("hidden", "weight", "targets", "weights"):
        assert loss(_batch(**{name: None})) == ff.FF_ERR_NULL, name
    for bad in (dict(logp=None), dict(stats=None), dict(ws=None)):
        assert loss(_batch(), **bad) == ff.FF_ERR_NULL, bad
    assert L.ff_head_loss(None, A16, None, 0, None, 0, A16, A16, None) == ff.FF_ERR_NULL
    for bad in (dict(dtype=0), dict(dtype=ff.FF_F32), dict(reserved=1), dict(vocab=0), dict(vocab=ff.FF_HEAD_MAX_VOCAB + 1), dict(n_tokens=ff.FF_HEAD_MAX_TOKENS + 1), dict(width=0),
                dict(width=65), dict(hidden_stride=63), dict(weight_stride=63), dict(weight_stride=1 << 60),
                dict(width=ff.FF_HEAD_MAX_WIDTH + 1, hidden_stride=1 << 20, weight_stride=1 << 20), dict(hidden=A16 + 1), dict(weight=A16 + 1), dict(targets=A16 + 4),
                dict(weights=A16 + 2), dict(loss_scale=0.0), dict(loss_scale=-1.0), dict(loss_scale=INF), dict(loss_scale=NAN)):
        assert loss(_batch(**bad)) == ff.FF_ERR_INVALID, bad
    for bad in (dict(logp=A16 + 2), dict(stats=A16 + 4), dict(ws=A16 + 16), dict(dh=A16 + 1, dh_stride=64), dict(dh=2 * A16, dh_stride=63),
                dict(dh=A16, dh_stride=72), dict(dw=2 * A16 + 1, dw_stride=64), dict(dw=2 * A16, dw_stride=63), dict(dw=A16, dw_stride=64)):
        assert loss(_batch(), **bad) == ff.FF_ERR_INVALID, bad
    assert L.ff_head_workspace_bytes(None, 1) == 0 and L.ff_head_workspace_bytes(ctypes.byref(_batch(dtype=ff.FF_F32)), 1) == 0


def test_workspaces_never_fall_with_any_size():
    L = ff.lib()
    tokens = [0, 1, 63, 64, 65, 128, 255, 256, 257, 1000, 1024, 2047, 2049, 4096, 100000, 1 << 20, 1 << 22]
    vocabs = [1, 255, 256, 257, 4099, 32000, 128256, 1 << 20]
    widths = [1, 8, 63, 64, 65, 256, 1000, 4096, 8192]
    for f in (lambda n, v, w: L.ff_embed_workspace_bytes(n, v, w), lambda n, v, w: L.ff_layer_norm_workspace_bytes(n, w) if v == 1 else 0):
        for v in vocabs:
            for w in widths:
                sizes = [f(n, v, w) for n in tokens]
                assert sizes == sorted(sizes)
        for n in tokens:
            for w in widths:
                sizes = [f(n, v, w) for v in vocabs[1:]]
                assert sizes == sorted(sizes)
    assert L.ff_layer_norm_workspace_bytes(4, ff.FF_NORM_MAX_WIDTH + 1) == L.ff_layer_norm_workspace_bytes(4, 0) == 0
    for aligned in (True, False):
        for grad in (0, 1):
            def size(n, v, w):
                b = _batch(n_tokens=n, vocab=v, width=w, hidden_stride=w, weight_stride=(w + 7) // 8 * 8 if aligned else w + 1)
                return L.ff_head_workspace_bytes(ctypes.byref(b), grad)
            for v in vocabs:
                for w in widths:
                    sizes = [size(n, v, w) for n in tokens]
                    assert sizes == sorted(sizes) and sizes[0] > 0, (v, w, grad)
            for n in tokens:
                for w in widths:
                    sizes = [size(n, v, w) for v in vocabs]
                    assert sizes == sorted(sizes), (n, w, grad)
                for v in vocabs:
                    sizes = [size(n, v, w) for w in ([8, 64, 256, 1000, 4096, 8192] if aligned else widths)]
                    assert sizes == sorted(sizes), (n, v, grad)


def test_binding_refuses_shapes_types_and_small_workspaces():
    bf, f, ids = torch.bfloat16, torch.zeros(4), torch.zeros(4, dtype=torch.int64)
    table, out = torch.zeros(10, 8, dtype=bf), torch.zeros(4, 8, dtype=bf)
    for args in ((table, ids.int(), out), (table, ids[::2], out), (table, ids, out.float()), (table, ids, out[:3]), (table.t(), ids, out), (table, ids, out[:, :7]),
                 (table[0], ids, out)):
        with pytest.raises(ValueError, match=SHAPE):
            ff.ff_embed(*args, stream=NOWHERE)
    with pytest.raises(ValueError, match="current"):  # the machine's own memory
        ff.ff_embed(table, ids, out, stream=NOWHERE)
    ws = ff.alloc_embed_workspace(4, 10, 8, "cpu")
    for args in ((out, ids, table, ws[:-1]), (out.float(), ids, table, ws), (out, ids[:3], table, ws), (out, ids, table.t(), ws)):
        with pytest.raises(ValueError, match=SHAPE):
            ff.ff_embed_grad(*args, stream=NOWHERE)
    with pytest.raises(ValueError, match="current"):
        ff.ff_embed_grad(out, ids, table, ws, stream=NOWHERE)
    w8 = torch.zeros(8, dtype=bf)
    for change in (dict(weight=w8.float()), dict(weight=w8[:7]), dict(bias=w8[:7]), dict(y=out.float()), dict(y=out[:3]), dict(mean=f.double()), dict(rstd=f[:3]), dict(x=out[0])):
        with pytest.raises(ValueError, match=SHAPE):
            ff.ff_layer_norm(**dict(dict(x=out, weight=w8, bias=w8, y=out), **change), stream=NOWHERE)
    with pytest.raises(ValueError, match="current"):
        ff.ff_layer_norm(out, w8, w8, out, stream=NOWHERE)
    ws = ff.alloc_norm_workspace(4, 8, "cpu")
    ok = dict(x=out, weight=w8, mean=f, rstd=f, dy=out, dx=out, dweight=w8, dbias=w8, workspace=ws)
    for change in (dict(workspace=ws[:-1]), dict(workspace=None), dict(dweight=w8.float()), dict(dbias=w8[:3]), dict(dy=out[:2]), dict(dx=out.float()), dict(mean=f[:3])):
        with pytest.raises(ValueError, match=SHAPE):
            ff.ff_layer_norm_grad(**dict(ok, **change), stream=NOWHERE)
    for change in (dict(), dict(dweight=None, dbias=None, workspace=None)):
        with pytest.raises(ValueError, match="current"):
            ff.ff_layer_norm_grad(**dict(ok, **change), stream=NOWHERE)
    b = ff.head_batch(out, table, ids, f, 2.0)
    assert (b.n_tokens, b.vocab, b.width, b.hidden_stride, b.weight_stride, b.dtype, b.loss_scale) == (4, 10, 8, 8, 8, ff.FF_BF16, 2.0)
    for args in ((out.t(), table, ids, f), (out, table.float(), ids, f), (out, table[:, :7], ids, f), (out, table, ids.int(), f), (out, table, ids, f[:3]), (out, table, ids, f.double())):
        with pytest.raises(ValueError, match=SHAPE):
            ff.head_batch(*args)
    stats, ws = ff.HeadStats("cpu"), ff.alloc_head_workspace(b, "cpu")
    for change in (dict(workspace=ws[:-1]), dict(logp=f[:3]), dict(dhidden=out.float()), dict(dhidden=out[:3]), dict(dweight=out), dict(dweight=table.t())):
        with pytest.raises(ValueError, match=SHAPE):
            ff.ff_head_loss(**dict(dict(batch=b, logp=f, stats=stats, workspace=ws, dhidden=out, dweight=table), **change), stream=NOWHERE)
    with pytest.raises(ValueError, match="current"):
        ff.ff_head_loss(b, f, stats, ws, stream=NOWHERE)


def test_a_head_batch_keeps_its_tensors_alive():
    def make():
        ts = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(10, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
        return ff.head_batch(*ts), [weakref.ref(t) for t in ts]

    batch, kept = make()
    assert {batch.hidden, batch.weight, batch.targets, batch.weights} == {r().data_ptr() for r in kept}
    del batch
    assert all(r() is None for r in kept)


# ---- the plain forms ------------------------------------------------------------------------------

def _difference(f, x, at, h=1e-6):
    """df/dx[at] in 64 bits."""
    a, b = x.clone(), x.clone()
    a[at] += h
    b[at] -= h
    return (f(a) - f(b)) / (2 * h)


def test_plain_head_is_its_differences():
    g = torch.Generator().manual_seed(0)
    h, w = torch.randn(5, 6, generator=g, dtype=torch.float64), torch.randn(9, 6, generator=g, dtype=torch.float64)
    y, weights = torch.tensor([0, 8, 3, -1, 9]), torch.tensor([0.5, 0.25, 0.0, 1.0, 1.0])
    modelref.HALF[torch.float64] = modelref.SMALL[torch.float64] = 0.0
    try:
        out = modelref.head(h, w, y, weights, 3.0)
        loss = lambda h, w: float(modelref.head(h, w, y, weights)["loss"])  # noqa: E731
        assert (out["n_tokens"], out["n_invalid"]) == (2, 2)
        for at in ((0, 0), (1, 5), (2, 1), (3, 3)):
            assert float(out["dhidden"][at]) == pytest.approx(3.0 * _difference(lambda x: loss(x, w), h, at), abs=1e-7)
        for at in ((0, 0), (8, 5), (4, 1)):
            assert float(out["dweight"][at]) == pytest.approx(3.0 * _difference(lambda x: loss(h, x), w, at), abs=1e-7)
    finally:
        del modelref.HALF[torch.float64], modelref.SMALL[torch.float64]
    z = h @ w.t()
    assert float(out["logp"][1]) == pytest.approx(float(z[1, 8] - z[1].exp().sum().log()))


def test_plain_norm_is_its_differences():
    g = torch.Generator().manual_seed(1)
    n, width = 3, 7
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((n, width), (width,), (width,), (n, width)))
    modelref.HALF[torch.float64] = modelref.SMALL[torch.float64] = 0.0
    try:
        f = lambda x, w, b: float((modelref.norm(x, w, b, 1e-5)["y"] * dy).sum())  # noqa: E731
        out = modelref.norm(x, w, b, 1e-5)
        grad = modelref.norm_grad(x, w, out["mean"], out["rstd"], dy)
        for at in ((0, 0), (1, 6), (2, 3)):
            assert float(grad["dx"][at]) == pytest.approx(_difference(lambda v: f(v, w, b), x, at), abs=1e-6)
        for k in range(width):
            assert float(grad["dweight"][k]) == pytest.approx(_difference(lambda v: f(x, v, b), w, k), abs=1e-6)
            assert float(grad["dbias"][k]) == pytest.approx(_difference(lambda v: f(x, w, v), b, k), abs=1e-6)
    finally:
        del modelref.HALF[torch.float64], modelref.SMALL[torch.float64]


def test_plain_embedding():
    table = torch.arange(12.0).view(4, 3)
    ids = torch.tensor([3, -1, 0, 3, 4])
    assert modelref.embed(table, ids, 2.0).tolist() == [[18.0, 20.0, 22.0], [0.0] * 3, [0.0, 2.0, 4.0], [18.0, 20.0, 22.0], [0.0] * 3]
    total, tol = modelref.embed_grad(torch.ones(5, 3), ids, 4, 2.0, table)
    assert total.tolist() == [[2.0, 3.0, 4.0], [3.0, 4.0, 5.0], [6.0, 7.0, 8.0], [13.0, 14.0, 15.0]]
    assert float(tol.max()) < 1e-5 and math.isfinite(float(tol.min()))


# ---- addresses that are an output's and another's ----------------------------------------------------

def _pairs(call, outputs, inputs, allowed):
    """Every output at every other output's and input's address, but for what is allowed; every other address its own."""
    names = outputs + inputs
    at = {name: (k + 2) * A16 for k, name in enumerate(names)}
    for k, out in enumerate(outputs):
        for other in outputs[k + 1:] + inputs:
            if (out, other) not in allowed:
                assert call(**dict(at, **{out: at[other]})) == ff.FF_ERR_INVALID, (out, other)


def test_outputs_at_the_addresses_of_others_are_refused():
    L = ff.lib()
    for dtype in (ff.FF_BF16, ff.FF_F32):
        _pairs(lambda table, ids, out: L.ff_embed(table, 10, 8, 8, dtype, ids, 4, 1.0, out, 8, None), ["out"], ["table", "ids"], ())
        for flags in (0, ff.FF_GRAD_ADD):
            _pairs(lambda dout, ids, dtable: L.ff_embed_grad(dout, 8, dtype, ids, 4, 10, 8, 1.0, dtable, 8, flags, A16, None), ["dtable"], ["dout", "ids"], ())
        _pairs(lambda x, weight, bias, y, mean, rstd: L.ff_layer_norm(x, 4, 8, 8, dtype, weight, bias, 1e-5, y, 8, mean, rstd, None),
               ["y", "mean", "rstd"], ["x", "weight", "bias"], [("y", "x")])
        _pairs(lambda x, weight, mean, rstd, dy, dx, dweight, dbias: L.ff_layer_norm_grad(x, 4, 8, 8, dtype, weight, mean, rstd, dy, 8, dx, 8, dweight, dbias, A16, None),
               ["dx", "dweight", "dbias"], ["x", "dy", "weight", "mean", "rstd"], [("dx", "x"), ("dx", "dy")])

    def loss(hidden, weight, targets, weights, logp, dhidden, dweight, stats):
        b = _batch(hidden=hidden, weight=weight, targets=targets, weights=weights)
        return L.ff_head_loss(ctypes.byref(b), logp, dhidden, 64, dweight, 64, stats, A16, None)

    _pairs(loss, ["dhidden", "dweight", "logp", "stats"], ["hidden", "weight", "targets", "weights"], [("dhidden", "hidden")])
    # what is not there is at no address, and arrays of no rows are nowhere either
    assert L.ff_layer_norm(None, 0, 8, 8, ff.FF_BF16, A16, A16, 1e-5, None, 8, None, None, None) == ff.FF_OK
    assert L.ff_layer_norm(A16, 0, 8, 8, ff.FF_BF16, A16, A16, 1e-5, A16, 8, A16, A16, None) == ff.FF_OK
    assert L.ff_embed(A16, 10, 8, 8, ff.FF_BF16, A16, 0, 1.0, A16, 8, None) == ff.FF_OK


def test_head_workspaces_are_within_what_is_documented():
    """The bound that ffsnap.h states, over all of the allowed range, corners included."""
    L, up = ff.lib(), lambda x, to: (x + to - 1) // to * to
    gib, mib = 1 << 30, 1 << 20
    nearest = 1.0
    for n in (0, 1, 16, 17, 20, 32, 33, 64, 65, 256, 300, 4096, 30000, 1 << 20, 1 << 21, (1 << 21) + 1, 3000000, 1 << 22):
        for vocab in (1, 300, 4099, 128256, 1 << 20, ff.FF_HEAD_MAX_VOCAB):
            for width in (1, 64, 72, 1000, 4096, 8192, ff.FF_HEAD_MAX_WIDTH):
                for grad in (0, 1):
                    for copied in (False, True):
                        b = _batch(n_tokens=n, vocab=vocab, width=width, hidden_stride=width, weight_stride=width + 1 if copied else up(width, 8))
                        copied = copied or width % 8 != 0
                        tiles, rows = up(vocab, 256) // 256, up(max(n, 1), 256)
                        bound = 40 * n + 8 * max(n * tiles, min(n, 32) * 4 * tiles) + (6 if grad else 2) * rows * up(width, 64) + 16 * mib + 4096
                        if grad:
                            bound += 128 * mib + max(3 * gib, 1536 * rows)
                        if copied:
                            bound += gib
                        size = L.ff_head_workspace_bytes(ctypes.byref(b), grad)
                        assert 0 < size <= bound, (n, vocab, width, grad, copied, size, bound)
                        nearest = min(nearest, 1 - size / bound)
    assert nearest < 0.01  # (it is no idle bound)


class _Elsewhere:
    """Stands for a tensor on a device: what the binding asks of one."""

    def __init__(self, *shape, dtype=torch.float32):
        self.dtype, self.shape, self.nbytes = dtype, shape, 1 << 40

    def get_device(self):
        return 5

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return A16


def test_binding_refuses_stats_in_host_memory_and_workspaces_that_only_look_large():
    bf = torch.bfloat16
    b = ff.head_batch(torch.zeros(4, 8, dtype=bf), torch.zeros(10, 8, dtype=bf), torch.zeros(4, dtype=torch.int64), torch.zeros(4))
    b.shapes = b.shapes[:-1] + (5,)
    with pytest.raises(ValueError, match="stats is a"):  # the kernel would write there
        ff.ff_head_loss(b, _Elsewhere(4), ff.HeadStats("cpu"), _Elsewhere(1 << 40), stream=NOWHERE)
    table, out, ids, w8, f = torch.zeros(10, 8, dtype=bf), torch.zeros(4, 8, dtype=bf), torch.zeros(4, dtype=torch.int64), torch.zeros(8, dtype=bf), torch.zeros(4)
    b = ff.head_batch(out, table, ids, f)
    one = torch.zeros(1, dtype=torch.uint8).expand(1 << 30)  # one byte
    for call in (lambda: ff.ff_embed_grad(out, ids, table, one, stream=NOWHERE), lambda: ff.ff_layer_norm_grad(out, w8, f, f, out, out, w8, None, one, stream=NOWHERE),
                 lambda: ff.ff_head_loss(b, f, ff.HeadStats("cpu"), one, stream=NOWHERE)):
        with pytest.raises(ValueError, match="workspace"):
            call()


def test_every_refusal_with_addresses_of_their_own():
    """One bad argument at a time, every array elsewhere."""
    L, null, bad = ff.lib(), ff.FF_ERR_NULL, ff.FF_ERR_INVALID
    P = [(k + 2) * A16 for k in range(10)]

    def check(call, ok, nulls, invalid):
        for name in nulls:
            assert call(**dict(ok, **{name: None})) == null, name
        for change in invalid:
            assert call(**dict(ok, **change)) == bad, change

    check(lambda x, n, width, stride, dtype, weight, bias, eps, y, y_stride, mean, rstd: L.ff_layer_norm(x, n, width, stride, dtype, weight, bias, eps, y, y_stride, mean, rstd, None),
          dict(x=P[0], n=4, width=8, stride=8, dtype=ff.FF_F32, weight=P[1], bias=P[2], eps=1e-5, y=P[3], y_stride=8, mean=P[4], rstd=P[5]), ["x", "weight", "y"],
          [dict(n=BIG), dict(width=0), dict(width=9), dict(width=ff.FF_NORM_MAX_WIDTH + 1, stride=1 << 20, y_stride=1 << 20), dict(stride=7), dict(y_stride=7), dict(dtype=0), dict(dtype=9),
           dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(x=P[0], y=P[0], y_stride=16)] + [{k: P[9] + 2} for k in ("x", "weight", "bias", "y", "mean", "rstd")])
    check(lambda x, n, width, stride, dtype, weight, mean, rstd, dy, dy_stride, dx, dx_stride, dw, db, ws:
          L.ff_layer_norm_grad(x, n, width, stride, dtype, weight, mean, rstd, dy, dy_stride, dx, dx_stride, dw, db, ws, None),
          dict(x=P[0], n=4, width=8, stride=8, dtype=ff.FF_F32, weight=P[1], mean=P[2], rstd=P[3], dy=P[4], dy_stride=8, dx=P[5], dx_stride=8, dw=P[6], db=P[7], ws=P[8]),
          ["x", "weight", "mean", "rstd", "dy", "dx", "ws"],
          [dict(n=BIG), dict(width=0), dict(stride=7), dict(dy_stride=7), dict(dx_stride=7), dict(dtype=3, width=9), dict(dx=P[0], dx_stride=16), dict(dx=P[4], dx_stride=16), dict(ws=P[8] + 8)] +
          [{k: P[9] + 2} for k in ("x", "weight", "mean", "rstd", "dy", "dx", "dw", "db")])

    def loss(logp, dh, dh_stride, dw, dw_stride, stats, ws, **batch):
        return L.ff_head_loss(ctypes.byref(_batch(**dict(dict(hidden=P[0], weight=P[1], targets=P[2], weights=P[3]), **batch))), logp, dh, dh_stride, dw, dw_stride, stats, ws, None)

    check(loss, dict(logp=P[4], dh=P[5], dh_stride=64, dw=P[6], dw_stride=64, stats=P[7], ws=P[8]), ["hidden", "weight", "targets", "weights", "logp", "stats", "ws"],
          [dict(hidden=P[9] + 1), dict(weight=P[9] + 1), dict(targets=P[9] + 4), dict(weights=P[9] + 2), dict(logp=P[9] + 2), dict(dh=P[9] + 1), dict(dw=P[9] + 1), dict(stats=P[9] + 4),
           dict(ws=P[9] + 128), dict(dh_stride=63), dict(dw_stride=63), dict(dh=P[0], dh_stride=72), dict(hidden_stride=63), dict(weight_stride=63), dict(reserved=1), dict(loss_scale=0.0),
           dict(loss_scale=NAN), dict(dtype=ff.FF_F32), dict(vocab=0), dict(width=0), dict(n_tokens=ff.FF_HEAD_MAX_TOKENS + 1), dict(vocab=ff.FF_HEAD_MAX_VOCAB + 1)])
