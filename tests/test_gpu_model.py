"""The operators at a model's two ends on the GPU against plain forms in 64 bits (modelref.py, which has the tolerances)."""
import math

import pytest
import torch

import modelref
from paper_2512_03644_amd import binding as ff

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALVES = pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
TYPES = pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "fp16", "fp32"])


def rows(n, width, dtype, gen, std=1.0, pad=0, first=0, fill=7.0):
    """n rows of normal values in an arena of `fill`, `pad` elements between them, `first` elements behind 16 bytes."""
    arena = torch.full((n * (width + pad) + first + 32,), fill, dtype=dtype, device=DEV)
    view = arena[8 + first:8 + first + n * (width + pad)].view(n, width + pad)[:, :width]
    if std:
        view.copy_(torch.randn(n, width, generator=gen, device=DEV) * std)
    return view, arena


def untouched(view, arena, fill=7.0):
    """Nothing but the view's elements has changed."""
    left = arena.clone()
    left.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(fill)
    assert bool((left == fill).all())


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


# ---- embedding ------------------------------------------------------------------------------------

def some_ids(n, vocab, g, kind):
    if kind == "same":
        return torch.full((n,), vocab // 2, device=DEV)
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    ids = (u * vocab).long() if kind == "even" else ((u * math.log(vocab)).exp() - 1).long()  # or as in text
    ids = ids.clamp_(0, vocab - 1)
    if n > 3:
        ids[::7] = -1
        ids[1] = vocab
        ids[2] = -(1 << 40)
        ids[3] = 1 << 40
    return ids


@TYPES
@pytest.mark.parametrize("n,vocab,width,pad,first,scale", [
    (1, 1, 1, 0, 0, 1.0), (1, 1000, 4096, 0, 0, 1.0), (5, 17, 7, 3, 1, 2.5), (100, 513, 512, 0, 0, -1.0), (33, 4099, 513, 1, 1, 16.03), (64, 5, 8, 8, 0, 0.0),
    (3001, 4099, 257, 3, 0, 16.0), (9, 40, 2000, 0, 3, 1e-3)])
def test_lookup_is_one_rounded_product(dtype, n, vocab, width, pad, first, scale):
    g = gen(1)
    table, _ = rows(vocab, width, dtype, g, 1.0, pad, first)
    ids = some_ids(n, vocab, g, "even")
    out, arena = rows(n, width, dtype, g, 0, pad, first)
    ff.ff_embed(table, ids, out, scale)
    torch.cuda.synchronize()
    want = modelref.embed(table.cpu(), ids.cpu(), scale)
    assert torch.equal(out.cpu(), want)
    untouched(out, arena)


@TYPES
@pytest.mark.parametrize("kind", ["even", "text", "same"])
@pytest.mark.parametrize("n,vocab,width,pad,first", [
    (1, 1, 1, 0, 0), (1, 1000, 64, 0, 0), (31, 3, 7, 3, 1), (32, 511, 512, 0, 0), (33, 512, 520, 0, 1), (500, 513, 1023, 1, 0), (3001, 4099, 257, 3, 0),
    (9000, 700, 40, 0, 0), (20000, 33, 16, 8, 0)])
def test_gradient_by_sorted_tokens(dtype, kind, n, vocab, width, pad, first):
    g = gen(2)
    ids = some_ids(n, vocab, g, kind)
    dout, _ = rows(n, width, dtype, g, 1.0, pad, first)
    ws = ff.alloc_embed_workspace(n, vocab, width, DEV).fill_(0xA5)
    for add in (False, True):
        dtable, arena = rows(vocab, width, dtype, g, 1.0 if add else 0, pad, first)
        start = dtable.clone() if add else None
        ff.ff_embed_grad(dout, ids, dtable, ws, 2.5, add)
        torch.cuda.synchronize()
        want, tol = modelref.embed_grad(dout, ids, vocab, 2.5, start)
        modelref.check(dtable, want, tol, "dtable")
        untouched(dtable, arena)
        if add:  # what no token asks for keeps its bits
            asked = torch.zeros(vocab, dtype=torch.bool, device=DEV)
            asked[ids[(ids >= 0) & (ids < vocab)]] = True
            assert torch.equal(dtable[~asked], start[~asked])
        first_bits = dtable.clone()
        if add:
            dtable.copy_(start)
        ff.ff_embed_grad(dout, ids, dtable, ws, 2.5, add)
        assert torch.equal(dtable, first_bits)  # the same bits every time


@TYPES
@pytest.mark.parametrize("kind", ["even", "text", "same"])
@pytest.mark.parametrize("n,vocab,width,pad,first", [(300, 40, 513, 0, 0), (9001, 300, 517, 1, 1), (5000, 64, 13, 0, 0), (4200, 33, 5, 0, 3), (6000, 2000, 1025, 0, 0)])
def test_gradient_of_rows_that_end_inside_a_lane(dtype, kind, n, vocab, width, pad, first):
    """The last elements lie with others in a lane, of the same wavefront or of another's."""
    test_gradient_by_sorted_tokens(dtype, kind, n, vocab, width, pad, first)


def test_embedding_of_nothing():
    table = torch.ones(4, 8, device=DEV)
    ids = torch.zeros(0, dtype=torch.int64, device=DEV)
    none = torch.zeros(0, 8, device=DEV)
    ws = ff.alloc_embed_workspace(0, 4, 8, DEV)
    ff.ff_embed(table, ids, none)
    ff.ff_embed_grad(none, ids, table, ws, add=True)
    assert bool((table == 1).all())
    ff.ff_embed_grad(none, ids, table, ws)
    assert bool((table == 0).all())
    table.fill_(3)
    ff.ff_embed_grad(torch.ones(3, 8, device=DEV), torch.full((3,), -1, device=DEV), table, ff.alloc_embed_workspace(3, 4, 8, DEV))
    assert bool((table == 0).all())


def test_padding_rows_may_hold_anything():
    table, dout = torch.ones(4, 8, device=DEV), torch.ones(3, 8, device=DEV)
    dout[1] = NAN
    ids = torch.tensor([2, -1, 2], device=DEV)
    ff.ff_embed_grad(dout, ids, table, ff.alloc_embed_workspace(3, 4, 8, DEV))
    assert table.tolist() == [[0.0] * 8, [0.0] * 8, [2.0] * 8, [0.0] * 8]


# ---- layer norm -------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (1, 4096), (3, 7), (5, 8), (70, 64), (33, 511), (40, 513), (20, 2048), (9, 2049), (7, 4097), (300, 1003), (5, 8192), (4, 8200), (3, 16384)]


def norm_inputs(n, width, dtype, pad, first, seed=3, offset=0.0):
    g = gen(seed)
    x, _ = rows(n, width, dtype, g, 1.5, pad, first)
    x += offset
    x[:, width // 2] += 20
    weight = (torch.randn(width, generator=g, device=DEV) * 0.3 + 1).to(dtype)
    bias = torch.randn(width, generator=g, device=DEV).to(dtype)
    dy, _ = rows(n, width, dtype, g, 1.0, pad, first)
    return x, weight, bias, dy, g


@TYPES
@pytest.mark.parametrize("n,width", NORM_SIZES, ids=lambda s: str(s))
@pytest.mark.parametrize("pad,first,with_bias", [(0, 0, True), (5, 1, False)])
def test_layer_norm_and_its_gradients(dtype, n, width, pad, first, with_bias):
    x, weight, bias, dy, g = norm_inputs(n, width, dtype, pad, first)
    bias = bias if with_bias else None
    y, arena = rows(n, width, dtype, g, 0, pad, first)
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ff.ff_layer_norm(x, weight, bias, y, mean, rstd, 1e-5)
    want = modelref.norm(x, weight, bias, 1e-5)
    for name, got in (("mean", mean), ("rstd", rstd), ("y", y)):
        modelref.check(got, want[name], want["tol_" + name], name)
    untouched(y, arena)
    dx, arena = rows(n, width, dtype, g, 0, pad, first)
    dw, db = torch.empty(width, dtype=dtype, device=DEV), torch.empty(width, dtype=dtype, device=DEV)
    ws = ff.alloc_norm_workspace(n, width, DEV).fill_(0xA5)
    ff.ff_layer_norm_grad(x, weight, mean, rstd, dy, dx, dw, db if with_bias else None, ws)
    want = modelref.norm_grad(x, weight, mean, rstd, dy)
    for name, got in (("dx", dx), ("dweight", dw)) + ((("dbias", db),) if with_bias else ()):
        modelref.check(got, want[name], want["tol_" + name], name)
    untouched(dx, arena)


@TYPES
def test_layer_norm_of_rows_far_from_zero_and_of_constant_rows(dtype):
    x, weight, bias, dy, _ = norm_inputs(6, 777, dtype, 0, 0, offset=300.0)
    x[2] = 5.0
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    ff.ff_layer_norm(x, weight, bias, y, mean, rstd, 1e-5)
    want = modelref.norm(x, weight, bias, 1e-5)
    keep = [0, 1, 3, 4, 5]
    for name, got in (("mean", mean), ("rstd", rstd), ("y", y)):
        modelref.check(got[keep], want[name][keep], want["tol_" + name][keep], name)
    assert bool((y[2] == bias).all()) and float(mean[2]) == 5.0 and float(rstd[2]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)


def test_layer_norm_in_place_and_without_statistics():
    x, weight, bias, dy, _ = norm_inputs(50, 1000, BF16, 8, 0)
    y, mean, rstd = torch.empty(50, 1000, dtype=BF16, device=DEV), torch.empty(50, device=DEV), torch.empty(50, device=DEV)
    ff.ff_layer_norm(x, weight, bias, y, mean, rstd)
    dx = torch.empty_like(y)
    ff.ff_layer_norm_grad(x, weight, mean, rstd, dy, dx)
    same = dy.clone()
    ff.ff_layer_norm_grad(x, weight, mean, rstd, same, same)
    assert torch.equal(same, dx)
    same = x.clone()
    ff.ff_layer_norm_grad(same, weight, mean, rstd, dy, same)
    assert torch.equal(same, dx)
    ff.ff_layer_norm(x, weight, bias, x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("n,width", [(1, 8), (50, 1000), (1024, 4096), (700, 16384), (1500, 300), (300, 9), (40, 1027), (2000, 513), (600, 8193), (1100, 8199), (20, 16383)])
@pytest.mark.parametrize("over", ["x", "dy"])
def test_layer_norm_gradients_of_weights_where_dx_replaces_its_inputs(over, n, width):
    x, weight, bias, dy, _ = norm_inputs(n, width, BF16, 0, 0)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ff.ff_layer_norm(x, weight, bias, y, mean, rstd)
    want = modelref.norm_grad(x, weight, mean, rstd, dy)
    dx, dw, db = (x if over == "x" else dy), torch.empty_like(weight), torch.empty_like(weight)
    ff.ff_layer_norm_grad(x, weight, mean, rstd, dy, dx, dw, db, ff.alloc_norm_workspace(n, width, DEV))
    for name, got in (("dx", dx), ("dweight", dw), ("dbias", db)):
        modelref.check(got, want[name], want["tol_" + name], name)


@pytest.mark.parametrize("n,width", [(3000, 64), (5000, 300), (2100, 2048)])
def test_layer_norm_of_many_rows_and_none(n, width):
    x, weight, bias, dy, _ = norm_inputs(n, width, F32, 0, 0)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ff.ff_layer_norm(x, weight, bias, y, mean, rstd)
    want = modelref.norm(x, weight, bias, 1e-5)
    modelref.check(y, want["y"], want["tol_y"], "y")
    dx, dw, db = torch.empty_like(x), torch.empty(width, device=DEV), torch.empty(width, device=DEV)
    ws = ff.alloc_norm_workspace(n, width, DEV)
    ff.ff_layer_norm_grad(x, weight, mean, rstd, dy, dx, dw, db, ws)
    want = modelref.norm_grad(x, weight, mean, rstd, dy)
    for name, got in (("dx", dx), ("dweight", dw), ("dbias", db)):
        modelref.check(got, want[name], want["tol_" + name], name)
    bits = dw.clone()
    ff.ff_layer_norm_grad(x, weight, mean, rstd, dy, dx, dw, db, ws)
    assert torch.equal(bits, dw)
    none = torch.empty(0, width, device=DEV)
    ff.ff_layer_norm(none, weight, bias, none)
    ff.ff_layer_norm_grad(none, weight, mean[:0], rstd[:0], none, none, dw, db, ws)
    assert bool((dw == 0).all()) and bool((db == 0).all())


# ---- head -------------------------------------------------------------------------------------------

def head_inputs(n, vocab, width, dtype, pad=0, first=0, masked=0.0, uneven=False, seed=4, std=None):
    g = gen(seed)
    weight, _ = rows(vocab, width, dtype, g, std or 1.5 / math.sqrt(width), pad, first, fill=NAN)
    hidden, _ = rows(n, width, dtype, g, 1.0, pad, first, fill=NAN)
    targets = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    weights = torch.full((n,), 1.0 / max(1, n), device=DEV)
    if uneven:
        weights *= torch.rand(n, generator=g, device=DEV) + 0.5
    off = torch.rand(n, generator=g, device=DEV) < masked
    weights[off] = 0.0
    hidden[off] = NAN  # not looked at
    return hidden, weight, targets, weights


def run_head(hidden, weight, targets, weights, scale=1.0, dh=True, dw=True, pad=0, first=0, ws=None):
    n, width = hidden.shape
    logp = torch.full((n,), 7.0, device=DEV)
    stats = ff.HeadStats(DEV)
    stats.words.fill_(-1)
    batch = ff.head_batch(hidden, weight, targets, weights, scale)
    if ws is None:
        ws = ff.alloc_head_workspace(batch, DEV, dh or dw).fill_(0xFF)  # NaNs
    out = dict(logp=logp, stats=stats)
    out["dhidden"], dh_arena = rows(n, width, hidden.dtype, None, 0, pad, first) if dh else (None, None)
    out["dweight"], dw_arena = rows(weight.shape[0], width, hidden.dtype, None, 0, pad, first) if dw else (None, None)
    ff.ff_head_loss(batch, logp, stats, ws, out["dhidden"], out["dweight"])
    torch.cuda.synchronize()
    if dh:
        untouched(out["dhidden"], dh_arena)
    if dw:
        untouched(out["dweight"], dw_arena)
    return out


def check_head(got, want):
    assert int(got["stats"].n_tokens) == want["n_tokens"] and int(got["stats"].n_invalid) == want["n_invalid"]
    for name in ("logp", "dhidden", "dweight"):
        if got[name] is not None:
            modelref.check(got[name], want[name], want["tol_" + name], name)
    modelref.check(got["stats"].loss, want["loss"], want["tol_loss"], "loss")


HEAD_SIZES = [(1, 1, 8), (1, 2, 1), (1, 1000, 64), (2, 257, 72), (3, 300, 65), (37, 4099, 256), (63, 511, 128), (64, 512, 192), (65, 513, 200), (130, 700, 31),
              (16, 129, 40), (17, 128, 264), (32, 1000, 520), (33, 130, 1001), (64, 3, 2056), (256, 256, 64), (257, 1025, 320), (300, 2000, 264), (600, 999, 100)]


@HALVES
@pytest.mark.parametrize("n,vocab,width", HEAD_SIZES, ids=lambda s: str(s))
@pytest.mark.parametrize("pad,first", [(0, 0), (8, 0), (3, 1)])
def test_head_over_sizes_and_strides(dtype, n, vocab, width, pad, first):
    args = head_inputs(n, vocab, width, dtype, pad, first)
    scale = 1024.0 if dtype == F16 else 1.0
    check_head(run_head(*args, scale, pad=pad, first=first), modelref.head(*args, scale))


@HALVES
@pytest.mark.parametrize("masked", [0.3, 0.97, 1.0])
@pytest.mark.parametrize("n", [5, 64, 300])
def test_head_leaves_masked_tokens_out(dtype, masked, n):
    args = head_inputs(n, 1500, 128, dtype, masked=masked, uneven=True)
    args[2][0] = -1
    args[2][min(3, n - 1)] = 1500
    args[3][0] = 0.25
    got = run_head(*args)
    check_head(got, modelref.head(*args))
    left = (args[3] == 0) | (args[2] < 0) | (args[2] >= 1500)
    assert bool((got["logp"][left] == 0).all()) and bool((got["dhidden"][left] == 0).all())


@HALVES
def test_head_gradients_one_at_a_time_and_scoring(dtype):
    args = head_inputs(100, 900, 136, dtype, masked=0.2)
    want = modelref.head(*args)
    both = run_head(*args)
    for dh, dw in ((True, False), (False, True), (False, False)):
        got = run_head(*args, dh=dh, dw=dw)
        check_head(got, want)
        assert torch.equal(got["logp"], both["logp"])
        for name in ("dhidden", "dweight"):
            if got[name] is not None:
                assert torch.equal(got[name], both[name])


def test_head_over_its_hidden_states():
    hidden, weight, targets, weights = head_inputs(300, 700, 96, BF16)
    weights[::3] = 0.0
    want = run_head(hidden, weight, targets, weights)
    batch = ff.head_batch(hidden, weight, targets, weights)
    logp = torch.empty(300, device=DEV)
    ff.ff_head_loss(batch, logp, ff.HeadStats(DEV), ff.alloc_head_workspace(batch, DEV), hidden)
    assert torch.equal(hidden, want["dhidden"]) and torch.equal(logp, want["logp"])


def test_head_of_nothing():
    weight = torch.ones(300, 64, dtype=BF16, device=DEV)
    none = torch.empty(0, 64, dtype=BF16, device=DEV)
    got = run_head(none, weight, torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV))
    assert bool((got["dweight"] == 0).all()) and got["stats"].words.tolist() == [0, 0, 0]
    got = run_head(none, weight, torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV), dh=False, dw=False)
    assert got["stats"].words.tolist() == [0, 0, 0]


@HALVES
def test_head_of_large_logits(dtype):
    """Targets far above and far below the others."""
    hidden, weight, targets, weights = head_inputs(64, 600, 64, dtype, std=0.5)
    for t in range(64):
        hidden[t] = weight[targets[t]] * (8.0 if t % 2 else -8.0)
    args = (hidden, weight, targets, weights)
    check_head(run_head(*args), modelref.head(*args))


def test_head_with_a_logit_that_is_not_finite():
    hidden, weight, targets, weights = head_inputs(40, 600, 64, BF16)
    weight[77, 3] = NAN
    got = run_head(hidden, weight, targets, weights)
    assert bool(torch.isnan(got["logp"]).all()) and math.isnan(float(got["stats"].loss))
    hidden, weight, targets, weights = head_inputs(40, 600, 64, BF16)
    hidden[5, 0] = INF
    got = run_head(hidden, weight, targets, weights)
    clean = torch.arange(40, device=DEV) != 5
    assert bool(torch.isnan(got["logp"][5])) and bool(torch.isfinite(got["logp"][clean]).all())
    assert bool(torch.isfinite(got["dhidden"][clean]).all()) and not bool(torch.isfinite(got["dhidden"][5]).any())


@HALVES
@pytest.mark.parametrize("n,vocab,width,pad,first", [(1000, 20011, 512, 0, 0), (2048, 8000, 1000, 8, 0), (16, 50021, 1032, 0, 0), (60, 50021, 777, 3, 1), (520, 22000, 72, 1, 0),
                                                     (257, 33000, 1096, 0, 1)])
def test_head_at_larger_sizes(dtype, n, vocab, width, pad, first):
    """In several workgroups along every axis, of either height; the reference on the GPU, in 64 bits."""
    args = head_inputs(n, vocab, width, dtype, pad, first, masked=0.1)
    scale = 1024.0 if dtype == F16 else 1.0
    check_head(run_head(*args, scale, pad=pad, first=first), modelref.head(*args, scale))


@HALVES
@pytest.mark.parametrize("n,vocab,width,pad,first", [(40000, 14000, 1032, 0, 0), (30011, 18000, 136, 8, 0), (70, 9000, 65528, 3, 1), (20, 9000, 65528, 3, 1)])
def test_head_in_several_pieces_of_the_vocabulary(dtype, n, vocab, width, pad, first):
    """Of logits, the last of which are kept or not, and of copied rows."""
    args = head_inputs(n, vocab, width, dtype, pad, first, masked=0.1)
    scale = 1024.0 if dtype == F16 else 1.0
    check_head(run_head(*args, scale, pad=pad, first=first), modelref.head(*args, scale))


FEW_TILES = [(21, 1240, 8128, 0, 0), (130, 700, 4096, 8, 0), (300, 256, 2000, 3, 1), (1500, 300, 1100, 0, 0), (2, 1689, 2578, 0, 0), (64, 4099, 2056, 0, 3), (17, 1, 1024, 0, 0), (1300, 500, 333, 3, 1)]


@HALVES
@pytest.mark.parametrize("n,vocab,width,pad,first", FEW_TILES)
def test_head_of_few_tiles_and_long_sums(dtype, n, vocab, width, pad, first):
    """The logits' sums in slices; with gradients and scored, masks that leave no token in."""
    args = head_inputs(n, vocab, width, dtype, pad, first, masked=0.2)
    scale = 1024.0 if dtype == F16 else 1.0
    want = modelref.head(*args, scale)
    both = run_head(*args, scale, pad=pad, first=first)
    check_head(both, want)
    scored = run_head(*args, scale, dh=False, dw=False)
    modelref.check(scored["logp"], want["logp"], want["tol_logp"], "logp")
    modelref.check(scored["stats"].loss, want["loss"], want["tol_loss"], "loss")
    again = run_head(*args, scale, pad=pad, first=first)
    assert all(torch.equal(both[k], again[k]) for k in ("logp", "dhidden", "dweight"))
    args[3].zero_()
    for grad in (True, False):
        got = run_head(*args, scale, dh=grad, dw=grad)
        assert bool((got["logp"] == 0).all()) and got["stats"].words.tolist() == [0, 0, 0]
        assert not grad or bool((got["dhidden"] == 0).all() and (got["dweight"] == 0).all())


def test_head_of_few_tiles_with_a_logit_that_is_not_finite_and_large_ones():
    hidden, weight, targets, weights = head_inputs(40, 600, 2048, BF16)
    hidden[5, 0] = INF
    hidden[6] = weight[targets[6]] * 200.0
    hidden[7] = weight[targets[7]] * -200.0
    clean = torch.arange(40, device=DEV) != 5
    got = run_head(hidden, weight, targets, weights)
    assert bool(torch.isnan(got["logp"][5])) and not bool(torch.isfinite(got["dhidden"][5]).any()) and math.isnan(float(got["stats"].loss))
    want = modelref.head(hidden[clean], weight, targets[clean], weights[clean])
    for name in ("logp", "dhidden"):
        modelref.check(got[name][clean], want[name], want["tol_" + name], name)


@HALVES
@pytest.mark.parametrize("vocab,width,pad,first", [(300, 65, 0, 0), (4099, 64, 3, 1), (1, 1, 0, 0), (9000, 65521, 0, 0)])
def test_head_of_nothing_on_rows_that_would_be_copied(dtype, vocab, width, pad, first):
    """Of widths and strides at which W's rows are copied for tokens; W may be absent."""
    weight, _ = rows(vocab, width, dtype, gen(8), 1.0, pad, first)
    none = torch.empty(0, width, dtype=dtype, device=DEV)
    ids, weights = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    got = run_head(none, weight, ids, weights, pad=pad, first=first)
    assert bool((got["dweight"] == 0).all()) and got["stats"].words.tolist() == [0, 0, 0]
    batch = ff.head_batch(none, weight, ids, weights)
    batch.weight = None
    dweight, arena = rows(vocab, width, dtype, None, 0, pad, first)
    stats = ff.HeadStats(DEV)
    stats.words.fill_(-1)
    ff.ff_head_loss(batch, weights, stats, ff.alloc_head_workspace(batch, DEV), dweight=dweight)
    torch.cuda.synchronize()
    assert bool((dweight == 0).all()) and stats.words.tolist() == [0, 0, 0]
    untouched(dweight, arena)


@TYPES
@pytest.mark.parametrize("width", [15, 41, 107, 777, 1003, 2049, 4097, 5000, 8191, 16383])
def test_rows_of_one_value_are_the_bias_and_have_no_gradient(dtype, width):
    """Of few bits: their sum is exact, and so is its quotient.  rstd is eps's alone, 316."""
    values = torch.tensor([5.0, 300.0, 1000.0, 20000.0], device=DEV)
    assert bool((values.to(dtype) == values.to(torch.float32)).all()) or dtype == BF16
    x = values.to(dtype)[:, None].repeat(1, width)
    weight, bias = torch.ones(width, dtype=dtype, device=DEV), torch.randn(width, generator=gen(9), device=DEV).to(dtype)
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    ff.ff_layer_norm(x, weight, bias, y, mean, rstd)
    assert torch.equal(y, bias[None].repeat(4, 1)) and torch.equal(mean, x[:, 0].float())
    ff.ff_layer_norm_grad(x, weight, mean, rstd, x, dx)
    assert bool((dx == 0).all())
