"""The policy loss at what its sums owe their accuracy to, and without a gradient.

Bounds, from what is done to a row's sum of exponentials (U32 = 2^-24, half a step of 32 bits).  A term is 2^t with t rounded once: U32 of
|t| log(2) = far, the logit's distance from its thread's largest; log2(e) in 24 bits: 0.22 U32 of far; the instruction is good to
a unit in the last place: 2 U32.  Up to 16 terms are added in a tree of 32 bits: 4 U32.  (Of up to 1024 slots of 16 bytes, a row's terms
are added in 64.)  A thread's sum meets a factor whenever its largest logit rises, and one in the end, 2 U32 each; it adds twice, and once more for every 1024
slots and at the row's end.  The rest is in 64 bits."""
import math

import pytest
import torch

import trainref
from test_gpu_train import BF16, F16, F32, INF, U32, _policy_inputs, _run_policy

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "fp16", "fp32"])


def _items(dtype):
    return 4 if dtype == F32 else 8


def _check(got, rows, v, y, old, adv, w, ref, beta, loss_scale=1.0, sum_error=None):
    """sum_error: a row's sum's relative error, if the module's bound is not the point."""
    z = rows[:, :v].double()
    want = trainref.policy(z, y, old, adv, w, ref, 0.2, 0.3, beta, loss_scale)
    assert [got[k] for k in ("n_tokens", "n_clipped", "n_invalid")] == [want[k] for k in ("n_tokens", "n_clipped", "n_invalid")]
    far = torch.where(z == -INF, 0.0, z.masked_fill(z == -INF, -1e30).amax(1, keepdim=True) - z)
    probs = torch.where(want["used"][:, None], z.softmax(1), 0.0)
    if sum_error is None:
        sum_error = U32 * (6 + 2 * (4 + v / _items(rows.dtype) / 1024) + 1.25 * (probs * far).sum(1))
    used = want["used"]
    err = torch.where(used, sum_error + 1e-12 + U32 * want["logp"].abs(), 0.0)
    assert ((got["logp"].double() - want["logp"]).abs() <= err).all()
    # what hangs on the log-probability, in 64 bits: the loss follows its slope (the slope its own, where that is not over a border)
    slack = torch.where(used, (sum_error + 1e-12) * want["size"] * 1.01, 0.0)
    assert ((got["token_loss"].double() - want["token_loss"]).abs() <= slack + U32 * want["token_loss"].abs() + 1e-30).all()
    ww = w.double().abs()
    assert abs(got["loss"] - want["loss"]) <= float((ww * slack).sum()) * 1.01 + U32 * abs(want["loss"]) + 1e-30
    if got["dlogits"] is None:
        return want
    # a term over the sum (its own error, the sum's, three operations; 2^-18 of it where it is rounded to 16 bits), and the result's rounding
    fi = torch.finfo(rows.dtype)
    own = U32 * (8 + 2.5 * far) if rows.dtype == F32 else 2.0 ** -18 + U32 * (8 + 2.5 * far)
    x = want["dlogits"]
    hot = torch.zeros_like(probs)
    inside = (y >= 0) & (y < v)
    hot[torch.arange(len(y))[inside], y[inside]] = 1.0
    parts = (want["coef"] * (sum_error + 4 * U32))[:, None] * torch.maximum(probs, hot)
    floor = fi.smallest_normal * fi.eps / 2 if rows.dtype == F16 else 2.0 ** -126
    g = got["dlogits"].double()
    assert ((g - x).abs() <= x.abs() * (fi.eps / 2 * 1.01 + own) + parts * 1.01 + floor).all()
    return want


# on both sides of the rules by which rows without a gradient go, rows that four slots a thread hold and rows that they do not, and split ones
SCORED = [(5, 1), (20, 100), (20, 256), (20, 257), (40, 1024), (300, 1025), (300, 2048), (300, 2049), (66, 4096), (300, 4097), (257, 8191),
          (300, 8192), (300, 8193), (66, 4097), (200, 6250), (256, 12505), (65, 16385), (64, 4097), (7, 12505), (2, 65537)]


@TYPES
@pytest.mark.parametrize("n,slots", SCORED)
def test_scoring_alone(n, slots, dtype):
    v = slots * _items(dtype) + 3
    rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, n + slots, 1)
    last = (slots - 1) * _items(dtype)
    y[0], y[1] = v - 1, last  # behind the whole slots, and in the last one
    if n > 8:
        w[2] = 0
        y[3], y[4], y[5] = v, -1, last // 2
        rows[6, :v] = -INF
        rows[7, 3:v - 2] = -INF
        y[7] = v - 1
        logp = rows[7, :v].double().log_softmax(0)[v - 1]
        old[7], ref[7] = float(logp - 0.1), float(logp + 0.2)
    for k in (0, 1, 5 if n > 8 else 0):
        logp = rows[k, :v].double().log_softmax(0)[y[k]]
        old[k], ref[k] = float(logp - 0.1), float(logp + 0.2)
    for beta in (0.1, 0.0):
        r = ref if beta else None
        got = _run_policy(rows, v, y, old, adv, w, r, beta, grad=False)
        _check(got, rows, v, y, old, adv, w, r, beta)


@TYPES
@pytest.mark.parametrize("n,slots", [(5, 100), (40, 1000), (300, 1500), (600, 2500), (300, 5000), (300, 9001), (300, 15001), (66, 5000), (9, 9000)])
@pytest.mark.parametrize("at", [0.0, 80.0, 5000.0])
def test_sums_whose_largest_logit_is_large(n, slots, dtype, at):
    """Its product with log2(e) is rounded to 24 bits: 3e-6 of a logit of 80, 2e-4 of 5000, which what a sum of 1 stands for takes account of."""
    v = slots * _items(dtype) + 1
    rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, slots, 0)
    # 24-bit logits, as far as the type has them
    rows = (rows.double() + at + torch.linspace(0.0, 0.7, n).double()[:, None]).to(dtype)
    logp = rows.double().log_softmax(1).gather(1, y[:, None])[:, 0]
    change = torch.linspace(-0.6, 0.6, n).double() + 0.0101
    old, ref = (logp - change).float(), (logp + 0.3).float()
    scale = 64.0 if dtype == F16 else 1.0
    got = _run_policy(rows, v, y, old, adv, w, ref, 0.1, scale)
    _check(got, rows, v, y, old, adv, w, ref, 0.1, scale)


@TYPES
@pytest.mark.parametrize("n,slots", [(40, 60), (40, 256), (40, 1000), (300, 1000)])
def test_a_logit_that_stands_out_leaves_the_others_probability(n, slots, dtype):
    """Rows whose terms are added in 64 bits: the largest logit's own term is 1 to more than 32 bits, and the target's log-probability is that of
    the rest, a few parts in 10,000 here, to six digits; 32 bits would leave three."""
    v = slots * _items(dtype) + 1
    rows, y, old, ref, adv, w = _policy_inputs(n, v, dtype, slots, 0, spread=0.5)
    rows = rows.float()
    rows[torch.arange(n), y] = torch.linspace(14.0, 17.0, n)
    rows = rows.to(dtype)
    z = rows.double()
    logp = z.log_softmax(1).gather(1, y[:, None])[:, 0]
    old, ref = (logp - 0.05).float(), (logp + 0.1).float()
    rest = -torch.expm1(logp)
    assert 1e-7 < float(rest.min()) and float(rest.max()) < 0.02
    far = z.gather(1, y[:, None])[:, 0] - z.masked_fill(torch.nn.functional.one_hot(y, v) == 1, 0.0).amin(1)
    # the others' terms, each with the errors of a term; what the largest leaves, squared: (2^-19)^2
    bound = rest * U32 * (6 + 2 * 5 + 1.25 * far) + 2.0 ** -38
    for grad in (True, False):
        got = _run_policy(rows, v, y, old, adv, w, ref, 0.1, grad=grad)
        _check(got, rows, v, y, old, adv, w, ref, 0.1, sum_error=bound)
