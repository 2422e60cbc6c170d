"""Plain forms of the operators at a model's two ends, in 64 bits, each with how far a computation in 32 bits may be from it.

U32 is half a step of 32 bits relative to the value, HALF[t] that of a format.  A sum of n terms in any order is off by at most n U32 times
the sum of their magnitudes; products of 16-bit values are exact in 32 bits."""
import torch

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: U32}
# half of the smallest step of a format
SMALL = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def head(hidden, weight, targets, weights, loss_scale=1.0):
    """Outputs of the head's loss with their tolerances; rows that are left out are not looked at."""
    t = hidden.dtype
    n, (vocab, width) = hidden.shape[0], weight.shape
    used = (weights != 0) & (targets >= 0) & (targets < vocab)
    at = used.nonzero()[:, 0]
    h, table, y, w = hidden[at].double(), weight.double(), targets[at], weights[at].double()
    z = h @ table.t()
    off = (width + 2) * U32 * (h.abs() @ table.abs().t()).amax(1)  # of any logit of the row
    logp_all = z.log_softmax(1)
    row = torch.arange(len(at), device=z.device)
    logp = logp_all[row, y]
    # of a term of the sum, relative: its logit's, and the exponential of a rounded argument
    term = off + U32 * (8 + 4 * z.abs().amax(1)) if len(at) else off
    probs = logp_all.exp()
    g = probs.clone()
    g[row, y] = torch.expm1(logp)
    c = w * loss_scale
    g = g * c[:, None]
    # a term's error, the target's as that of its probability; G's rounding; the factors' (three rounded operations)
    dg = probs * (2 * term * c.abs())[:, None] + g.abs() * (HALF[t] + 4 * U32)
    if t == torch.float16 and len(at):
        dg = dg + c.abs().amax() * 2.0 ** -39  # steps of what is smallest in G
    dh, dw = g @ table, g.t() @ h
    tol_h = dg @ table.abs() + vocab * U32 * (g.abs() @ table.abs()) + (HALF[t] + U32) * dh.abs() + SMALL[t]
    tol_w = dg.t() @ h.abs() + len(at) * U32 * (g.abs().t() @ h.abs()) + (HALF[t] + U32) * dw.abs() + SMALL[t]
    wide = lambda x: torch.zeros(n, *x.shape[1:], dtype=torch.float64, device=x.device).index_copy_(0, at, x)  # noqa: E731
    tol_logp = off + term + U32 * logp.abs() + 1e-300
    loss = -(w * logp).sum()
    return dict(loss=loss, tol_loss=(w.abs() * (tol_logp + U32 * logp.abs())).sum() + U32 * loss.abs(), logp=wide(logp), tol_logp=wide(tol_logp),
                n_tokens=len(at), n_invalid=int(((weights != 0) & ~used).sum()), dhidden=wide(dh), tol_dhidden=wide(tol_h), dweight=dw, tol_dweight=tol_w)


def embed(table, ids, scale):
    """One product in 32 bits, rounded: bits have one value."""
    inside = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(inside, ids, 0)].float() * torch.tensor(scale, dtype=torch.float32)
    return torch.where(inside[:, None], rows, torch.zeros(())).to(table.dtype)


def embed_grad(dout, ids, vocab, scale, start=None):
    """(gradient of the table, tolerance); start: what it is added to."""
    inside = (ids >= 0) & (ids < vocab)
    at, rows = ids[inside], dout[inside].double()
    scale = float(torch.tensor(scale, dtype=torch.float32))
    total = torch.zeros(vocab, dout.shape[1], dtype=torch.float64, device=dout.device).index_add_(0, at, rows) * scale
    size = torch.zeros_like(total).index_add_(0, at, rows.abs()) * abs(scale)
    most = int(torch.bincount(at, minlength=1).max()) if len(at) else 0
    tol = (most + 2) * U32 * size
    if start is not None:
        total = total + start.double()
        tol = tol + U32 * total.abs()
    return total, tol + HALF[dout.dtype] * (total.abs() + tol) + SMALL[dout.dtype]


_ADDS = 48  # one after the other in a row's sum: of a thread 3 + K, of a wavefront 6, of its group 16, and what is done to a term


def norm(x, weight, bias, eps):
    t, x = x.dtype, x.double()
    w = weight.double()
    b = bias.double() if bias is not None else torch.zeros_like(w)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    mean = x.mean(1)
    d = x - mean[:, None]
    var = d.square().mean(1)
    rstd = 1.0 / (var + eps).sqrt()
    xh = d * rstd[:, None]
    y = xh * w + b
    tol_mean = _ADDS * U32 * x.abs().mean(1) + SMALL[torch.float32]
    tol_d = tol_mean[:, None] + U32 * d.abs()
    # relative: of a sum of squares of what is off by tol_d, halved by the root, and the root and division themselves
    tol_rstd = ((2 * d.abs() * tol_d + tol_d.square()).mean(1) / (var + eps) / 2 + _ADDS * U32)
    tol_y = w.abs() * (rstd[:, None] * tol_d + xh.abs() * (tol_rstd[:, None] + 4 * U32)) * 1.01 + U32 * y.abs()
    return dict(y=y, tol_y=tol_y + HALF[t] * (y.abs() + tol_y) + SMALL[t], mean=mean, tol_mean=tol_mean, rstd=rstd, tol_rstd=tol_rstd * rstd * 1.01)


def norm_grad(x, weight, mean, rstd, dy):
    """From the statistics as they are given."""
    t, x, w, dy = x.dtype, x.double(), weight.double(), dy.double()
    n, width = x.shape
    r = rstd.double()[:, None]
    xh = (x - mean.double()[:, None]) * r
    g = dy * w
    c0, c1 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - c0 - xh * c1)
    tol = r * U32 * (4 * g.abs() + _ADDS * g.abs().mean(1, keepdim=True) + xh.abs() * (_ADDS + 8) * (g * xh).abs().mean(1, keepdim=True)) * 1.01
    out = dict(dx=dx, tol_dx=tol + HALF[t] * (dx.abs() + tol) + SMALL[t])
    for name, terms in (("dweight", dy * xh), ("dbias", dy)):
        total, size = terms.sum(0), terms.abs().sum(0)
        tol = (n + 8) * U32 * size
        out[name], out["tol_" + name] = total, tol + HALF[t] * (total.abs() + tol) + SMALL[t]
    return out


def check(got, want, tol, what=""):
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    off = (got - want).abs()
    bad = ~(off <= tol.cpu())
    if bad.any():
        k = int(torch.where(torch.isnan(off), torch.inf, off / tol.cpu()).argmax())
        raise AssertionError("%s: %d of %d are off; at %d got %r, want %r, tolerance %r" % (
            what, int(bad.sum()), bad.numel(), k, got.reshape(-1)[k].item(), want.reshape(-1)[k].item(), tol.reshape(-1)[k].item()))
