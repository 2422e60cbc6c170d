"""Plain forms of the calls between loss and step, on the CPU: sums and the policy loss in 64 bits; the update in
separately rounded 32-bit operations, whose bytes have one value."""
import math

import numpy as np
import torch


def sum_of_squares(tensors):
    """Of the finite elements' squares, correctly rounded; and how many are not finite."""
    sums, bad = [], 0
    for t in tensors:
        x = t.detach().cpu().double().reshape(-1).numpy()
        bad += int((~np.isfinite(x)).sum())
        sums.append(math.fsum((x * x).tolist()))
    return math.fsum(sums), bad


def factor(norm, inv_scale, max_norm):
    return min(1.0, max_norm / norm) * inv_scale if norm > 0 else inv_scale


def clipped(t, scale):
    """t * scale in fp32, rounded to t's format."""
    x = t.detach().cpu().float().numpy() * np.float32(scale)
    return torch.from_numpy(x).to(t.dtype)


NAN32 = np.float32(np.uint32(0x7FC00000).view(np.float32))


def _canonical(x):
    return np.where(np.isnan(x), NAN32, x)


def _to16(x, dtype):
    """fp32 numpy array rounded to nearest even; NaNs in the format's canonical form (processors differ)."""
    bits = torch.from_numpy(np.ascontiguousarray(x)).to(dtype).view(torch.int16)
    bits[torch.from_numpy(np.isnan(x))] = 0x7FC0 if dtype == torch.bfloat16 else 0x7E00
    return bits.view(dtype)


def step(w, p, m, v, grad, hp, scale, skip):
    """New (w16 tensor, p, m, v as fp32 numpy arrays) of one group; grad a 16-bit tensor."""
    f = np.float32
    p, m, v = (x.detach().cpu().numpy() for x in (p, m, v))
    if skip:
        return _to16(p, w.dtype), p, m, v
    lr, b1, b2, wd = (float(f(hp[k])) for k in ("lr", "beta1", "beta2", "weight_decay"))
    t = float(hp["step"])
    with np.errstate(all="ignore"):
        g = grad.detach().cpu().float().numpy() * f(scale)
        m1 = f(b1) * m + f(1.0 - b1) * g
        v1 = f(b2) * v + (f(1.0 - b2) * g) * g
        d = np.sqrt(v1) / f(math.sqrt(1.0 - b2 ** t)) + f(hp["eps"])
        p1 = p * f(1.0 - lr * wd) - f(lr / (1.0 - b1 ** t)) * (m1 / d)
    p1, m1, v1 = _canonical(p1), _canonical(m1), _canonical(v1)
    return _to16(p1, w.dtype), p1, m1, v1


def step64(p, m, v, g, hp):
    """The update in 64 bits on 64-bit arrays."""
    b1, b2, t = hp["beta1"], hp["beta2"], hp["step"]
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    rate = (m1 / (1 - b1 ** t)) / (np.sqrt(v1 / (1 - b2 ** t)) + hp["eps"])
    return p - hp["lr"] * (hp["weight_decay"] * p + rate), m1, v1


def policy(z, y, old, adv, w, ref=None, low=0.2, high=0.2, beta=0.0, loss_scale=1.0):
    """Outputs of the policy loss in 64 bits, as a dict; size: per token what bounds the slope's rounding error."""
    z, old, adv, w = z.detach().cpu().double(), old.cpu().double(), adv.cpu().double(), w.cpu().double()
    y = y.cpu()
    n, v = z.shape
    low, high = float(np.float32(low)), float(np.float32(high))
    beta = float(np.float32(beta))
    inside = (y >= 0) & (y < v)
    empty = (z == -math.inf).all(1)
    used = (w != 0) & inside & ~empty
    at = torch.where(inside, y, 0)[:, None]
    logp = torch.where(used, z.log_softmax(1).gather(1, at)[:, 0], 0.0)
    r = (logp - old).exp()
    kept, cut = r * adv, r.clamp(1 - low, 1 + high) * adv
    flat = used & (cut < kept)
    token, slope = -torch.minimum(kept, cut), torch.where(flat, 0.0, -kept)
    size = torch.where(flat, 0.0, kept.abs())
    kl = torch.zeros(n, dtype=torch.float64)
    if ref is not None:
        d = ref.cpu().double() - logp
        kl = d.expm1() - d
        if beta:
            token, slope = token + beta * kl, slope - beta * d.expm1()
            size = size + beta * (1 + d.exp())
    zero = torch.zeros(n, dtype=torch.float64)
    token, kl, c = (torch.where(used, x, zero) for x in (token, kl, w * slope * loss_scale))
    probs = torch.where(used[:, None], z.softmax(1), 0.0)
    grad = -c[:, None] * probs
    grad.scatter_(1, at, (c * -torch.where(used, logp, -1.0).expm1())[:, None])
    ww = torch.where(used, w, zero)
    return dict(logp=logp, token_loss=token, loss=float((ww * token).sum()), kl=float((ww * kl).sum()),
                n_tokens=int(used.sum()), n_clipped=int(flat.sum()),
                n_invalid=int(((w != 0) & ~(inside & ~empty)).sum()), dlogits=grad, used=used, size=size,
                coef=torch.where(used, (w * size * loss_scale).abs(), zero))
