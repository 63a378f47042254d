"""Plain 64-bit forms of the training step's operators, on CPU tensors, with the error bounds their tests compare against.

The kernels compute in 32 bits (E = 2^-24 an operation) and round a result to its type once (U). A sum of k terms in a
workgroup's order has at most k / 64 + 32 additions one after another to each term (a wavefront to a row is the longest), so its error is
at most that many E times the sum of the magnitudes; sums over rows, in parts of any length, take the number of rows.
Exponentials by the hardware's instruction are within 2^-21 of themselves, plus the rounding of their argument.  Every
bound is doubled once, for second-order terms.
"""
import math

import torch
from key_holder_reference import E, TINY, U, assert_close  # noqa: F401

F32 = torch.float32


def _deep(k):
    return k / 64 + 32


def norm(x, residual, weight, bias, eps):
    """total (in its type), y, its bound, mean, its bound, rstd, its bound."""
    dt = x.dtype
    total = x if residual is None else (x.float() + residual.float()).to(dt)
    s = total.double()
    d = s.shape[1]
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(d, dtype=torch.float64) if bias is None else bias.double()
    mean = s.mean(1, keepdim=True)
    c = s - mean
    var = c.square().mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    y = w * c * rstd + b
    dm = (_deep(d) + 2) * E * s.abs().mean(1, keepdim=True)
    # what a wrong mean adds to the squares: its own square (the deviations' sum is zero), and the rounding of each deviation
    dv = (_deep(d) + 4) * E * var + dm * dm + 2 * E * c.square().mean(1, keepdim=True) + 4 * E * dm * c.abs().mean(1, keepdim=True)
    rel = dv / (2 * (var + eps)) + 4 * E
    by = w.abs() * rstd * (dm + E * c.abs()) + (w * c * rstd).abs() * (rel + 3 * E) + E * b.abs() + U[dt] * y.abs()
    return total, y, 2 * by + TINY[dt], mean[:, 0], 2 * (dm + E * mean.abs())[:, 0], rstd[:, 0], 2 * (rstd * (rel + E))[:, 0]


def norm_gradients(dy, x, weight, mean, rstd, dx_base, weight_dtype):
    """(dx, bound), (dweight, bound), (dbias, bound)."""
    dt = x.dtype
    n, d = x.shape
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double()
    g, r = dy.double(), rstd.double()[:, None]
    c = x.double() - mean.double()[:, None]
    xh, u = c * r, w * g
    s1, s2 = u.mean(1, keepdim=True), (u * xh).mean(1, keepdim=True)
    dx = r * (u - s1 - xh * s2)
    d1 = (_deep(d) + 3) * E * u.abs().mean(1, keepdim=True)
    d2 = (_deep(d) + 6) * E * (u * xh).abs().mean(1, keepdim=True)
    b = r.abs() * (d1 + xh.abs() * d2 + 6 * E * (u.abs() + s1.abs() + 2 * (xh * s2).abs()))
    if dx_base is not None:
        dx = dx + dx_base.double()
        b = b + E * dx_base.double().abs()
    b = 2 * (b + (U[dt] + E) * dx.abs()) + TINY[dt]
    dw, db, uw = (g * xh).sum(0), g.sum(0), U[weight_dtype]
    bw = 2 * ((n + 6) * E * (g * xh).abs().sum(0) + uw * dw.abs()) + TINY[weight_dtype]
    bb = 2 * ((n + 2) * E * g.abs().sum(0) + uw * db.abs()) + TINY[weight_dtype]
    return (dx, b), (dw, bw), (db, bb)


def scores(logits, targets):
    """Log-probabilities (0 for tokens that do not count), their bounds, log softmax rows, and the bounds of p, relative."""
    z = logits.double()
    n, V = z.shape
    live = (targets >= 0) & (targets < V)
    z = torch.where(live[:, None], z, 0.0)
    m = z.amax(1, keepdim=True)
    lse = torch.logsumexp(z, 1, keepdim=True)
    lp = z - lse
    p = lp.exp()
    away = torch.where(p > 0, (z - m).abs(), 0.0)
    rel = (p * (2.0 ** -21 + 4 * E * away)).sum(1, keepdim=True) + _deep(V) * E
    dlse = rel + 2 * E * (lse.abs() + m.abs()) + 2.0 ** -21 * (lse - m).abs()
    at = targets.long().clamp(0, V - 1)[:, None]
    l = torch.where(live, lp.gather(1, at)[:, 0], 0.0)
    dl = torch.where(live, dlse[:, 0] + E * l.abs(), 0.0)
    far = torch.where(p > 0, lp.abs(), 0.0)
    return l, dl, lp, dlse + 2.0 ** -21 + 4 * E * far, live, at


def _dlogits(dt, lp, rel, live, at, coef, dcoef):
    """The gradient's rows and their bounds."""
    p = lp.exp()
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    use = (live & (coef != 0))[:, None]
    c, dc = coef[:, None], dcoef[:, None]
    dz = torch.where(use, c * (hot - p), 0.0)
    b = torch.where(use, dc * (hot - p).abs() + c.abs() * p * rel + 4 * E * c.abs() * (hot + p), 0.0)
    return dz, 2 * (b + U[dt] * dz.abs()) + TINY[dt]


def preference(logits, targets, offsets, reference, weights, beta, smoothing):
    """(loss, bound), (logps, bound), (dlogits, bound)."""
    l, dl, lp, rel, live, at = scores(logits, targets)
    n, S = l.shape[0], reference.shape[0]
    ends = offsets.clamp(0, n).tolist()
    seq = torch.full((n,), -1)
    L, dL = torch.zeros(S, dtype=torch.float64), torch.zeros(S, dtype=torch.float64)
    for s in range(S):
        seq[ends[s]:ends[s + 1]] = s
        L[s], dL[s] = l[ends[s]:ends[s + 1]].sum(), dl[ends[s]:ends[s + 1]].sum()
    w = torch.full((S // 2,), 1 / (S // 2) if S else 0.0, dtype=torch.float64) if weights is None else weights.double()
    beta, smoothing = float(torch.tensor(beta)), float(torch.tensor(smoothing))      # (32-bit arguments)
    ratio = L - reference.double()
    h = beta * (ratio[0::2] - ratio[1::2])
    dh = beta * (dL[0::2] + dL[1::2])
    up, down = torch.sigmoid(h), torch.sigmoid(-h)
    loss = -w * ((1 - smoothing) * torch.nn.functional.logsigmoid(h) + smoothing * torch.nn.functional.logsigmoid(-h))
    g = w * beta * (smoothing * up - (1 - smoothing) * down)
    dg = w.abs() * beta * up * down * dh + 2 * E * g.abs()
    both = torch.stack((g, -g), 1).flatten()
    dboth = torch.stack((dg, dg), 1).flatten()
    coef = torch.where(seq >= 0, both[seq.clamp(min=0)] if S else torch.zeros(n, dtype=torch.float64), 0.0)
    dcoef = torch.where(seq >= 0, dboth[seq.clamp(min=0)] if S else torch.zeros(n, dtype=torch.float64), 0.0)
    dz, bz = _dlogits(logits.dtype, lp, rel, live, at, coef, dcoef)
    return (loss, 2 * (w.abs() * dh + 2 * E * loss.abs())), (L, 2 * (dL + 2 * E * L.abs())), (dz, bz)


def policy(logits, targets, old, advantages, reference, weights, clip_low, clip_high, kl):
    """(loss, bound), (logps, bound), (dlogits, bound).  The caller keeps the ratios off the clip's ends."""
    l, dl, lp, rel, live, at = scores(logits, targets)
    n = l.shape[0]
    w = torch.full((n,), 1 / n, dtype=torch.float64) if weights is None else weights.double()
    kl = float(torch.tensor(kl))
    zero = torch.zeros(n, dtype=torch.float64)
    pick = lambda t: torch.where(live, t.double(), 0.0)
    a, x = pick(advantages), l - pick(old)
    r = x.exp()
    dr = r * (dl + 2 * E * (x.abs() + 1) + 2.0 ** -21)
    open_, held = r * a, r.clamp(1 - clip_low, 1 + clip_high) * a
    free = open_ <= held
    s, c = -torch.minimum(open_, held), torch.where(free, -open_, 0.0)
    ds = a.abs() * torch.where(free, dr, 4 * E * r.clamp(1 - clip_low, 1 + clip_high)) + 4 * E * s.abs()
    dc = torch.where(free, a.abs() * dr + 2 * E * open_.abs(), 0.0)
    if kl > 0:
        d = pick(reference) - l
        e = torch.expm1(d)
        s, c = s + kl * (e - d), c - kl * e
        off = dl + E * (d.abs() + 1)                                    # of d
        ds = ds + kl * (e.abs() * off + 2.0 ** -21 * e.abs() + 4 * E * (e.abs() + d.abs()))
        dc = dc + kl * ((e + 1) * off + 2.0 ** -21 * e.abs())
    s, c, ds, dc = (torch.where(live, t, zero) for t in (s, c, ds, dc))
    coef, dcoef = w * c, w.abs() * (dc + 4 * E * c.abs())
    dz, bz = _dlogits(logits.dtype, lp, rel, live, at, coef, dcoef)
    return (w * s, 2 * w.abs() * (ds + 4 * E * s.abs())), (l, 2 * dl), (dz, bz)


def adamw(p, g, m, v, lr, t, beta1, beta2, eps, decay, scale=1.0, new=False):
    """(p, bound), (m, bound), (v, bound) in 32 bits, from 32-bit states; new: m and v are this step's already."""
    p, g, m0, v0 = p.double(), g.double() * scale, m.double(), v.double()
    lr = float(torch.tensor(lr))
    m = beta1 * m0 + (1 - beta1) * g
    v = beta2 * v0 + (1 - beta2) * g * g
    if new:
        m, v = m0, v0
    dm = 4 * E * ((beta1 * m0).abs() + ((1 - beta1) * g).abs())
    dv = 6 * E * (beta2 * v0 + (1 - beta2) * g * g)
    c1, c2 = 1 - beta1 ** t, 1 - beta2 ** t
    root = (v / c2).sqrt() + eps
    step = m / c1 / root
    # a variance off by 6 E of itself, roots, quotients and corrections within a few E each
    dstep = dm / c1 / root + step.abs() * 24 * E
    to = p - lr * decay * p - lr * step
    b = 2 * (E * (3 * p.abs() + to.abs() + 3 * abs(lr) * (decay * p.abs() + step.abs())) + abs(lr) * dstep) + TINY[F32]
    return (to, b), (m, 2 * dm + TINY[F32]), (v, 2 * dv + TINY[F32])


def mix(x):
    x = x ^ (x >> 16)
    x = (x * 0xA3D8B167) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xC94F6E2B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def dither(step, seed, first, n):
    key = int(mix(torch.tensor((step * 0x9E3779B1 + seed) & 0xFFFFFFFF)))
    h = mix(((first + torch.arange(n)) & 0xFFFFFFFF) ^ key)
    return ((h & 0xFFFF).float() + 0.5) / 65536, ((h >> 16).float() + 0.5) / 65536


def _spread(x, n):
    """x [n] in blocks of 256, the last filled with zeros."""
    out = torch.zeros(-(-n // 256) * 256, dtype=torch.float64)
    out[:n] = x
    return out.view(-1, 256)


def to_codes(x, up, positive):
    """x [n] as e4m3 values, in 64 bits: (codes [n], scales, and the other neighbour [n] where a value and its dither come within
    2^-15 of a step to the border between the two)."""
    n = x.numel()
    x, up = _spread(x.double(), n).double(), _spread(up, n).double()
    top = x.abs().amax(1, keepdim=True)
    top = torch.where(top < 2.0 ** -100, torch.zeros((), dtype=torch.float64), top)
    y = x.abs() * torch.where(top > 0, 448.0 / top, torch.zeros((), dtype=torch.float64))
    e = torch.frexp(y)[1].clamp(min=-5)
    unit = torch.ldexp(torch.ones_like(y), e - 4)

    def values(k):
        if positive:
            k = torch.where(x > 0, k.clamp(min=1.0), torch.zeros((), dtype=torch.float64))
        k = torch.where(top > 0, k, torch.zeros((), dtype=torch.float64))
        return (torch.sign(x) * k * unit).clamp(-448, 448).flatten()[:n].float().to(torch.float8_e4m3fn)

    # 32 bits leave y / unit, below 16, off by a few 2^-24 of itself: by 16 * 16 * 2^-24 = 2^-16 of a step at most, and the sum by
    # half of 2^-20; y just below a power of two may count as that power, whose steps are twice as long: the same values
    at = y / unit + up
    return values(torch.floor(at)), (top / 448.0)[:, 0].float(), torch.stack([values(torch.floor(at + s * 2.0 ** -15)).float() for s in (-1, 1)])


def states8(g, m, v, m_scale, v_scale, beta1, beta2, step, seed, first, scale=1.0):
    """The new 8-bit states (to_codes of m and of v's root), and m and v, in 64 bits."""
    n = g.numel()
    each = lambda s: s.double().repeat_interleave(256)[:n]
    g = g.double() * scale
    m, v = m.double() * each(m_scale), (v.double() * each(v_scale)) ** 2
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    um, uv = dither(step, seed, first, n)
    return to_codes(m, um, False), to_codes(v.sqrt(), uv, True), m, v
