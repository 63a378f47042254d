"""Plain 64-bit forms of the key holder's operators, on CPU tensors, with the
error bounds their tests compare against.

A kernel sums products of T-typed values in 32 bits and rounds the result to T
once, so against the value y in 64 bits its error is at most

    u_T |y|  +  n 2^-24 * (sum of the products' magnitudes)

(u_T half the spacing at 1; n the number of terms, the worst case of any
summation order).  Where a kernel multiplies an intermediate f32 value on the
matrix cores in 16 bits, the rounding of that operand adds its unit times the
same sum: u_T for softmax weights, 2^-16 for an adapter's inner values, kept as
two bfloat16 parts.  Every bound is doubled once, for second-order terms.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}   # underflow
E = 2.0 ** -24


def rotate(x, cos, sin, interleaved):
    """x [n][heads][d] in 64 bits; cos, sin [n][half]."""
    y = x.double().clone()
    h = cos.shape[-1]
    ia = torch.arange(h) * 2 if interleaved else torch.arange(h)
    ib = ia + 1 if interleaved else ia + h
    a, b = x[..., ia].double(), x[..., ib].double()
    c, s = cos.double()[:, None], sin.double()[:, None]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    mag = x.double().abs()
    mag[..., ia], mag[..., ib] = (a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()
    return y, mag


def rotate_bound(y, mag, dtype):
    """Two products and a sum in 32 bits, one rounding."""
    return 2 * (U[dtype] * y.abs() + 3 * E * mag) + TINY[dtype]


def attention(q, keys, values, scale, softcap, dtype):
    """One sequence: q [H][d], keys, values [n][KV][d] in 64 bits.  Returns out, its bound, lse, its bound."""
    H, d = q.shape
    n, KV, _ = keys.shape
    if n == 0:
        z = torch.zeros(H, d, dtype=torch.float64)
        return z, z.clone(), torch.full((H,), -math.inf, dtype=torch.float64), torch.zeros(H, dtype=torch.float64)
    k, v = keys.double().repeat_interleave(H // KV, 1), values.double().repeat_interleave(H // KV, 1)
    s = scale * torch.einsum("hd,nhd->hn", q.double(), k)
    # a score: d products in 32 bits, the scale, the factor of the exponent's base
    ds = ((d + 6) * E * scale * torch.einsum("hd,nhd->hn", q.double().abs(), k.abs()) + 4 * E * s.abs()).amax(1)
    if softcap:
        s = softcap * torch.tanh(s / softcap)
        ds = ds + softcap * 2.0 ** -20   # a hyperbolic tangent from an exponential and a quotient
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    out = torch.einsum("hn,nhd->hd", p, v)
    weight = torch.einsum("hn,nhd->hd", p, v.abs())
    # exponentials and their rescaling: a few units each; softmax weights in T on the matrix cores
    rel = 2 * ds + 2.0 ** -20 + n * E
    bound = 2 * (U[dtype] * out.abs() + (rel[:, None] + (U[dtype] if dtype != torch.float32 else 0)) * weight) + TINY[dtype]
    return out, bound, lse, 2 * (ds + 2.0 ** -20 + n * E + 2 * E * lse.abs())


def _inner_unit(dtype):
    return 0.0 if dtype == torch.float32 else 2.0 ** -16


def adapter(x, ids, A, B, base, ranks, scaling, dtype):
    """y and its bound; base may be None."""
    n, d_in = x.shape
    nA, R, _ = A.shape
    y = torch.zeros(n, B.shape[1], dtype=torch.float64) if base is None else base.double().clone()
    mag = y.abs()
    for t in range(n):
        a = int(ids[t])
        if not 0 <= a < nA:
            continue
        r, c = int(ranks[a]), float(scaling[a])
        h, hm = A[a, :r].double() @ x[t].double(), A[a, :r].double().abs() @ x[t].double().abs()
        y[t] += c * (B[a, :, :r].double() @ h)
        mag[t] += abs(c) * (B[a, :, :r].double().abs() @ hm)
    return y, 2 * (U[dtype] * y.abs() + ((d_in + R + 8) * E + _inner_unit(dtype)) * mag) + TINY[dtype]


def adapter_gradients(x, ids, A, B, dy, dx_base, ranks, scaling, dtype):
    """(dx, bound), (dA, bound), (dB, bound)."""
    n, d_in = x.shape
    nA, R, _ = A.shape
    d_out = B.shape[1]
    dx = torch.zeros(n, d_in, dtype=torch.float64) if dx_base is None else dx_base.double().clone()
    mx = dx.abs()
    dA, dB = torch.zeros(A.shape, dtype=torch.float64), torch.zeros(B.shape, dtype=torch.float64)
    mA, mB = torch.zeros_like(dA), torch.zeros_like(dB)
    for a in range(nA):
        t = (ids == a).nonzero()[:, 0]
        r, c = int(ranks[a]), float(scaling[a])
        a_, b_, x_, dy_ = A[a, :r].double(), B[a, :, :r].double(), x[t].double(), dy[t].double()
        g, gm = c * (dy_ @ b_), abs(c) * (dy_.abs() @ b_.abs())
        h, hm = x_ @ a_.t(), x_.abs() @ a_.abs().t()
        dx[t] += g @ a_
        mx[t] += gm @ a_.abs()
        dA[a, :r], mA[a, :r] = g.t() @ x_, gm.t() @ x_.abs()
        dB[a, :, :r], mB[a, :, :r] = c * (dy_.t() @ h), abs(c) * (dy_.abs().t() @ hm)
    inner = _inner_unit(dtype)
    ex = (d_out + R + 8) * E + inner
    # where both factors of a product come in 16-bit floats of a wider span, each is held in two parts
    ea, eb = (n + d_out + 8) * E + 2 * inner, (n + d_in + 8) * E + 2 * inner
    u, tiny = U[dtype], TINY[dtype]
    return ((dx, 2 * (u * dx.abs() + ex * mx) + tiny), (dA, 2 * (u * dA.abs() + ea * mA) + tiny),
            (dB, 2 * (u * dB.abs() + eb * mB) + tiny))


def assert_close(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))   # infinities and NaN in the same places
    bad = ~same & ~((got - want).abs() <= bound)
    if bool(bad.any()):
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d off, first at %s: %r, not %r (bound %.3g)" % (
            what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(bound[i])))
