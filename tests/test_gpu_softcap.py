"""fiona_paged_attention's capped scores: their error is relative to the score, whatever the cap.

A capped score c tanh(s / c) is computed with some roundings of 2^-24 each, all relative: s (the scale with the factor of
the exponent's base, its product: 3), s / c (2; a hyperbolic tangent's relative error is at most its argument's), the
hyperbolic tangent itself (an exponential and a reciprocal of one unit in the last place each, a sum and a difference
whose result is at least half the smaller term: 12), the product with the cap and the way back to natural units (3).
20 in all, doubled once for second-order terms.
"""
import math

import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import key_holder_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
CAP_UNITS = 2 * 20 * ref.E


def _dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fiona.lib()
    return torch.device("cuda:0")


def _cap(s, cap):
    return cap * torch.tanh(s / cap)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [0.5, 1.0, 30.0, 1000.0, 1e5, 1e8, 3e38])
@pytest.mark.parametrize("scale", [1.0, 0.088])
def test_one_key_shows_its_capped_score(cap, scale, dtype):
    """Over one key the log-sum-exp is the capped score: one product, exact before the scale."""
    dev = _dev()
    x = torch.logspace(-4, 4.7, 500, dtype=torch.float64)
    x = torch.cat((x, -x, cap * torch.linspace(0.05, 3, 200, dtype=torch.float64) / scale, torch.zeros(1, dtype=torch.float64)))
    x = x[x.abs() < (6e4 if dtype is F16 else 1e30)].to(dtype)
    n = len(x)
    q, k = torch.zeros(n, 1, 8, dtype=dtype), torch.zeros(1, 1, 1, 8, dtype=dtype)
    q[:, 0, 2], k[0, 0, 0, 2] = x, 1
    v = torch.ones(1, 1, 1, 8, dtype=dtype, device=dev)
    out, lse = torch.empty(n, 1, 8, dtype=dtype, device=dev), torch.empty(n, 1, device=dev)
    fiona.paged_attention(fiona.Attention(dtype, 1, 1, 8, 1, n, 1), q.to(dev), k.to(dev), v,
                          torch.zeros(n, 1, dtype=torch.int32, device=dev), torch.ones(n, dtype=torch.int32, device=dev), out,
                          scale=scale, softcap=cap, lse=lse)
    want = _cap(float(torch.tensor(scale)) * x.double(), float(torch.tensor(cap)))
    ref.assert_close(lse[:, 0], want, CAP_UNITS * want.abs() + 2.0 ** -120, "cap %g" % cap)
    assert torch.equal(out.cpu(), torch.ones_like(out.cpu()))


def _expected(q, keys, values, scale, cap, dtype):
    """One sequence in 64 bits with bounds, as the reference module's without a cap, and the cap's own units."""
    H, d = q.shape
    n, KV, _ = keys.shape
    if n == 0:
        z = torch.zeros(H, d, dtype=torch.float64)
        return z, z.clone(), torch.full((H,), -math.inf, dtype=torch.float64), torch.zeros(H, dtype=torch.float64)
    k, v = keys.double().repeat_interleave(H // KV, 1), values.double().repeat_interleave(H // KV, 1)
    raw = scale * torch.einsum("hd,nhd->hn", q.double(), k)
    s = _cap(raw, cap)
    ds = ((d + 6) * ref.E * scale * torch.einsum("hd,nhd->hn", q.double().abs(), k.abs()) + CAP_UNITS * s.abs()).amax(1)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    out, weight = torch.einsum("hn,nhd->hd", p, v), torch.einsum("hn,nhd->hd", p, v.abs())
    rel = 2 * ds + 2.0 ** -20 + n * ref.E
    unit = ref.U[dtype] if dtype is not F32 else 0
    bound = 2 * (ref.U[dtype] * out.abs() + (rel[:, None] + unit) * weight) + ref.TINY[dtype]
    return out, bound, lse, 2 * (ds + 2.0 ** -20 + n * ref.E + 2 * ref.E * lse.abs())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [5.0, 20.0, 50.0, 1000.0, 1e5, 1e7, 3e38])
@pytest.mark.parametrize("H,KV,d,page,lengths", [(2, 1, 8, 5, [60, 7, 0, 1]), (8, 2, 64, 16, [0, 1, 33, 300, 1500]),
                                                 (35, 7, 80, 24, [17, 129])])
def test_caps_of_every_size(H, KV, d, page, lengths, cap, dtype):
    dev = _dev()
    g = torch.Generator().manual_seed(d + len(lengths))
    held = [-(-n // page) for n in lengths]
    pages = sum(held) + 1
    kc, vc = (torch.randn(pages, page, KV, d, generator=g).to(dtype) for _ in range(2))
    q = (2 * torch.randn(len(lengths), H, d, generator=g)).to(dtype)
    table = torch.full((len(lengths), max(held)), -1, dtype=torch.int32)
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = torch.arange(at, at + h, dtype=torch.int32)
        at += h
    out, lse = torch.empty(q.shape, dtype=dtype, device=dev), torch.empty(q.shape[:2], device=dev)
    scale, c32 = 0.25, float(torch.tensor(cap))
    fiona.paged_attention(fiona.Attention(dtype, H, KV, d, page, len(lengths), max(lengths)), q.to(dev), kc.to(dev),
                          vc.to(dev), table.to(dev), torch.tensor(lengths, dtype=torch.int32, device=dev), out, scale=scale,
                          softcap=cap, lse=lse)
    for i, n in enumerate(lengths):
        j = torch.arange(n)
        p = table[i, j // page].long()
        y, yb, l, lb = _expected(q[i], kc[p, j % page], vc[p, j % page], scale, c32, dtype)
        ref.assert_close(out[i], y, yb, "cap %g, %d keys: out" % (cap, n))
        ref.assert_close(lse[i], l, lb, "cap %g, %d keys: lse" % (cap, n))


def test_a_cap_far_below_every_score():
    """All scores meet at the cap or, where they are zero, at zero: the mean of the values, no NaN."""
    dev = _dev()
    g = torch.Generator().manual_seed(7)
    k, v = (torch.randn(3, 16, 1, 64, generator=g).to(dev) for _ in range(2))
    q = torch.stack((torch.zeros(1, 64), torch.randn(1, 64, generator=g))).to(dev)
    out, lse = torch.empty_like(q), torch.empty(2, 1, device=dev)
    table = torch.arange(3, dtype=torch.int32, device=dev).repeat(2, 1)
    fiona.paged_attention(fiona.Attention(F32, 1, 1, 64, 16, 2, 48), q, k, v, table,
                          torch.tensor([48, 48], dtype=torch.int32, device=dev), out, softcap=2e-38, lse=lse)
    want = v.double().cpu().view(48, 64).mean(0)
    bound = 2 * (2.0 ** -20 + 48 * ref.E) * v.double().cpu().view(48, 64).abs().mean(0)
    for i in range(2):
        ref.assert_close(out[i, 0], want, bound, "mean")
        assert abs(float(lse[i, 0]) - math.log(48)) <= 2 * (2.0 ** -20 + 48 * ref.E)
