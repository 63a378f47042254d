"""fiona_paged_attention with scores far from one: in 32 bits a score of 2^33 is known to 2^9, but the largest is
still the largest, and its weight is one."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import key_holder_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fiona.lib()
    return torch.device("cuda:0")


def _call(dev, q, keys, values, scale):
    """Sequences of equal length, pages of 16 in order: q [n][H][d], keys, values [n][m][H][d]."""
    n, m, H, d = keys.shape
    pad = -m % 16
    cache = [torch.cat((t, t.new_zeros(n, pad, H, d)), 1).reshape(-1, 16, H, d).to(dev) for t in (keys, values)]
    table = torch.arange(cache[0].shape[0], dtype=torch.int32, device=dev).view(n, -1)
    out, lse = torch.empty_like(q, device=dev), torch.empty(n, H, device=dev)
    fiona.paged_attention(fiona.Attention(q.dtype, H, H, d, 16, n, m), q.to(dev), *cache, table,
                          torch.full((n,), m, dtype=torch.int32, device=dev), out, scale=scale, lse=lse)
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,m", [(40, 50), (6, 1500)])
def test_the_largest_of_very_large_scores_takes_all(n, m, dtype):
    dev = _dev()
    g = torch.Generator().manual_seed(m)
    size = 2e4 if dtype is F16 else 4e6
    q, k = ((size * torch.randn(n, *s, 2, 64, generator=g)).clamp(-6e4 if dtype is F16 else -1e30, 6e4 if dtype is F16 else 1e30)
            .to(dtype) for s in ((), (m,)))
    v = torch.randn(n, m, 2, 64, generator=g).to(dtype)
    s = torch.einsum("nhd,nmhd->nmh", q.double(), k.double())
    err = 70 * ref.E * torch.einsum("nhd,nmhd->nmh", q.double().abs(), k.double().abs()).amax(1)
    top = s.topk(2, 1).values
    clear = top[:, 0] - top[:, 1] > 2 * err + 200      # (the second's weight is below 2^-24 of the first's)
    assert int(clear.sum()) >= n
    out, lse = _call(dev, q, k, v, 1.0)
    best = s.argmax(1)
    for i, h in clear.nonzero().tolist():
        assert torch.equal(out[i, h], v[i, best[i, h], h]), (i, h)
        assert abs(float(lse[i, h]) - float(top[i, 0, h])) <= float(err[i, h]) + 8 * ref.E * abs(float(top[i, 0, h]))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m", [48, 1500])
def test_very_large_equal_scores_share_alike(m, dtype):
    dev = _dev()
    g = torch.Generator().manual_seed(m)
    n, size = 24, 2e4 if dtype is F16 else 4e6
    q = (size * (1 + torch.rand(n, 2, 64, generator=g))).to(dtype)
    k = (size * (1 + torch.rand(n, 1, 2, 64, generator=g))).to(dtype).expand(n, m, 2, 64)
    v = torch.randn(n, m, 2, 64, generator=g).to(dtype)
    out, _ = _call(dev, q, k, v, 1.0)
    want, mag = v.double().mean(1), v.double().abs().mean(1)
    bound = 2 * (ref.U[dtype] * want.abs() + (2.0 ** -20 + m * ref.E + (ref.U[dtype] if dtype is not F32 else 0)) * mag) + ref.TINY[dtype]
    ref.assert_close(out, want, bound, "equal scores")
