"""Caches whose keys and values lie side by side in a page, a token or a head: filled by fiona_kv_append, read by
fiona_paged_attention, neither touching the other's elements."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import key_holder_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
LAYOUTS = {  # the store's axes, and (keys, values) as [page][token][head][d]
    "page": (lambda P, T, H, d: (P, 2, T, H, d), lambda s: (s[:, 0], s[:, 1])),
    "page, heads first": (lambda P, T, H, d: (P, 2, H, T, d), lambda s: (s[:, 0].transpose(1, 2), s[:, 1].transpose(1, 2))),
    "token": (lambda P, T, H, d: (P, T, 2, H, d), lambda s: (s[:, :, 0], s[:, :, 1])),
    "head": (lambda P, T, H, d: (P, T, H, 2, d), lambda s: (s[..., 0, :], s[..., 1, :])),
    "head, heads first": (lambda P, T, H, d: (P, H, T, 2, d), lambda s: (s[..., 0, :].transpose(1, 2), s[..., 1, :].transpose(1, 2))),
    "row": (lambda P, T, H, d: (P, T, H, 2 * d), lambda s: (s[..., :s.shape[-1] // 2], s[..., s.shape[-1] // 2:])),
}


@pytest.mark.parametrize("dtype,d", [(F32, 64), (F16, 80), (BF16, 128), (BF16, 33)])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("pages", [1, 5])
def test_append_and_attend(pages, layout, dtype, d):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(pages + d)
    page, KV, H = 16, 2, 4
    shape, views = LAYOUTS[layout]
    store = torch.full(shape(pages, page, KV, d), 5.0, dtype=dtype, device=dev)
    kc, vc = views(store)
    assert kc.shape == (pages, page, KV, d)
    n = pages * page - 3
    k, v = (torch.randn(n, KV, d, generator=g).to(dtype) for _ in range(2))
    q = torch.randn(1, H, d, generator=g).to(dtype)
    slots = torch.randperm(pages, generator=g)[torch.arange(n) // page] * page + torch.arange(n) % page
    table = (slots[::page] // page).to(torch.int32)[None].contiguous()
    fiona.kv_append(k.to(dev), v.to(dev), slots.to(dev), kc, vc)
    out, lse = torch.empty(1, H, d, dtype=dtype, device=dev), torch.empty(1, H, device=dev)
    fiona.paged_attention(fiona.Attention(dtype, H, KV, d, page, 1, n), q.to(dev), kc, vc, table.to(dev),
                          torch.tensor([n], dtype=torch.int32, device=dev), out, lse=lse)
    p, at = slots // page, slots % page
    for cache, rows in ((kc.cpu(), k), (vc.cpu(), v)):
        assert torch.equal(cache[p, at], rows)
        rest = torch.ones(pages, page, dtype=torch.bool)
        rest[p, at] = False
        assert bool((cache[rest] == 5).all())
    y, yb, l, lb = ref.attention(q[0], k, v, d ** -0.5, 0.0, dtype)
    ref.assert_close(out[0], y, yb, layout)
    ref.assert_close(lse[0], l, lb, layout)
