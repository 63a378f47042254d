"""Limits of the key holder's operators: refusals by stride and handle, infinities, a cache's last places."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fiona.lib()
    return torch.device("cuda:0")


def _adapter(dev, n=2, d=64, R=8):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).to(dev)
    return dict(x=r(n, d), A=r(1, R, d), B=r(1, d, R), base=r(n, d), ids=torch.zeros(n, dtype=torch.int32, device=dev))


def test_rows_too_far_apart_are_refused():
    dev = _dev()
    t = _adapter(dev)
    far = torch.zeros((1 << 24) + 1 + 64, device=dev).as_strided((2, 64), ((1 << 24) + 1, 1))
    h = fiona.Adapters(F32, 1, 8, 64, 64, 2)
    y = torch.empty(2, 64, device=dev)
    for over in (dict(x=far), dict(base=far)):
        a = dict(t, **over)
        with pytest.raises(fiona.FionaError) as e:
            fiona.adapter_linear(h, a["x"], a["ids"], a["A"], a["B"], a["base"], y)
        assert e.value.status == -3, over.keys()
    # at the limit they are read
    edge = torch.zeros((1 << 24) + 64, device=dev).as_strided((2, 64), (1 << 24, 1))
    edge.copy_(t["x"])
    want = torch.empty_like(y)
    fiona.adapter_linear(h, t["x"], t["ids"], t["A"], t["B"], t["base"], want)
    fiona.adapter_linear(h, edge, t["ids"], t["A"], t["B"], t["base"], y)
    assert torch.equal(y, want)


def test_a_forward_handle_has_no_gradients():
    dev = _dev()
    t = _adapter(dev)
    h = fiona.Adapters(F32, 1, 8, 64, 64, 2, forward_only=True)
    with pytest.raises(fiona.FionaError) as e:
        fiona.adapter_backward(h, t["x"], t["ids"], t["A"], t["B"], t["base"], None, torch.empty_like(t["x"]),
                               torch.empty_like(t["A"]), torch.empty_like(t["B"]))
    assert e.value.status == -1


@pytest.mark.parametrize("dtype", [F32, torch.float16, BF16])
def test_infinities_stay_with_their_token(dtype):
    dev = _dev()
    t = {k: v if k == "ids" else v.to(dtype) for k, v in _adapter(dev, n=40).items()}
    h = fiona.Adapters(dtype, 1, 8, 64, 64, 40)
    want, y = torch.empty_like(t["base"]), torch.empty_like(t["base"])
    fiona.adapter_linear(h, t["x"], t["ids"], t["A"], t["B"], t["base"], want)
    t["x"][7, 3] = float("inf")
    fiona.adapter_linear(h, t["x"], t["ids"], t["A"], t["B"], t["base"], y)
    others = [i for i in range(40) if i != 7]
    assert torch.equal(y[others], want[others])
    assert not torch.isfinite(y[7].float()).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page", [1, 8, 16, 24])
def test_a_cache_up_to_its_last_place(dtype, page):
    """Sequences that end anywhere in the cache's last page, which ends the allocation."""
    dev = _dev()
    g = torch.Generator().manual_seed(page)
    n_pages, H, d = 48 // page, 2, 64
    store = torch.randn(2, n_pages * page * H * d, generator=g).to(dtype).to(dev)
    k, v = (s.view(n_pages, page, H, d) for s in store)
    lengths = list(range(max(1, n_pages * page - 17), n_pages * page + 1))
    n = len(lengths)
    q = torch.randn(n, H, d, generator=g).to(dtype).to(dev)
    table = torch.arange(n_pages, dtype=torch.int32, device=dev).expand(n, n_pages).contiguous()
    out = torch.empty_like(q)
    fiona.paged_attention(fiona.Attention(dtype, H, H, d, page, n, n_pages * page), q, k, v, table,
                          torch.tensor(lengths, dtype=torch.int32, device=dev), out)
    kf, vf, qf = (t.double().cpu() for t in (k.reshape(-1, H, d), v.reshape(-1, H, d), q))
    # weights rounded to the type (half a unit of the sum), the result once more
    tol = 2 ** -7 if dtype is BF16 else 1e-5
    for i, m in enumerate(lengths):
        for h in range(H):
            w = torch.softmax(kf[:m, h] @ qf[i, h] * d ** -0.5, 0)
            want = w @ vf[:m, h]
            assert (out[i, h].double().cpu() - want).abs().max() <= tol * vf.abs().max(), (i, h)
