"""fiona_paged_attention where one key outweighs the rest and holds no value: the rest is all there is to see."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import key_holder_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("gap", [8.0, 11.0, 14.0, 16.0, 17.0, 17.5, 19.0])
@pytest.mark.parametrize("m,sink", [(512, 0), (512, 300), (3000, 7), (40, 39)])
def test_keys_far_below_a_key_without_a_value(m, sink, gap, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(m)
    d, page, H = 64, 16, 2
    q, k = torch.zeros(1, H, d, dtype=dtype), torch.zeros(m, H, d, dtype=dtype)
    q[0, :, 0], k[:, :, 0] = 1, 0
    k[sink, :, 0] = gap                                   # (exact in every type)
    v = (1000 * (1 + torch.rand(m, H, d, generator=g))).to(dtype)
    v[sink] = 0
    pad = -m % page
    cache = [torch.cat((t, t.new_zeros(pad, H, d))).view(-1, page, H, d).to(dev) for t in (k, v)]
    table = torch.arange(cache[0].shape[0], dtype=torch.int32, device=dev)[None]
    out, lse = torch.empty(1, H, d, dtype=dtype, device=dev), torch.empty(1, H, device=dev)
    fiona.paged_attention(fiona.Attention(dtype, H, H, d, page, 1, m), q.to(dev), *cache, table,
                          torch.tensor([m], dtype=torch.int32, device=dev), out, scale=1.0, lse=lse)
    y, yb, l, lb = ref.attention(q[0], k, v, 1.0, 0.0, dtype)
    ref.assert_close(out[0], y, yb, "gap %g" % gap)
    ref.assert_close(lse[0], l, lb, "gap %g: lse" % gap)
