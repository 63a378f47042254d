"""fiona_kv_append with rotation tables of no rows: every position lies outside them, and nothing is read there."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 32), (80, 48), (33, 10)])
@pytest.mark.parametrize("table", ["empty", "null", "of no rows in a longer one"])
def test_every_rotated_element_is_nan(table, d, rot, interleaved, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(d)
    n, H, KV, page = 9, 3, 2, 4
    q, k, v = (torch.randn(n, h, d, generator=g).to(dtype).to(dev) for h in (H, KV, KV))
    kc, vc = (torch.full((4, page, KV, d), 5.0, dtype=dtype, device=dev) for _ in range(2))
    slots = torch.arange(2, 2 + n, device=dev)
    positions = torch.arange(n, dtype=torch.int32, device=dev) - 2
    q_out = torch.empty_like(q)
    if table == "empty":
        empty = torch.empty(0, rot // 2, device=dev)
        fiona.kv_append(k, v, slots, kc, vc, positions=positions, cos=empty, sin=empty, interleaved=interleaved, q=q, q_out=q_out)
    else:
        some = torch.ones(8, rot // 2, device=dev)
        at = 0 if table == "null" else some.data_ptr()
        cache = fiona._cache_desc(kc, vc)[0]
        args = fiona._APPEND_ARGS.pack(n, H, fiona._type_code(dtype), rot, 0, int(interleaved), k.data_ptr(), v.data_ptr(), q.data_ptr(),
                                       q_out.data_ptr(), KV * d, d, KV * d, d, H * d, d, H * d, d, slots.data_ptr(),
                                       positions.data_ptr(), at, at)
        assert fiona.lib().fiona_kv_append(cache, args, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    kf, vf = kc.flatten(0, 1), vc.flatten(0, 1)
    for got, rows in ((q_out, q), (kf[slots], k)):
        assert bool(torch.isnan(got[..., :rot]).all()) and torch.equal(got[..., rot:], rows[..., rot:])
    assert torch.equal(vf[slots], v)
    assert bool((kf[:2] == 5).all()) and bool((vf[2 + n:] == 5).all())
