"""Windows of fiona_paged_attention in every type, over one and several parts of a sequence."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import key_holder_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("window", [1, 15, 33, 700, 1300])
@pytest.mark.parametrize("H,KV,d,page", [(8, 2, 128, 16), (35, 7, 80, 24), (3, 3, 36, 5)])
def test_windows(H, KV, d, page, window, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(window + d)
    lengths = [0, 1, 14, 34, 701, 2000]
    held = [-(-n // page) for n in lengths]
    kc, vc = (torch.randn(sum(held), page, KV, d, generator=g).to(dtype) for _ in range(2))
    q = (2 * torch.randn(len(lengths), H, d, generator=g)).to(dtype)
    table = torch.full((len(lengths), max(held)), -1, dtype=torch.int32)
    order, at = torch.randperm(sum(held), generator=g).int(), 0
    for i, h in enumerate(held):
        table[i, :h] = order[at:at + h]
        at += h
    out, lse = torch.empty(q.shape, dtype=dtype, device=dev), torch.empty(q.shape[:2], device=dev)
    fiona.paged_attention(fiona.Attention(dtype, H, KV, d, page, len(lengths), 2000), q.to(dev), kc.to(dev), vc.to(dev), table.to(dev),
                          torch.tensor(lengths, dtype=torch.int32, device=dev), out, window=window, lse=lse)
    for i, n in enumerate(lengths):
        j = torch.arange(max(0, n - window), n)
        p = table[i, j // page].long()
        y, yb, l, lb = ref.attention(q[i], kc[p, j % page], vc[p, j % page], d ** -0.5, 0.0, dtype)
        ref.assert_close(out[i], y, yb, "%d keys of %d: out" % (len(j), n))
        ref.assert_close(lse[i], l, lb, "%d keys of %d: lse" % (len(j), n))
