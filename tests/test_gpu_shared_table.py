"""fiona_paged_attention with page tables whose rows lie over each other: one for all sequences, or sliding over one list."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import key_holder_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("stride", [0, 1, 5])
def test_rows_over_each_other(stride, n, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(stride + n)
    H, KV, d, page, width = 4, 2, 64, 8, 12
    pages = torch.randperm(40, generator=g)[:width + stride * (n - 1)].to(torch.int32)
    table = pages.to(dev).as_strided((n, width), (stride, 1))
    kc, vc = (torch.randn(40, page, KV, d, generator=g).to(dtype) for _ in range(2))
    q = torch.randn(n, H, d, generator=g).to(dtype)
    lengths = [90, 37, 61][:n]
    out, lse = torch.empty(n, H, d, dtype=dtype, device=dev), torch.empty(n, H, device=dev)
    fiona.paged_attention(fiona.Attention(dtype, H, KV, d, page, n, 96), q.to(dev), kc.to(dev), vc.to(dev), table,
                          torch.tensor(lengths, dtype=torch.int32, device=dev), out, lse=lse)
    for i, m in enumerate(lengths):
        j = torch.arange(m)
        p = pages[stride * i + j // page].long()
        y, yb, l, lb = ref.attention(q[i], kc[p, j % page], vc[p, j % page], d ** -0.5, 0.0, dtype)
        ref.assert_close(out[i], y, yb, "sequence %d" % i)
        ref.assert_close(lse[i], l, lb, "sequence %d lse" % i)
