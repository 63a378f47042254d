"""A step writes the memory that its optimiser was made for, not what has taken its place."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_masters_that_ask_for_a_gradient():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    new = lambda dtype=torch.float32: torch.ones(5000, dtype=dtype, device=dev)
    param, master = torch.nn.Parameter(new(torch.float16)), torch.nn.Parameter(new())
    with torch.no_grad():
        opt = fiona.AdamW([param], [new(torch.float16)], [new() * 0], [new() * 0], masters=[master], weight_decay=0.0)
    old = opt._tensors["masters"][0]
    master.data = torch.zeros(5000, device=dev)
    assert old.data_ptr() != master.data_ptr() and bool((old == 1).all())
    fiona.adamw_step(opt, torch.full((1,), 0.125, device=dev), torch.ones(1, dtype=torch.int32, device=dev))
    torch.cuda.synchronize()
    assert not master.any() and bool(((old - 0.875).abs() < 1e-5).all()) and bool(((param.float() - 0.875).abs() < 1e-3).all())
