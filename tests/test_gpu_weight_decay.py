"""Weight decay at small learning rates, over many steps."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import training_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16, F8 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


def _dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fiona.lib()
    return torch.device("cuda:0")


def _run(dev, x0, dtype, bits, lr, decay, steps):
    n = x0.numel()
    x = x0.to(dev)
    param = x.to(dtype) if dtype is not F32 else x.clone()
    state = lambda: torch.zeros(n, device=dev).to(F8 if bits == 8 else F32)
    scale = lambda: [torch.zeros(-(-n // 256), device=dev)] if bits == 8 else None
    grad = torch.empty(n, dtype=dtype, device=dev)
    opt = fiona.AdamW([param], [grad], [state()], [state()], masters=[x] if dtype is not F32 else None, m_scales=scale(), v_scales=scale(),
                      weight_decay=decay, seed=3)
    g = torch.Generator(device=dev).manual_seed(11)
    rate, at = torch.tensor([lr], device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    for _ in range(steps):
        at += 1
        grad.copy_(torch.randn(n, generator=g, device=dev))
        fiona.adamw_step(opt, rate, at)
    torch.cuda.synchronize()
    return (param if dtype is F32 else x).cpu().double()


@pytest.mark.parametrize("dtype,bits", [(F32, 32), (F32, 8), (BF16, 32), (F16, 32), (BF16, 8)])
@pytest.mark.parametrize("lr", [5e-7, 2e-6, 1e-5, 5e-5])
def test_the_decay_asked_for_is_applied(lr, dtype, bits):
    """The same gradients with decay and without: the states do not depend on the parameters, so the updates are the same, and
    what lies between the two, along the first parameters, is lr decay a step.

    A step rounds a parameter x once to 32 bits, by at most 2^-24 |x|, up or down as the update falls.  Along the parameters
    (magnitudes in [1, 2), n of them, 1.14 the ratio of their fourth moment to the square of their second) the sum over `steps`
    and both runs stays within 7 deviations of at most 2^-24 sqrt(2 steps 1.14 / n) (Hoeffding's bound: 5e-11).  Parameters move by
    at most 10 lr a step, |m| / sqrt(v) with these betas never passing (1 - beta1) / sqrt(1 - beta2) < 3.2 times the
    corrections' ratio (below 1 but for rounding after the first step), in directions that do not depend on them; the decay
    itself shrinks them by lr decay a step: together at most 20 lr steps of the difference."""
    dev = _dev()
    n, steps, decay = 1 << 19, 128, 0.01
    g = torch.Generator().manual_seed(1)
    x0 = (1 + torch.rand(n, generator=g)) * (torch.randint(2, (n,), generator=g) * 2 - 1)
    with_, without = (_run(dev, x0, dtype, bits, lr, d, steps) for d in (decay, 0.0))
    x = x0.double()
    applied = float(((without - with_) * x).sum() / (x * x).sum())
    asked = steps * float(torch.tensor(lr)) * decay
    rounding = 7 * 2.0 ** -24 * (2 * steps * 1.14 / n) ** 0.5
    assert abs(applied - asked) <= rounding + 20 * lr * steps * asked, (applied, asked)
    assert rounding < 0.03 * asked                # (what the test can see)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.0, 0.01, 2.0])
def test_infinite_parameters_stay(bits, decay):
    """An infinite parameter with no gradient stays infinite, decayed or not; its neighbours' steps are their own."""
    dev = _dev()
    x = torch.ones(600, device=dev)
    x[5], x[300] = float("inf"), -float("inf")
    s = lambda: torch.zeros(600, device=dev).to(F8 if bits == 8 else F32)
    k = lambda: [torch.zeros(3, device=dev)] if bits == 8 else None
    opt = fiona.AdamW([x], [torch.zeros(600, device=dev)], [s()], [s()], m_scales=k(), v_scales=k(), weight_decay=decay)
    fiona.adamw_step(opt, torch.tensor([1e-3], device=dev), torch.ones(1, dtype=torch.int32, device=dev))
    got = x.cpu()
    assert got[5] == float("inf") and got[300] == -float("inf")
    rest = torch.cat((got[:5], got[6:300], got[301:])).double()
    want = 1 - float(torch.tensor(1e-3)) * float(torch.tensor(decay))
    assert bool(((rest - want).abs() <= 4 * ref.E).all())
