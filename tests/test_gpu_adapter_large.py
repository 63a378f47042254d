"""Adapters over thousands of tokens and columns: wavefronts that take several steps of columns one after the other, workgroups
whose 64 tokens all have one adapter, and gradients that look over more than one window of tokens.  The 64-bit forms and
their bounds are the reference module's, computed on the device adapter by adapter."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import key_holder_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
# More than 85 blocks of 64 tokens leave a wavefront two to three steps of 256 columns of these widths; 12 adapters leave
# the gradients' tokens in one piece, which is looked over 2048 tokens (32 bits) or 4096 (16 bits) at a time.
SHAPES = [(5600, 5, 16, 2085, 4133), (5600, 5, 64, 2085, 4133), (9000, 12, 16, 2085, 1100), (9000, 12, 64, 1100, 2085),
          (5504, 12, 20, 2048, 2048), (4700, 3, 128, 1100, 4133)]


def _inputs(n, nA, R, d_in, d_out, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fiona.lib()
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(n + R)
    rnd = lambda *s, k=1.0: (k * torch.randn(*s, generator=g, device=dev)).to(dtype)
    c = dict(x=rnd(n, d_in), A=rnd(nA, R, d_in, k=d_in ** -0.5), B=rnd(nA, d_out, R, k=0.5), base=rnd(n, d_out),
             dy=rnd(n, d_out), dx_base=rnd(n, d_in), scaling=torch.rand(nA, generator=g, device=dev) + 0.5)
    # runs of tokens with one adapter, a stretch of any in any order, single tokens of the first one and of none throughout
    ids = torch.arange(n, device=dev) * 2 * nA // n % nA
    some = torch.arange(n, device=dev)
    ids = torch.where((some > n // 3) & (some < n // 3 + 500), torch.randint(0, nA, (n,), generator=g, device=dev), ids)
    ids[777::1000] = 0
    ids[::913] = -1
    c["ids"] = ids.int()
    c["ranks"] = torch.tensor([R if i % 3 != 1 else R // 2 + 1 for i in range(nA)], dtype=torch.int32, device=dev)
    for a, r in enumerate(c["ranks"].tolist()):
        c["A"][a, r:], c["B"][a, :, r:] = float("nan"), float("nan")
    return c


def _close(got, want, bound, what):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), "%s: %d of %d off, first at %s" % (what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist())


def _inner(dtype):
    return 0.0 if dtype is F32 else 2.0 ** -16


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,nA,R,d_in,d_out", SHAPES)
def test_forward(n, nA, R, d_in, d_out, dtype):
    c = _inputs(n, nA, R, d_in, d_out, dtype)
    part = torch.zeros(n, d_out, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(part)
    for a, r in enumerate(c["ranks"].tolist()):
        t, k = (c["ids"] == a).nonzero()[:, 0], float(c["scaling"][a])
        x, A, B = c["x"][t].double(), c["A"][a, :r].double().t().contiguous(), c["B"][a, :, :r].double().t().contiguous()
        part[t] = k * ((x @ A) @ B)
        mag[t] = k * ((x.abs() @ A.abs()) @ B.abs())
    unit = (d_in + R + 8) * ref.E + _inner(dtype)
    h = fiona.Adapters(dtype, nA, R, d_in, d_out, n)
    for kind in ("base", "no base", "in place"):
        base = None if kind == "no base" else c["base"].clone()
        y = base if kind == "in place" else torch.full_like(c["base"], 7.0)
        fiona.adapter_linear(h, c["x"], c["ids"], c["A"], c["B"], base, y, ranks=c["ranks"], scaling=c["scaling"])
        want, m = (part, mag) if base is None else (part + c["base"].double(), mag + c["base"].double().abs())
        _close(y, want, 2 * (ref.U[dtype] * want.abs() + unit * m) + ref.TINY[dtype], kind)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,nA,R,d_in,d_out", SHAPES)
def test_backward(n, nA, R, d_in, d_out, dtype):
    c = _inputs(n, nA, R, d_in, d_out, dtype)
    part = torch.zeros(n, d_in, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(part)
    dA, dB = torch.zeros(nA, R, d_in, dtype=torch.float64, device="cuda"), torch.zeros(nA, d_out, R, dtype=torch.float64, device="cuda")
    mA, mB = torch.zeros_like(dA), torch.zeros_like(dB)
    for a, r in enumerate(c["ranks"].tolist()):
        t, k = (c["ids"] == a).nonzero()[:, 0], float(c["scaling"][a])
        x, dy, A, B = c["x"][t].double(), c["dy"][t].double(), c["A"][a, :r].double(), c["B"][a, :, :r].double().contiguous()
        At = A.t().contiguous()
        g, gm = k * (dy @ B), k * (dy.abs() @ B.abs())
        part[t], mag[t] = g @ A, gm @ A.abs()
        dA[a, :r], mA[a, :r] = g.t().contiguous() @ x, gm.t().contiguous() @ x.abs()
        dB[a, :, :r] = k * (dy.t().contiguous() @ (x @ At))
        mB[a, :, :r] = k * (dy.t().contiguous().abs() @ (x.abs() @ At.abs()))
    inner, u, tiny = _inner(dtype), ref.U[dtype], ref.TINY[dtype]
    ex, ea, eb = (d_out + R + 8) * ref.E + inner, (n + d_out + 8) * ref.E + 2 * inner, (n + d_in + 8) * ref.E + 2 * inner
    h = fiona.Adapters(dtype, nA, R, d_in, d_out, n)
    for kind in ("base", "no base", "in place"):
        base = None if kind == "no base" else c["dx_base"].clone()
        dx = base if kind == "in place" else torch.full_like(c["x"], 7.0)
        gA, gB = torch.full_like(c["A"], 7.0), torch.full_like(c["B"], 7.0)
        fiona.adapter_backward(h, c["x"], c["ids"], c["A"], c["B"], c["dy"], base, dx, gA, gB, ranks=c["ranks"], scaling=c["scaling"])
        want, m = (part, mag) if base is None else (part + c["dx_base"].double(), mag + c["dx_base"].double().abs())
        _close(dx, want, 2 * (u * want.abs() + ex * m) + tiny, kind + " dx")
        _close(gA, dA, 2 * (u * dA.abs() + ea * mA) + tiny, kind + " dA")
        _close(gB, dB, 2 * (u * dB.abs() + eb * mB) + tiny, kind + " dB")
