"""fiona_adapter_linear and fiona_adapter_backward against a plain form in 64
bits, and the gradients against differences of the forward pass."""
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


def _ids(kind, n, nA, g):
    if kind == "runs":
        return (torch.arange(n) * max(1, nA) // max(1, n)).int()
    if kind == "mixed":
        return torch.randint(-1, nA, (n,), generator=g, dtype=torch.int32)
    if kind == "one":
        return torch.full((n,), nA - 1, dtype=torch.int32)
    if kind == "none":
        return torch.full((n,), -1, dtype=torch.int32)
    bad = torch.randint(0, nA, (n,), generator=g, dtype=torch.int32)   # "outside": ids that are no adapter's
    bad[::2] = nA
    bad[::3] = -2 ** 31
    bad[::5] = 2 ** 31 - 1
    return bad


def _inputs(n, nA, R, d_in, d_out, dtype, kind, seed, low_ranks=True):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s, k=1.0: (k * torch.randn(*s, generator=g)).to(dtype)
    c = dict(x=rnd(n, d_in), A=rnd(nA, R, d_in, k=d_in ** -0.5), B=rnd(nA, d_out, R, k=0.5), base=rnd(n, d_out),
             dy=rnd(n, d_out), dx_base=rnd(n, d_in), ids=_ids(kind, n, nA, g), scaling=torch.randn(nA, generator=g),
             ranks=torch.tensor([R if i % 3 != 1 else max(0, R // 2) for i in range(nA)], dtype=torch.int32))
    if low_ranks and nA > 2:
        c["ranks"][2] = 0
    # what an adapter's rank leaves out holds anything
    for a in range(nA):
        c["A"][a, c["ranks"][a]:] = float("nan")
        c["B"][a, :, c["ranks"][a]:] = float("nan")
    return c


def _forward(c, dev, with_base=True, ranks=True, scaling=True, **over):
    t = {n: v.to(dev) for n, v in c.items()}
    t.update(over)
    n, d_in = t["x"].shape
    nA, d_out, R = t["B"].shape
    h = fiona.Adapters(t["A"].dtype, nA, R, d_in, d_out, max(1, n))
    y = over.get("y", torch.full((n, d_out), 7.0, dtype=t["A"].dtype, device=dev))
    fiona.adapter_linear(h, t["x"], t["ids"], t["A"], t["B"], t["base"] if with_base else None, y,
                         ranks=t["ranks"] if ranks else None, scaling=t["scaling"] if scaling else None)
    torch.cuda.synchronize()
    return y


def _backward(c, dev, with_base=True, **over):
    t = {n: v.to(dev) for n, v in c.items()}
    t.update(over)
    n, d_in = t["x"].shape
    nA, d_out, R = t["B"].shape
    h = fiona.Adapters(t["A"].dtype, nA, R, d_in, d_out, max(1, n))
    dx = over.get("dx", torch.full((n, d_in), 7.0, dtype=t["A"].dtype, device=dev))
    dA, dB = torch.full_like(t["A"], 7.0), torch.full_like(t["B"], 7.0)
    fiona.adapter_backward(h, t["x"], t["ids"], t["A"], t["B"], t["dy"], t["dx_base"] if with_base else None, dx, dA, dB,
                           ranks=t["ranks"], scaling=t["scaling"])
    torch.cuda.synchronize()
    return dx, dA, dB


def _check_forward(c, y, base=True, what=""):
    want, bound = ref.adapter(c["x"], c["ids"], c["A"], c["B"], c["base"] if base else None, c["ranks"], c["scaling"],
                              c["A"].dtype)
    ref.assert_close(y, want, bound, what + " y")


def _check_backward(c, got, base=True, what=""):
    want = ref.adapter_gradients(c["x"], c["ids"], c["A"], c["B"], c["dy"], c["dx_base"] if base else None, c["ranks"],
                                 c["scaling"], c["A"].dtype)
    for name, g, (y, b) in zip(("dx", "dA", "dB"), got, want):
        ref.assert_close(g, y, b, "%s %s" % (what, name))


SHAPES = [  # n, nA, R, d_in, d_out, ids
    (1, 1, 1, 1, 1, "one"), (1, 3, 8, 64, 96, "one"), (16, 16, 8, 768, 256, "runs"), (17, 4, 16, 100, 333, "mixed"),
    (33, 5, 20, 129, 65, "outside"), (5, 2, 4, 7, 1000, "mixed"), (64, 64, 16, 256, 512, "runs"), (40, 3, 64, 512, 128, "runs"),
    (21, 4, 128, 96, 160, "mixed"), (130, 2, 33, 72, 40, "runs"), (9, 2, 5, 2048, 64, "none"), (300, 3, 12, 64, 64, "mixed"),
    (1000, 2, 16, 48, 56, "runs"),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,nA,R,d_in,d_out,kind", SHAPES)
def test_forward(n, nA, R, d_in, d_out, kind, dtype):
    dev = _dev()
    c = _inputs(n, nA, R, d_in, d_out, dtype, kind, seed=n + R)
    _check_forward(c, _forward(c, dev), what=kind)
    _check_forward(c, _forward(c, dev, with_base=False), base=False, what=kind + " no base")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,nA,R,d_in,d_out,kind", SHAPES)
def test_backward(n, nA, R, d_in, d_out, kind, dtype):
    dev = _dev()
    c = _inputs(n, nA, R, d_in, d_out, dtype, kind, seed=n + R)
    _check_backward(c, _backward(c, dev), what=kind)
    _check_backward(c, _backward(c, dev, with_base=False), base=False, what=kind + " no base")


@pytest.mark.parametrize("n,d", [(2000, 64), (700, 320)])
def test_many_tokens_of_one_adapter(n, d):
    dev = _dev()
    c = _inputs(n, 1, 16, d, d, BF16, "one", seed=n)
    _check_forward(c, _forward(c, dev))
    _check_backward(c, _backward(c, dev))


def test_without_ranks_and_scaling():
    dev = _dev()
    c = _inputs(20, 3, 8, 64, 64, F32, "mixed", seed=3, low_ranks=False)
    for name in ("A", "B"):
        c[name] = torch.nan_to_num(c[name], nan=0.25)
    y = _forward(c, dev, ranks=False, scaling=False)
    c["ranks"][:], c["scaling"][:] = 8, 1.0
    _check_forward(c, y)


def test_ranks_outside_their_range_are_clamped():
    dev = _dev()
    c = _inputs(20, 3, 8, 64, 64, BF16, "mixed", seed=4, low_ranks=False)
    for name in ("A", "B"):
        c[name] = torch.nan_to_num(c[name], nan=0.25)
    given = torch.tensor([1 << 30, -7, 8], dtype=torch.int32)
    t = dict(c, ranks=given)
    y, grads = _forward(t, dev), _backward(t, dev)
    c["ranks"] = torch.tensor([8, 0, 8], dtype=torch.int32)
    _check_forward(c, y)
    _check_backward(c, grads)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_nan_rows_stay_with_their_own_tokens(dtype):
    """Another request's NaN or infinity reaches neither this request's rows nor its adapter's gradients."""
    dev = _dev()
    c = _inputs(48, 3, 16, 96, 96, dtype, "mixed", seed=6, low_ranks=False)
    clean_y, clean = _forward(c, dev), _backward(c, dev)
    poisoned = (c["ids"] == 0).nonzero()[:, 0]
    for name in ("x", "dy"):
        c[name][poisoned] = float("nan")
    c["A"][0], c["B"][0] = float("inf"), float("nan")
    y, (dx, dA, dB) = _forward(c, dev), _backward(c, dev)
    rest = (c["ids"] != 0).nonzero()[:, 0].to(dev)
    assert torch.equal(y[rest], clean_y[rest]) and torch.equal(dx[rest], clean[0][rest])
    assert torch.equal(dA[1:], clean[1][1:]) and torch.equal(dB[1:], clean[2][1:])
    assert bool(torch.isnan(y[poisoned.to(dev)]).all()) and bool(torch.isnan(dA[0]).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_values_outside_half_range_inside(dtype):
    """Inner values far above and below binary16's range, results inside it."""
    dev = _dev()
    c = _inputs(30, 2, 8, 256, 64, dtype, "runs", seed=8, low_ranks=False)
    c["x"] = (c["x"].float() * 3000).to(dtype)
    c["A"] = (c["A"].float() * 500).to(dtype)
    c["B"] = (c["B"].float() * 2 ** -13).to(dtype)
    c["scaling"] = torch.tensor([2.0 ** -10, 2.0 ** -8])
    _check_forward(c, _forward(c, dev), what="large inner values")
    c["x"] = (c["x"].float() * 2 ** -11).to(dtype)
    c["dy"] = (c["dy"].float() * 2 ** -6).to(dtype)
    _check_backward(c, _backward(c, dev), what="small gradients")


@pytest.mark.parametrize("shift", [0, 1])
def test_strided_rows_and_in_place(shift):
    dev = _dev()
    n, d_in, d_out = 25, 80, 104
    c = _inputs(n, 3, 16, d_in, d_out, BF16, "mixed", seed=10)
    room = torch.zeros(n, d_in + d_out + 24, dtype=BF16, device=dev)
    x, y = room[:, 8 + shift:8 + shift + d_in], room[:, 8 + d_in + 8 + shift:8 + d_in + 8 + shift + d_out]
    x.copy_(c["x"])
    y.copy_(c["base"])
    _forward(c, dev, x=x, base=y, y=y)               # side by side in one matrix, base updated in place
    _check_forward(c, y, what="in place")
    assert torch.equal(x.cpu(), c["x"])
    dx = c["dx_base"].to(dev)
    wide = torch.zeros(n, d_out + 9, dtype=BF16, device=dev)
    wide[:, shift:shift + d_out] = c["dy"].to(dev)
    grads = _backward(c, dev, x=x, dy=wide[:, shift:shift + d_out], dx_base=dx, dx=dx)
    _check_backward(c, grads, what="in place")


def test_broadcast_input_rows():
    dev = _dev()
    c = _inputs(18, 3, 8, 64, 64, F32, "mixed", seed=11)
    c["x"][:], c["base"][:] = c["x"][:1], c["base"][:1]
    y = _forward(c, dev, x=c["x"][:1].to(dev).expand(18, 64), base=c["base"][:1].to(dev).expand(18, 64))
    _check_forward(c, y)


def test_no_tokens():
    dev = _dev()
    c = _inputs(1, 2, 8, 64, 48, BF16, "one", seed=12)
    for n in ("x", "dy", "base", "dx_base", "ids"):
        c[n] = c[n][:0]
    _forward(c, dev)
    dx, dA, dB = _backward(c, dev)
    assert not bool(dA.any()) and not bool(dB.any())


@pytest.mark.parametrize("n,nA,R,d_in,d_out", [(50, 3, 8, 64, 96), (33, 2, 20, 50, 70)])
def test_gradients_against_differences(n, nA, R, d_in, d_out):
    """The loss sum(w y) is linear in each of x, A and B, so its central difference along any direction is
    exact up to rounding: (L(+D) - L(-D)) / 2 = <gradient, D>, with the forward pass in float32."""
    dev = _dev()
    c = _inputs(n, nA, R, d_in, d_out, F32, "mixed", seed=n, low_ranks=False)
    for name in ("A", "B"):
        c[name] = torch.nan_to_num(c[name], nan=0.0)
    dx, dA, dB = (t.cpu().double() for t in _backward(c, dev, with_base=False))
    g = torch.Generator().manual_seed(1)
    w = c["dy"].double()
    for name, grad in (("x", dx), ("A", dA), ("B", dB)):
        D = torch.randn(c[name].shape, generator=g) * c[name].std()
        ys = []
        for sign in (1, -1):
            y = _forward(dict(c, **{name: c[name] + sign * D}), dev, with_base=False)
            ys.append(y.cpu().double())
        diff = float(((ys[0] - ys[1]) / 2 * w).sum())
        want = float((grad * D.double()).sum())
        # each y carries at most (d_in + R + 8) 2^-24 of its products' magnitudes, and c + D is rounded once
        mag = ref.adapter(c["x"].abs() + (D.abs() if name == "x" else 0), c["ids"],
                          c["A"].abs() + (D.abs() if name == "A" else 0), c["B"].abs() + (D.abs() if name == "B" else 0),
                          None, c["ranks"], c["scaling"].abs(), F32)[0]
        bound = 4 * (d_in + d_out + n + R + 8) * ref.E * float((mag * w.abs()).sum())
        assert abs(diff - want) <= bound, (name, diff, want, bound)


def test_same_bits_twice_other_stream_and_graph_replay():
    dev = _dev()
    c = _inputs(200, 4, 16, 128, 192, BF16, "mixed", seed=15)
    t = {n: v.to(dev) for n, v in c.items()}
    h = fiona.Adapters(BF16, 4, 16, 128, 192, 200)
    y, dx = torch.empty_like(t["base"]), torch.empty_like(t["x"])
    dA, dB = torch.empty_like(t["A"]), torch.empty_like(t["B"])

    def call():
        kw = dict(ranks=t["ranks"], scaling=t["scaling"])
        fiona.adapter_linear(h, t["x"], t["ids"], t["A"], t["B"], t["base"], y, **kw)
        fiona.adapter_backward(h, t["x"], t["ids"], t["A"], t["B"], t["dy"], t["dx_base"], dx, dA, dB, **kw)

    outs = (y, dx, dA, dB)
    call()
    torch.cuda.synchronize()
    _check_forward(c, y)
    _check_backward(c, (dx, dA, dB))
    first = [o.clone() for o in outs]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, first))
    t["ids"].copy_(t["ids"].flip(0))       # the captured call follows the ids
    c["ids"] = c["ids"].flip(0)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    _check_forward(c, y)
    _check_backward(c, (dx, dA, dB))


def test_refusals():
    dev = _dev()
    for desc, status in [((BF16, 0, 8, 64, 64, 1), -1), ((BF16, 1, 0, 64, 64, 1), -1), ((BF16, 1, 129, 64, 64, 1), -3),
                         ((BF16, 1, 8, 0, 64, 1), -1), ((BF16, 1, 8, 64, 0, 1), -1), ((BF16, 1, 8, 64, 64, 0), -1),
                         ((BF16, 1, 8, (1 << 20) + 1, 64, 1), -3), ((BF16, 70000, 8, 64, 64, 1), -3)]:
        with pytest.raises(fiona.FionaError) as e:
            fiona.Adapters(*desc)
        assert e.value.status == status, desc
    c = _inputs(6, 2, 8, 64, 64, BF16, "mixed", seed=16)
    t = {n: v.to(dev) for n, v in c.items()}
    h = fiona.Adapters(BF16, 2, 8, 64, 64, 6)

    def forward(handle=h, **over):
        a = dict(t, y=torch.empty_like(t["base"]))
        a.update(over)
        fiona.adapter_linear(handle, a["x"], a["ids"], a["A"], a["B"], a["base"], a["y"])

    def backward(**over):
        a = dict(t, dx=torch.empty_like(t["x"]), dA=torch.empty_like(t["A"]), dB=torch.empty_like(t["B"]))
        a.update(over)
        fiona.adapter_backward(h, a["x"], a["ids"], a["A"], a["B"], a["dy"], a["dx_base"], a["dx"], a["dA"], a["dB"])

    def status(f, **over):
        with pytest.raises(fiona.FionaError) as e:
            f(**over)
        return e.value.status

    assert status(forward, y=t["x"]) == -5
    assert status(forward, y=torch.empty(1, 64, dtype=BF16, device=dev).expand(6, 64)) == -5
    both = torch.zeros(7, 64, dtype=BF16, device=dev)
    assert status(forward, base=both[:6], y=both[1:]) == -5        # base shifted by a row
    assert status(forward, handle=fiona.Adapters(BF16, 2, 8, 64, 64, 5)) == -1   # more tokens than the handle's
    assert status(backward, dA=t["A"]) == -5 and status(backward, dx=t["x"]) == -5 and status(backward, dB=t["B"]) == -5
    assert status(backward, dx=t["dy"]) == -5
    same = torch.zeros(2, 8, 64, dtype=BF16, device=dev)
    assert status(backward, dA=same, dB=same.view(2, 64, 8)) == -5
    for bad in (dict(ids=t["ids"].long()), dict(x=t["x"].float()), dict(A=t["A"][:1]), dict(B=t["B"].transpose(1, 2)),
                dict(y=torch.empty(6, 63, dtype=BF16, device=dev)), dict(ids=t["ids"].cpu())):
        with pytest.raises(ValueError):
            forward(**bad)
