"""fiona_layer_norm and fiona_layer_norm_backward against plain forms in 64 bits, and the gradients against differences."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import training_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 1e-5


def _dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fiona.lib()
    return torch.device("cuda:0")


def _inputs(n, d, dtype, wt, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, k=1.0, m=0.0: (m + k * torch.randn(*s, generator=g))
    return dict(x=r(n, d, m=0.3).to(dtype), residual=r(n, d, k=2.0).to(dtype), weight=r(d, k=0.3, m=1.0).to(wt),
                bias=r(d, k=0.3).to(wt), dy=r(n, d).to(dtype), dx_base=r(n, d).to(dtype))


def _forward(c, dev, residual=True, affine=True, eps=EPS):
    n, d = c["x"].shape
    t = {k: v.to(dev) for k, v in c.items()}
    new = lambda: torch.full((n, d), 7.0, dtype=c["x"].dtype, device=dev)
    y, total = new(), new() if residual else None
    mean, rstd = torch.full((n,), 7.0, device=dev), torch.full((n,), 7.0, device=dev)
    fiona.layer_norm(t["x"], t["weight"] if affine else None, t["bias"] if affine else None, y, eps=eps,
                     residual=t["residual"] if residual else None, total=total, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    return y, total, mean, rstd


def _check_forward(c, got, residual=True, affine=True, eps=EPS):
    y, total, mean, rstd = got
    want = ref.norm(c["x"], c["residual"] if residual else None, c["weight"] if affine else None, c["bias"] if affine else None, eps)
    if residual:
        assert torch.equal(total.cpu(), want[0])
    ref.assert_close(y, want[1], want[2], "y")
    ref.assert_close(mean, want[3], want[4], "mean")
    ref.assert_close(rstd, want[5], want[6], "rstd")


def _stats(c):
    x = c["x"].float()
    mean = x.mean(1)
    return mean, ((x - mean[:, None]).square().mean(1) + EPS) ** -0.5


def _backward(c, dev, base=True, affine=True, sums=True, handle=None):
    n, d = c["x"].shape
    t = {k: v.to(dev) for k, v in c.items()}
    mean, rstd = (s.to(dev) for s in _stats(c))
    wt = c["weight"].dtype
    h = handle or fiona.LayerNorm(c["x"].dtype, d, max(1, n), weight_dtype=wt)
    dx = torch.full((n, d), 7.0, dtype=c["x"].dtype, device=dev)
    dw, db = (torch.full((d,), 7.0, dtype=wt, device=dev) for _ in range(2)) if sums else (None, None)
    fiona.layer_norm_backward(h, t["dy"], t["x"], t["weight"] if affine else None, mean, rstd, t["dx_base"] if base else None, dx, dw, db)
    torch.cuda.synchronize()
    return dx, dw, db


def _check_backward(c, got, base=True, affine=True):
    mean, rstd = _stats(c)
    want = ref.norm_gradients(c["dy"], c["x"], c["weight"] if affine else None, mean, rstd, c["dx_base"] if base else None,
                              c["weight"].dtype)
    for name, g, (w, b) in zip(("dx", "dweight", "dbias"), got, want):
        if g is not None:
            ref.assert_close(g, w, b, name)


SHAPES = [(1, 1), (3, 5), (1, 768), (8, 768), (33, 1000), (17, 1373), (5, 2048), (6, 4096), (3, 5000), (2, 8192), (3, 16384),
          (2, 20011), (2, 32768), (5, 700), (3, 2500), (2, 9001), (300, 64), (1000, 7), (515, 257), (2049, 96)]
TYPES = [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)]


@pytest.mark.parametrize("dtype,wt", TYPES)
@pytest.mark.parametrize("n,d", SHAPES)
def test_forward(n, d, dtype, wt):
    dev = _dev()
    c = _inputs(n, d, dtype, wt, seed=n + d)
    _check_forward(c, _forward(c, dev))
    _check_forward(c, _forward(c, dev, residual=False, affine=False), residual=False, affine=False)


@pytest.mark.parametrize("dtype,wt", TYPES)
@pytest.mark.parametrize("n,d", SHAPES)
def test_backward(n, d, dtype, wt):
    dev = _dev()
    c = _inputs(n, d, dtype, wt, seed=n + d)
    _check_backward(c, _backward(c, dev))
    _check_backward(c, _backward(c, dev, base=False, affine=False), base=False, affine=False)
    _check_backward(c, _backward(c, dev, sums=False))


@pytest.mark.parametrize("dtype,n,d", [(F16, 2, 1373), (F16, 3, 1373), (F16, 1025, 1373), (BF16, 4099, 1100), (F16, 513, 4096), (BF16, 300, 8190),
                                       (F32, 4, 2500), (F32, 770, 1030), (F32, 300, 4099), (F32, 18, 999), (F32, 2051, 771), (BF16, 4101, 509),
                                       (BF16, 1026, 1500), (F16, 4110, 1100), (F16, 2051, 2500), (BF16, 3, 2001), (BF16, 515, 5001), (F32, 4, 1300), (F32, 1029, 1500)])
def test_backward_of_more_rows_than_groups(dtype, n, d):
    """Rows that fill one workgroup's groups, leave one of them a row short, or come again after every group's first."""
    dev = _dev()
    c = _inputs(n, d, dtype, F32, seed=n + d)
    _check_backward(c, _backward(c, dev))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_mean_far_from_zero(dtype):
    """Deviations of one part in 300: the square's mean less the mean's square would lose them in 32 bits."""
    dev = _dev()
    c = _inputs(9, 1000, dtype, F32, seed=5)
    c["x"] = (300 + torch.randn(9, 1000, generator=torch.Generator().manual_seed(6))).to(dtype)
    _check_forward(c, _forward(c, dev, residual=False), residual=False)
    c["x"][:] = 300                                    # no deviation at all
    _check_forward(c, _forward(c, dev, residual=False), residual=False)


def test_gradients_against_differences():
    """d loss / d (x, weight, bias) of loss = sum(a * y): the forward pass at both ends of a small step, in 64 bits."""
    dev = _dev()
    c = _inputs(7, 50, F32, F32, seed=8)
    a = c["dy"].double()
    dx, dw, db = (t.cpu().double() for t in _backward(c, dev, base=False))

    def loss(x, w, b):
        m = x.mean(1, keepdim=True)
        return float((a * ((x - m) * ((x - m).square().mean(1, keepdim=True) + EPS) ** -0.5 * w + b)).sum())

    g = torch.Generator().manual_seed(9)
    at = [c[k].double() for k in ("x", "weight", "bias")]
    for i, got in enumerate((dx, dw, db)):
        way = torch.randn(at[i].shape, generator=g, dtype=torch.float64)
        ends = []
        for sign in (1, -1):
            p = list(at)
            p[i] = at[i] + sign * 1e-5 * way
            ends.append(loss(*p))
        want, have = (ends[0] - ends[1]) / 2e-5, float((got * way).sum())
        # 64-bit differences: 1e-10 of the curvature and 1e-11 of cancellation; the kernel's 32-bit values
        assert abs(want - have) <= 1e-6 + 1e-5 * float((got * way).abs().sum()), i


def _spaced(t, dev, gap, shift):
    """The rows `gap` elements further apart than their width, from element `shift` on; everything else 7."""
    n, d = t.shape
    store = torch.full((n * (d + gap) + shift + 8,), 7.0, dtype=t.dtype, device=dev)
    rows = store.as_strided((n, d), (d + gap, 1), shift)
    rows.copy_(t)
    return store, rows


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("d", [5, 64, 1373, 4096, 9000])
def test_strides_and_alignments(d, dtype):
    dev = _dev()
    n = 5
    c = _inputs(n, d, dtype, F32, seed=d)
    t = {k: _spaced(v, dev, gap, shift)[1] for (k, v), gap, shift in
         zip(((k, c[k]) for k in ("x", "residual", "dy", "dx_base")), (3, 8, 1, 5), (1, 8, 3, 0))}
    w, b = c["weight"].to(dev), c["bias"].to(dev)
    store_y, y = _spaced(c["x"], dev, 5, 3)
    store_t, total = _spaced(c["x"], dev, 1, 1)
    mean, rstd = torch.empty(n, device=dev), torch.empty(n, device=dev)
    fiona.layer_norm(t["x"], w, b, y, residual=t["residual"], total=total, mean=mean, rstd=rstd)
    _check_forward(c, (y, total, mean, rstd))
    store_g, dx = _spaced(c["x"], dev, 7, 1)
    m, r = (s.to(dev) for s in _stats(c))
    dw, db = torch.empty(d, device=dev), torch.empty(d, device=dev)
    fiona.layer_norm_backward(fiona.LayerNorm(dtype, d, n, weight_dtype=F32), t["dy"], t["x"], w, m, r, t["dx_base"], dx, dw, db)
    _check_backward(c, (dx, dw, db))
    for store, rows in ((store_y, y), (store_t, total), (store_g, dx)):   # nothing beside the rows is written
        rows.fill_(7.0)
        assert bool((store == 7).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [768, 4096, 9000])
def test_in_place(d, dtype):
    dev = _dev()
    c = _inputs(6, d, dtype, F32, seed=11)
    y, total, mean, rstd = _forward(c, dev)
    w, b = c["weight"].to(dev), c["bias"].to(dev)
    for first in ("x", "residual"):
        x, r = c["x"].to(dev), c["residual"].to(dev)
        outs = (x, r) if first == "x" else (r, x)
        fiona.layer_norm(x, w, b, outs[0], residual=r, total=outs[1])
        assert torch.equal(outs[0], y) and torch.equal(outs[1], total), first
    dx, dw, db = _backward(c, dev)
    mean, rstd = (s.to(dev) for s in _stats(c))
    for own in ("dy", "x", "dx_base"):
        t = {k: v.to(dev) for k, v in c.items()}
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        fiona.layer_norm_backward(fiona.LayerNorm(dtype, d, 6, weight_dtype=F32), t["dy"], t["x"], w, mean, rstd, t["dx_base"], t[own],
                                  dw2, db2)
        assert torch.equal(t[own], dx) and torch.equal(dw2, dw) and torch.equal(db2, db), own


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 4096])
def test_infinities_stay_with_their_row(d, dtype):
    dev = _dev()
    c = _inputs(40, d, dtype, F32, seed=12)
    y = _forward(c, dev, residual=False)[0]
    dx = _backward(c, dev)[0]
    bad = dict(c, x=c["x"].clone(), dy=c["dy"].clone())
    bad["x"][7, 3], bad["dy"][7, 5] = float("inf"), float("nan")
    others = [i for i in range(40) if i != 7]
    z = _forward(bad, dev, residual=False)[0]
    assert torch.equal(z[others], y[others]) and bool(torch.isnan(z[7]).any())
    bad["x"] = c["x"]
    dz = _backward(bad, dev)[0]
    assert torch.equal(dz[others], dx[others]) and bool(torch.isnan(dz[7]).all())


def test_rows_that_are_one_row():
    """Inputs whose rows lie over each other (a stride of zero)."""
    dev = _dev()
    c = _inputs(9, 96, BF16, F32, seed=13)
    for k in ("x", "residual", "dy", "dx_base"):
        c[k] = c[k][:1].expand(9, 96)
    t = {k: (v[:1].to(dev).expand(9, 96) if v.dim() == 2 else v.to(dev)) for k, v in c.items()}
    y, total = torch.empty(9, 96, dtype=BF16, device=dev), torch.empty(9, 96, dtype=BF16, device=dev)
    mean, rstd = torch.empty(9, device=dev), torch.empty(9, device=dev)
    fiona.layer_norm(t["x"], t["weight"], t["bias"], y, residual=t["residual"], total=total, mean=mean, rstd=rstd)
    _check_forward(c, (y, total, mean, rstd))
    m, r = (s.to(dev) for s in _stats(c))
    dx, dw, db = torch.empty_like(y), torch.empty(96, device=dev), torch.empty(96, device=dev)
    fiona.layer_norm_backward(fiona.LayerNorm(BF16, 96, 9, weight_dtype=F32), t["dy"], t["x"], t["weight"], m, r, t["dx_base"], dx, dw, db)
    _check_backward(c, (dx, dw, db))


def test_no_rows():
    dev = _dev()
    e = torch.empty(0, 64, dtype=BF16, device=dev)
    w, none = torch.ones(64, dtype=BF16, device=dev), torch.empty(0, device=dev)
    fiona.layer_norm(e, w, w, e.clone())
    dw, db = torch.full_like(w, 7), torch.full_like(w, 7)
    fiona.layer_norm_backward(fiona.LayerNorm(BF16, 64, 4), e, e, w, none, none, None, e.clone(), dw, db)
    assert not dw.any() and not db.any()


def test_a_handle_for_more_rows_and_one_sum_alone():
    dev = _dev()
    c = _inputs(70, 320, BF16, F32, seed=14)
    dx, dw, db = _backward(c, dev)
    big = fiona.LayerNorm(BF16, 320, 9000, weight_dtype=F32)
    again = _backward(c, dev, handle=big)
    _check_backward(c, again)
    t = {k: v.to(dev) for k, v in c.items()}
    m, r = (s.to(dev) for s in _stats(c))
    for which in ("dweight", "dbias"):
        one = torch.full((320,), 7.0, device=dev)
        fiona.layer_norm_backward(big, t["dy"], t["x"], t["weight"], m, r, t["dx_base"], torch.empty_like(t["x"]), **{which: one})
        assert torch.equal(one, again[1 if which == "dweight" else 2])


@pytest.mark.parametrize("n,d", [(200, 192), (1500, 2048)])
def test_same_bits_twice_other_stream_and_graph_replay(n, d):
    dev = _dev()
    c = _inputs(n, d, BF16, BF16, seed=15)
    t = {k: v.to(dev) for k, v in c.items()}
    m, r = (s.to(dev) for s in _stats(c))
    h = fiona.LayerNorm(BF16, d, n)
    y, total, dx = (torch.empty_like(t["x"]) for _ in range(3))
    mean, rstd = torch.empty(n, device=dev), torch.empty(n, device=dev)
    dw, db = torch.empty_like(t["weight"]), torch.empty_like(t["bias"])

    def call():
        fiona.layer_norm(t["x"], t["weight"], t["bias"], y, residual=t["residual"], total=total, mean=mean, rstd=rstd)
        fiona.layer_norm_backward(h, t["dy"], t["x"], t["weight"], m, r, t["dx_base"], dx, dw, db)

    outs = (y, total, mean, rstd, dx, dw, db)
    call()
    torch.cuda.synchronize()
    _check_forward(c, outs[:4])
    _check_backward(c, outs[4:])
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


def test_refusals():
    dev = _dev()
    c = _inputs(6, 64, BF16, F32, seed=16)
    t = {k: v.to(dev) for k, v in c.items()}
    new = lambda: torch.empty_like(t["x"])

    def forward(**over):
        a = dict(x=t["x"], weight=t["weight"], bias=t["bias"], y=new(), residual=t["residual"], total=new())
        a.update(over)
        fiona.layer_norm(**a)

    h = fiona.LayerNorm(BF16, 64, 6, weight_dtype=F32)
    m, r = (s.to(dev) for s in _stats(c))

    def backward(ln=h, **over):
        a = dict(dy=t["dy"], x=t["x"], weight=t["weight"], mean=m, rstd=r, dx_base=t["dx_base"], dx=new(),
                 dweight=torch.empty(64, device=dev), dbias=torch.empty(64, device=dev))
        a.update(over)
        fiona.layer_norm_backward(ln, **a)

    def status(f, **over):
        with pytest.raises(fiona.FionaError) as e:
            f(**over)
        return e.value.status

    both = torch.zeros(7, 64, dtype=BF16, device=dev)
    same = new()
    assert status(forward, y=same, total=same) == -5 and status(forward, x=both[:6], y=both[1:]) == -5
    assert status(forward, y=both[:1].expand(6, 64)) == -5
    assert status(forward, eps=0.0) == -1 and status(forward, eps=float("nan")) == -1
    stats = torch.zeros(6, device=dev)
    assert status(forward, mean=stats, rstd=stats) == -5
    wide = torch.zeros(1, 32769, dtype=BF16, device=dev)
    assert status(forward, x=wide, weight=None, bias=None, y=wide.clone(), residual=None, total=None) == -3
    assert status(backward, ln=fiona.LayerNorm(BF16, 64, 5, weight_dtype=F32)) == -1          # more rows than the handle's
    sums = torch.zeros(64, device=dev)
    assert status(backward, dweight=sums, dbias=sums) == -5 and status(backward, dweight=t["weight"]) == -5
    assert status(backward, x=both[:6], dx=both[1:]) == -5
    for bad in (dict(y=new().float()), dict(weight=t["weight"][:63]), dict(bias=t["bias"].to(BF16)), dict(residual=t["residual"].cpu()),
                dict(y=torch.empty(6, 128, dtype=BF16, device=dev)[:, ::2])):
        with pytest.raises(ValueError):
            forward(**bad)
    for desc, status_ in [((BF16, 0, 4), -1), ((BF16, 64, 0), -1), ((BF16, 32769, 4), -3), ((BF16, 64, 4, F16), -3)]:
        with pytest.raises(fiona.FionaError) as e:
            fiona.LayerNorm(*desc)
        assert e.value.status == status_, desc
