"""Limits of the training step's operators: rows beyond 2^32 bytes, many pairs, rows left alone, graphs beside eager work."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import training_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _dev(gib=0):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("needs %d GiB" % gib)
    fiona.lib()
    return torch.device("cuda:0")


def _far(rows, dev):
    """The rows 2^32 elements apart (8 GiB in 16 bits)."""
    n, d = rows.shape
    store = torch.empty((n - 1) * 2 ** 32 + d, dtype=rows.dtype, device=dev)
    out = store.as_strided((n, d), (2 ** 32, 1))
    out.copy_(rows)
    return out


def test_rows_far_apart():
    dev = _dev(64)
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).to(BF16)
    x, w, b = r(2, 300), r(300), r(300)
    far, y = _far(x, dev), _far(torch.zeros(2, 300, dtype=BF16), dev)
    mean, rstd = torch.empty(2, device=dev), torch.empty(2, device=dev)
    fiona.layer_norm(far, w.to(dev), b.to(dev), y, mean=mean, rstd=rstd)
    want = ref.norm(x, None, w, b, 1e-5)
    ref.assert_close(y, want[1], want[2], "y")
    dw, db = torch.empty(300, dtype=BF16, device=dev), torch.empty(300, dtype=BF16, device=dev)
    dy = r(2, 300)
    fiona.layer_norm_backward(fiona.LayerNorm(BF16, 300, 2), dy.to(dev), far, w.to(dev), mean, rstd, None, y, dw, db)
    for got, (v, bound) in zip((y, dw, db), ref.norm_gradients(dy, x, w, mean.cpu(), rstd.cpu(), None, BF16)):
        ref.assert_close(got, v, bound, "gradients")
    z, t = r(2, 200), torch.tensor([3, 150], dtype=torch.int32)
    old = ref.scores(z, t)[0].float() - 0.1
    zf = _far(z, dev)
    loss, logps = torch.empty(2, device=dev), torch.empty(2, device=dev)
    one = torch.ones(2)
    fiona.policy_loss(fiona.TokenLoss(BF16, 200, 2), zf, t.to(dev), old.to(dev), one.to(dev), loss, logps, zf)
    (v, bound), _, (dz, bz) = ref.policy(z, t, old, one, old, None, 0.2, 0.2, 0.0)
    ref.assert_close(loss, v, bound, "loss")
    ref.assert_close(zf, dz, bz, "dlogits")


@pytest.mark.parametrize("V", [100000, 300000])
def test_logits_beyond_two_to_the_32_bytes(V):
    """Whole rows and parts of rows; the last rows lie past 4 GiB."""
    dev = _dev(48)
    n = 2 ** 32 // (2 * V) + 40
    z = torch.empty(n, V, dtype=BF16, device=dev).normal_(0, 2, generator=torch.Generator(device="cuda").manual_seed(2))
    t = torch.full((n,), -1, dtype=torch.int32, device=dev)
    last = [0, n - 30, n - 1]
    t[last] = torch.tensor([5, V - 1, 77], dtype=torch.int32, device=dev)
    rows, targets = z[last].cpu(), t[last].cpu()
    l = ref.scores(rows, targets)[0]
    old, adv = torch.zeros(n, device=dev), torch.ones(n, device=dev)
    old[last] = (l - 0.1).float().to(dev)
    loss, logps, dz = torch.empty(n, device=dev), torch.empty(n, device=dev), torch.empty_like(z)
    h = fiona.TokenLoss(BF16, V, n, 1)
    fiona.policy_loss(h, z, t, old, adv, loss, logps, dz, weights=adv)
    want = ref.policy(rows, targets, (l - 0.1).float(), torch.ones(3), old[:3].cpu(), torch.ones(3), 0.2, 0.2, 0.0)
    for got, (v, b) in zip((loss[last], logps[last], dz[last]), want):
        ref.assert_close(got, v, b, "policy")
    offsets = torch.tensor([0, 1, n], dtype=torch.int32, device=dev)
    reference, one, two = torch.zeros(2, device=dev), torch.empty(1, device=dev), torch.empty(2, device=dev)
    fiona.preference_loss(h, z, t, offsets, reference, one, two, dz, beta=0.01)
    want = ref.preference(rows, targets, torch.tensor([0, 1, 3]), torch.zeros(2), None, 0.01, 0.0)
    for got, (v, b) in zip((one, two, dz[last]), want):
        ref.assert_close(got, v, b, "preference")
    others = torch.ones(n, dtype=torch.bool, device=dev)
    others[last] = False
    assert not any(bool(rows.any()) for rows in dz[others].split(2000))


def test_many_pairs():
    dev = _dev()
    g = torch.Generator().manual_seed(3)
    P, V = 3000, 40
    lengths = torch.randint(0, 3, (2 * P,), generator=g)
    off = torch.cat((torch.zeros(1, dtype=torch.long), lengths.cumsum(0))).int()
    n = int(off[-1])
    z, t = torch.randn(n, V, generator=g), torch.randint(-1, V, (n,), generator=g, dtype=torch.int32)
    r = torch.randn(2 * P, generator=g)
    loss, logps, dz = torch.empty(P, device=dev), torch.empty(2 * P, device=dev), torch.empty(n, V, device=dev)
    fiona.preference_loss(fiona.TokenLoss(F32, V, n, P), z.to(dev), t.to(dev), off.to(dev), r.to(dev), loss, logps, dz, beta=0.5)
    for got, (v, b) in zip((loss, logps, dz), ref.preference(z, t, off, r, None, 0.5, 0.0)):
        ref.assert_close(got, v, b, "many pairs")


def test_captured_beside_eager_calls_on_handles_of_their_own():
    """A captured training step replayed between eager calls of other sizes: each has its own workspace."""
    dev = _dev()
    g = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=g).to(dev)
    n, d, V = 60, 96, 700
    x, w, b, dy, z = r(n, d), r(d), r(d), r(n, d), r(n, V)
    t = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).to(dev)
    off, ref_l = torch.tensor([0, 20, 60], dtype=torch.int32, device=dev), torch.zeros(2, device=dev)
    lr, step = torch.full((1,), 0.0, device=dev), torch.ones(1, dtype=torch.int32, device=dev)

    def make():
        o = dict(y=torch.empty_like(x), mean=torch.empty(n, device=dev), rstd=torch.empty(n, device=dev), dx=torch.empty_like(x),
                 dw=torch.empty_like(w), db=torch.empty_like(b), loss=torch.empty(1, device=dev), logps=torch.empty(2, device=dev),
                 dz=torch.empty_like(z))
        ln, tl = fiona.LayerNorm(F32, d, n), fiona.TokenLoss(F32, V, n, 1)
        m, v = torch.zeros_like(w), torch.zeros_like(w)
        opt = fiona.AdamW([w], [o["dw"]], [m], [v])

        def call():
            fiona.layer_norm(x, w, b, o["y"], mean=o["mean"], rstd=o["rstd"])
            fiona.preference_loss(tl, z, t, off, ref_l, o["loss"], o["logps"], o["dz"])
            fiona.layer_norm_backward(ln, dy, x, w, o["mean"], o["rstd"], None, o["dx"], o["dw"], o["db"])
            fiona.adamw_step(opt, lr, step)

        return o, call

    eager, call = make()
    call()
    torch.cuda.synchronize()
    captured, record = make()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        record()
    small = fiona.TokenLoss(F32, 50, 9), fiona.LayerNorm(F32, 31, 9)
    for _ in range(3):
        for o in captured.values():
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        zs, ys = r(9, 50), r(9, 31)
        fiona.policy_loss(small[0], zs, t[:9] % 50, torch.zeros(9, device=dev), torch.ones(9, device=dev), torch.empty(9, device=dev),
                          torch.empty(9, device=dev), zs)
        fiona.layer_norm_backward(small[1], ys, ys, None, torch.zeros(9, device=dev), torch.ones(9, device=dev), None, ys.clone(),
                                  torch.empty(31, device=dev))
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(captured[k], eager[k]) for k in eager)


def test_an_optimisers_memory_outlives_the_tensors_given():
    dev = _dev()
    p, g = torch.ones(5000, device=dev), torch.ones(5000, device=dev)
    kept = p
    opt = fiona.AdamW([p], [g], [torch.zeros(5000, device=dev)], [torch.zeros(5000, device=dev)], weight_decay=0.0)
    p.data = torch.zeros(3, device=dev)                # the tensor is given other memory
    del g
    torch.cuda.empty_cache()
    fiona.adamw_step(opt, torch.full((1,), 0.1, device=dev), torch.ones(1, dtype=torch.int32, device=dev))
    torch.cuda.synchronize()
    assert not kept.any() and kept.numel() == 3
