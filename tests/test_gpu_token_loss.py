"""fiona_preference_loss and fiona_policy_loss against plain forms in 64 bits, and their gradients against differences."""
import pytest

import paper_2609_35352_amd as fiona

torch = pytest.importorskip("torch")
import training_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fiona.lib()
    return torch.device("cuda:0")


def _logits(n, V, dtype, g):
    z = (2 * torch.randn(n, V, generator=g)).to(dtype)
    y = torch.randint(V, (n,), generator=g, dtype=torch.int32)
    z[torch.arange(n), y.long()] += (6 * torch.rand(n, generator=g)).to(dtype)
    return z, y


def _pairs(lengths, V, dtype, seed, masked=0.25):
    """lengths: of the sequences; before the first and behind the last lie tokens of none."""
    g = torch.Generator().manual_seed(seed)
    ends = torch.cumsum(torch.tensor([1] + lengths), 0)
    n = int(ends[-1]) + 2
    z, y = _logits(n, V, dtype, g)
    off = torch.rand(n, generator=g) < masked
    y[off] = torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)[torch.arange(int(off.sum())) % 4]
    z[off] = float("nan")                            # rows that do not count hold anything
    p = len(lengths) // 2
    l = ref.scores(torch.nan_to_num(z), y)[0]
    L = torch.stack([l[a:b].sum() for a, b in zip(ends[:-1], ends[1:])]) if lengths else torch.zeros(0)
    return dict(logits=z, targets=y, offsets=ends.int(), reference=(L + 4 * torch.randn(2 * p, generator=g)).float(),
                weights=torch.randn(p, generator=g))


def _prefer(c, dev, weights=True, gradient=True, handle=None, beta=0.1, smoothing=0.0):
    n, V = c["logits"].shape
    p = len(c["reference"]) // 2
    t = {k: v.to(dev) for k, v in c.items()}
    h = handle or fiona.TokenLoss(c["logits"].dtype, V, max(1, n), p)
    loss, logps = torch.full((p,), 7.0, device=dev), torch.full((2 * p,), 7.0, device=dev)
    dz = torch.full_like(t["logits"], 7.0) if gradient else None
    fiona.preference_loss(h, t["logits"], t["targets"], t["offsets"], t["reference"], loss, logps, dz, beta=beta,
                          label_smoothing=smoothing, weights=t["weights"] if weights else None)
    torch.cuda.synchronize()
    return loss, logps, dz


def _check_prefer(c, got, weights=True, beta=0.1, smoothing=0.0):
    want = ref.preference(c["logits"], c["targets"], c["offsets"], c["reference"], c["weights"] if weights else None, beta, smoothing)
    for name, g, (w, b) in zip(("loss", "logps", "dlogits"), got, want):
        if g is not None:
            ref.assert_close(g, w, b, name)


def _tokens(n, V, dtype, seed, masked=0.25, clip=(0.2, 0.2)):
    g = torch.Generator().manual_seed(seed)
    z, y = _logits(n, V, dtype, g)
    off = torch.rand(n, generator=g) < masked
    l = ref.scores(z, y)[0]
    shift = 0.3 * torch.randn(n, generator=g).double()
    # off the clip's ends, where the derivative jumps: by more than a log-probability in 32 bits is off
    for end in (1 - clip[0], 1 + clip[1]):
        if end > 0:
            at = torch.tensor(end, dtype=torch.float64).log()
            shift = torch.where((shift - at).abs() < 2e-3, at + 4e-3, shift)
    c = dict(logits=z, targets=y, old=(l - shift).float(), advantages=torch.randn(n, generator=g),
             reference=(l + 0.4 * torch.randn(n, generator=g)).float(), weights=torch.randn(n, generator=g))
    y[off] = torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)[torch.arange(int(off.sum())) % 4]
    for k in ("logits", "old", "advantages", "reference"):
        c[k][off] = float("nan")
    return c


def _policy(c, dev, weights=True, gradient=True, handle=None, kl=0.05, clip=(0.2, 0.2)):
    n, V = c["logits"].shape
    t = {k: v.to(dev) for k, v in c.items()}
    h = handle or fiona.TokenLoss(c["logits"].dtype, V, max(1, n))
    loss, logps = torch.full((n,), 7.0, device=dev), torch.full((n,), 7.0, device=dev)
    dz = torch.full_like(t["logits"], 7.0) if gradient else None
    fiona.policy_loss(h, t["logits"], t["targets"], t["old"], t["advantages"], loss, logps, dz,
                      reference=t["reference"] if kl else None, clip_low=clip[0], clip_high=clip[1], kl=kl,
                      weights=t["weights"] if weights else None)
    torch.cuda.synchronize()
    return loss, logps, dz


def _check_policy(c, got, weights=True, kl=0.05, clip=(0.2, 0.2)):
    want = ref.policy(c["logits"], c["targets"], c["old"], c["advantages"], c["reference"], c["weights"] if weights else None, *clip, kl)
    for name, g, (w, b) in zip(("loss", "logps", "dlogits"), got, want):
        if g is not None:
            ref.assert_close(g, w, b, name)


LENGTHS = [([1, 1], 1), ([3, 2], 7), ([5, 0, 1, 9], 100), ([4, 6], 1000), ([12, 7, 3, 30, 0, 0], 2049), ([2, 3], 32000), ([3, 2, 4, 1], 50021),
           ([1, 2], 131072), ([300, 280], 64), ([2, 1], 300007)]
ROWS = [(1, 1), (5, 7), (33, 100), (9, 1000), (40, 2049), (4, 32000), (5, 50021), (3, 131072), (700, 64), (1, 300007), (2, 8191)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("lengths,V", LENGTHS)
def test_preference(lengths, V, dtype):
    dev = _dev()
    c = _pairs(lengths, V, dtype, seed=len(lengths) + V)
    _check_prefer(c, _prefer(c, dev))
    _check_prefer(c, _prefer(c, dev, weights=False, smoothing=0.1, beta=0.5), weights=False, smoothing=0.1, beta=0.5)
    got = _prefer(c, dev, gradient=False)
    _check_prefer(c, got)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,V", ROWS)
def test_policy(n, V, dtype):
    dev = _dev()
    c = _tokens(n, V, dtype, seed=n + V)
    _check_policy(c, _policy(c, dev))
    c = _tokens(n, V, dtype, seed=n + V, clip=(0.1, 0.3))
    _check_policy(c, _policy(c, dev, weights=False, kl=0.0, clip=(0.1, 0.3)), weights=False, kl=0.0, clip=(0.1, 0.3))
    _check_policy(c, _policy(c, dev, gradient=False, clip=(0.1, 0.3)), clip=(0.1, 0.3))


def test_many_tokens():
    """More rows than fill the GPU once, and sequences of hundreds of tokens."""
    dev = _dev()
    c = _pairs([700, 650, 3, 500], 1500, BF16, seed=3)
    _check_prefer(c, _prefer(c, dev))
    c = _tokens(2100, 1500, BF16, seed=4)
    _check_policy(c, _policy(c, dev))


@pytest.mark.parametrize("n,V,dtype", [(300, 2000, F16), (300, 20000, F32), (270, 30000, BF16), (260, 50016, F16), (100, 70000, F32), (105, 152064, BF16),
                                       (90, 131072, F16), (60, 65536, F32), (40, 50016, BF16), (258, 70000, BF16), (257, 131072, F16), (259, 98301, BF16),
                                       (258, 120001, BF16), (257, 33000, F32), (258, 64000, F32)])
def test_policy_of_whole_rows(n, V, dtype):
    """Rows that a workgroup holds whole, in registers alone and partly in LDS, for more and fewer rows than compute units."""
    dev = _dev()
    c = _tokens(n, V, dtype, seed=n + V)
    _check_policy(c, _policy(c, dev))


def test_no_token_counts():
    dev = _dev()
    c = _pairs([3, 4], 500, F32, seed=5, masked=2.0)
    _check_prefer(c, _prefer(c, dev))
    c = _tokens(6, 500, F32, seed=6, masked=2.0)
    loss, logps, dz = _policy(c, dev)
    assert not loss.any() and not logps.any() and not dz.any()


def test_nothing_at_all():
    dev = _dev()
    h = fiona.TokenLoss(F32, 10, 4, 2)
    e, i32 = torch.empty(0, device=dev), torch.empty(0, dtype=torch.int32, device=dev)
    z = torch.empty(0, 10, device=dev)
    fiona.policy_loss(h, z, i32, e, e, e.clone(), e.clone(), z.clone())
    loss, logps = torch.full((1,), 7.0, device=dev), torch.full((2,), 7.0, device=dev)
    offsets, zero = torch.zeros(3, dtype=torch.int32, device=dev), torch.zeros(2, device=dev)
    fiona.preference_loss(h, z, i32, offsets, zero, loss, logps, z.clone())
    assert abs(float(loss) - 0.6931472) < 1e-6 and not logps.any()        # two empty sequences: h = 0
    z, y = torch.randn(3, 10, device=dev), torch.zeros(3, dtype=torch.int32, device=dev)
    dz = torch.full_like(z, 7.0)
    fiona.preference_loss(h, z, y, offsets[:1], e, e.clone(), e.clone(), dz)      # no pairs: no token counts
    assert not dz.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_and_infinite_logits(dtype):
    dev = _dev()
    c = _tokens(6, 3000, dtype, seed=7, masked=0.0)
    z = c["logits"]
    z[0] += 3e4                                           # far from zero
    z[1, 5:2000] = float("-inf")                          # a vocabulary cut down
    z[1, int(c["targets"][1])] = 1.0
    z[2, :] = -300.0                                      # all but one far below
    z[2, int(c["targets"][2])] = 300.0
    z[3, :] = float("-inf")                               # only the target is left
    z[3, int(c["targets"][3])] = 2.0
    l = ref.scores(z, c["targets"])[0]
    c["old"] = (l - 0.1).float()
    c["reference"] = (l + 0.3).float()
    _check_policy(c, _policy(c, dev))


def test_rows_without_a_number_stay_with_their_token():
    dev = _dev()
    c = _tokens(8, 900, F32, seed=8, masked=0.0)
    want = _policy(c, dev)
    c["logits"][3, 10] = float("nan")
    c["logits"][5] = float("-inf")
    got = _policy(c, dev)
    others = [i for i in range(8) if i not in (3, 5)]
    for g, w in zip(got, want):
        assert torch.equal(g[others], w[others])
        assert bool(torch.isnan(g[3]).all()) and bool(torch.isnan(g[5]).all())


def test_offsets_outside_the_tokens_are_clamped():
    dev = _dev()
    c = _pairs([4, 5], 200, F32, seed=9)
    c["offsets"] = torch.tensor([-5, 3, 2 ** 31 - 1], dtype=torch.int32)
    _check_prefer(c, _prefer(c, dev))
    c["offsets"] = torch.tensor([6, 6, 2], dtype=torch.int32)              # an end before its start: empty
    _check_prefer(c, _prefer(c, dev))


def test_a_weight_of_zero_gives_zeros():
    dev = _dev()
    c = _pairs([4, 5, 6, 2], 200, F32, seed=10, masked=0.0)
    c["weights"][1] = 0
    c["logits"][11, 3] = float("nan")             # of the pair without weight
    loss, logps, dz = _prefer(c, dev)
    assert not dz[10:18].any() and bool((dz[1:10] != 0).any(1).all())


def test_ratios_at_the_clips_ends():
    """Where the clipped and the free product are the same the free one's derivative is taken; a ratio of one with a clip of
    zero is such a place for either sign."""
    dev = _dev()
    c = _tokens(4, 50, F32, seed=11, masked=0.0)
    z, h = torch.zeros(4, 50, device=dev), fiona.TokenLoss(F32, 50, 4)
    y = c["targets"].to(dev)
    loss, logps = torch.empty(4, device=dev), torch.empty(4, device=dev)
    one = torch.ones(4, device=dev)
    fiona.policy_loss(h, z, y, one, one, loss, logps, torch.empty_like(z))
    a = torch.tensor([1.0, -1.0, 2.0, -2.0], device=dev)
    dz = torch.empty_like(z)
    fiona.policy_loss(h, z, y, logps.clone(), a, loss, logps, dz, clip_low=0.0, clip_high=0.0, weights=one)
    got = dz[torch.arange(4), y.long()].cpu()
    assert torch.allclose(got, -a.cpu() * (1 - 1 / 50), rtol=1e-5)


def _spaced(t, dev, gap, shift):
    n, d = t.shape
    store = torch.full((n * (d + gap) + shift + 8,), 7.0, dtype=t.dtype, device=dev)
    rows = store.as_strided((n, d), (d + gap, 1), shift)
    rows.copy_(t)
    return store, rows


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("V", [3, 64, 1373, 40000])
def test_strides_and_alignments(V, dtype):
    dev = _dev()
    for make, run, check in ((lambda: _pairs([2, 3], V, dtype, seed=V), "preference_loss", _check_prefer),
                             (lambda: _tokens(6, V, dtype, seed=V), "policy_loss", _check_policy)):
        c = make()
        n = len(c["targets"])
        t = {k: v.to(dev) for k, v in c.items()}
        z = _spaced(c["logits"], dev, 3, 1)[1]
        store, dz = _spaced(c["logits"], dev, 5, 3)
        h = fiona.TokenLoss(dtype, V, n, 1)
        if run == "preference_loss":
            loss, logps = torch.empty(1, device=dev), torch.empty(2, device=dev)
            fiona.preference_loss(h, z, t["targets"], t["offsets"], t["reference"], loss, logps, dz, weights=t["weights"])
        else:
            loss, logps = torch.empty(n, device=dev), torch.empty(n, device=dev)
            fiona.policy_loss(h, z, t["targets"], t["old"], t["advantages"], loss, logps, dz, reference=t["reference"], kl=0.05,
                              weights=t["weights"])
        check(c, (loss, logps, dz))
        dz.fill_(7.0)
        assert bool((store == 7).all())                 # nothing beside the rows is written


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1000, 140001])
def test_in_place(V, dtype):
    dev = _dev()
    c = _pairs([3, 4], V, dtype, seed=12)
    want = _prefer(c, dev)
    t = {k: v.to(dev) for k, v in c.items()}
    loss, logps = torch.empty(1, device=dev), torch.empty(2, device=dev)
    fiona.preference_loss(fiona.TokenLoss(dtype, V, 20, 1), t["logits"], t["targets"], t["offsets"], t["reference"], loss, logps,
                          t["logits"], weights=t["weights"])
    assert torch.equal(t["logits"], want[2]) and torch.equal(loss, want[0])
    c = _tokens(7, V, dtype, seed=13)
    want = _policy(c, dev)
    t = {k: v.to(dev) for k, v in c.items()}
    loss, logps = torch.empty(7, device=dev), torch.empty(7, device=dev)
    fiona.policy_loss(fiona.TokenLoss(dtype, V, 20), t["logits"], t["targets"], t["old"], t["advantages"], loss, logps, t["logits"],
                      reference=t["reference"], kl=0.05, weights=t["weights"])
    assert torch.equal(t["logits"], want[2]) and torch.equal(loss, want[0])


@pytest.mark.parametrize("n,V,dtype", [(346, 50021, BF16), (132, 131071, F16), (1870, 9001, F16), (121, 140001, BF16), (1040, 8193, F32),
                                       (2040, 8229, BF16), (135, 199999, F16), (262, 125001, BF16)])
def test_long_rows_from_their_lines(n, V, dtype):
    """Logits of over 32 MiB whose rows start at every place of a line of memory; their gradients at others, and in place."""
    dev = _dev()
    half = (n - 3) // 2
    for c, name, check in ((_pairs([half, n - 3 - half], V, dtype, seed=V), "preference_loss", _check_prefer),
                           (_tokens(n, V, dtype, seed=V), "policy_loss", _check_policy)):
        t = {k: v.to(dev) for k, v in c.items()}
        h = fiona.TokenLoss(dtype, V, n, 1)

        def run(z, dz):
            if name == "preference_loss":
                loss, logps = torch.empty(1, device=dev), torch.empty(2, device=dev)
                fiona.preference_loss(h, z, t["targets"], t["offsets"], t["reference"], loss, logps, dz, weights=t["weights"])
            else:
                loss, logps = torch.empty(n, device=dev), torch.empty(n, device=dev)
                fiona.policy_loss(h, z, t["targets"], t["old"], t["advantages"], loss, logps, dz, reference=t["reference"], kl=0.05,
                                  weights=t["weights"])
            return loss, logps, dz

        gap = 4 if V % 2 else 3                          # (odd strides)
        z_store, z = _spaced(c["logits"], dev, gap, 1)
        store, dz = _spaced(c["logits"], dev, gap + 2, 3)
        got = run(z, dz)
        check(c, got)
        again = run(z, z)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        dz.fill_(7.0), z.fill_(7.0)
        assert bool((store == 7).all()) and bool((z_store == 7).all())


def test_gradients_against_differences():
    """The sum of the losses, in 64 bits, at both ends of a small step of the logits."""
    dev = _dev()
    g = torch.Generator().manual_seed(14)
    c = _pairs([3, 5, 2, 4], 40, F32, seed=15, masked=0.0)
    way = torch.randn(c["logits"].shape, generator=g, dtype=torch.float64)
    ends = [_loss64(c, s * 1e-5 * way) for s in (1, -1)]
    have = float((_prefer(c, dev, smoothing=0.1)[2].cpu().double() * way).sum())
    assert abs((ends[0] - ends[1]) / 2e-5 - have) <= 1e-6
    c = _tokens(9, 40, F32, seed=16, masked=0.0)
    way = torch.randn(c["logits"].shape, generator=g, dtype=torch.float64)
    ends = [_policy64(c, s * 1e-5 * way) for s in (1, -1)]
    have = float((_policy(c, dev)[2].cpu().double() * way).sum())
    assert abs((ends[0] - ends[1]) / 2e-5 - have) <= 1e-5


def _loss64(c, change):
    lp = torch.log_softmax(c["logits"].double() + change, 1).gather(1, c["targets"].long()[:, None])[:, 0]
    e = c["offsets"].tolist()
    L = torch.stack([lp[a:b].sum() for a, b in zip(e, e[1:])]) - c["reference"].double()
    h = 0.1 * (L[0::2] - L[1::2])
    s = torch.nn.functional.logsigmoid
    return float((-c["weights"].double() * (0.9 * s(h) + 0.1 * s(-h))).sum())


def _policy64(c, change):
    lp = torch.log_softmax(c["logits"].double() + change, 1).gather(1, c["targets"].long()[:, None])[:, 0]
    a, r, d = c["advantages"].double(), (lp - c["old"].double()).exp(), c["reference"].double() - lp
    loss = -torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.05 * (d.exp() - d - 1)
    return float((c["weights"].double() * loss).sum())


@pytest.mark.parametrize("V,lengths", [(2000, [30, 40, 20, 10]), (60000, [3, 2, 2, 3])])
def test_same_bits_twice_other_stream_and_graph_replay(V, lengths):
    dev = _dev()
    c = _pairs(lengths, V, BF16, seed=17)
    q = _tokens(len(c["targets"]), V, BF16, seed=18)
    n = len(c["targets"])
    t, u = ({k: v.to(dev) for k, v in x.items()} for x in (c, q))
    h = fiona.TokenLoss(BF16, V, n, 2)
    outs = (torch.empty(2, device=dev), torch.empty(4, device=dev), torch.empty_like(t["logits"]),
            torch.empty(n, device=dev), torch.empty(n, device=dev), torch.empty_like(t["logits"]))

    def call():
        fiona.preference_loss(h, t["logits"], t["targets"], t["offsets"], t["reference"], *outs[:3], weights=t["weights"])
        fiona.policy_loss(h, u["logits"], u["targets"], u["old"], u["advantages"], *outs[3:], reference=u["reference"], kl=0.05,
                          weights=u["weights"])

    call()
    torch.cuda.synchronize()
    _check_prefer(c, outs[:3])
    _check_policy(q, outs[3:])
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
    t["targets"].copy_(t["targets"].flip(0))            # the captured call follows its inputs
    c["targets"] = c["targets"].flip(0)
    c["logits"], t["logits"][:] = c["logits"].flip(0), t["logits"].flip(0)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    _check_prefer(c, outs[:3])


def test_a_larger_call_then_a_smaller_one_on_a_handle():
    dev = _dev()
    h = fiona.TokenLoss(F16, 5000, 400, 5)
    for lengths, seed in (([100, 90, 80, 70], 19), ([2, 3], 20)):
        c = _pairs(lengths, 5000, F16, seed=seed)
        _check_prefer(c, _prefer(c, dev, handle=h))
    c = _tokens(3, 5000, F16, seed=21)
    _check_policy(c, _policy(c, dev, handle=h))


def test_refusals():
    dev = _dev()
    for desc, status in [((BF16, 0, 8, 1), -1), ((BF16, 8, 0, 1), -1), ((BF16, (1 << 21) + 1, 8, 1), -3), ((BF16, 8, (1 << 21) + 1, 1), -3)]:
        with pytest.raises(fiona.FionaError) as e:
            fiona.TokenLoss(*desc)
        assert e.value.status == status, desc
    c, q = _pairs([2, 3], 64, BF16, seed=22), _tokens(8, 64, BF16, seed=23)
    t, u = ({k: v.to(dev) for k, v in x.items()} for x in (c, q))
    h = fiona.TokenLoss(BF16, 64, 8, 1)
    f = lambda k: torch.empty(k, device=dev)

    def prefer(tl=h, **over):
        a = dict(t, loss=f(1), logps=f(2), dlogits=torch.empty_like(t["logits"]))
        a.update(over)
        fiona.preference_loss(tl, **a)

    def policy(tl=h, **over):
        a = dict(u, loss=f(8), logps=f(8), dlogits=torch.empty_like(u["logits"]))
        a.update(over)
        fiona.policy_loss(tl, **a)

    def status(call, **over):
        with pytest.raises(fiona.FionaError) as e:
            call(**over)
        return e.value.status

    assert status(prefer, beta=0.0) == -1 and status(prefer, beta=float("inf")) == -1 and status(prefer, label_smoothing=1.0) == -1
    assert status(prefer, tl=fiona.TokenLoss(BF16, 64, 7, 1)) == -1 and status(prefer, tl=fiona.TokenLoss(BF16, 64, 8)) == -1
    assert status(policy, kl=0.1, reference=None) == -1 and status(policy, clip_low=1.5) == -1 and status(policy, clip_high=-0.1) == -1
    assert status(policy, kl=-1.0) == -1 and status(policy, tl=fiona.TokenLoss(BF16, 64, 7)) == -1
    assert status(policy, loss=u["old"]) == -5
    same = f(8)
    assert status(policy, loss=same, logps=same) == -5
    both = torch.zeros(9, 64, dtype=BF16, device=dev)
    assert status(policy, logits=both[:8], dlogits=both[1:]) == -5 and status(prefer, logits=both[:8], dlogits=both[1:]) == -5
    assert status(policy, dlogits=both[:1].expand(8, 64)) == -5
    for bad in (dict(targets=u["targets"].long()), dict(logits=u["logits"][:, :63]), dict(old=u["old"][:7]), dict(loss=f(8).double()),
                dict(dlogits=torch.empty(8, 128, dtype=BF16, device=dev)[:, ::2])):
        with pytest.raises(ValueError):
            policy(**bad)
    for bad in (dict(offsets=t["offsets"][:2]), dict(reference=t["reference"][:1]), dict(logps=f(3))):
        with pytest.raises(ValueError):
            prefer(**bad)
