"""Logits with an offset common to a row: log-probabilities, losses and gradients are as near the 64-bit ones as without it."""
import pytest

torch = pytest.importorskip("torch")
import test_gpu_token_loss as tl  # noqa: E402
import training_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16, E = torch.float32, torch.float16, torch.bfloat16, ref.E


def _scores(logits, targets):
    """ref.scores with bounds that the offset does not enter.

    With a row's maximum m and sum s of exp(z - m), l = (z_y - m) - log s and p = exp((z - m) - log s).  Differences from m
    are at most |l| (log s is not negative) and are rounded once, by E of themselves; the sum's relative error (its terms'
    exponentials, arguments and additions, as in ref.scores) is an error of its logarithm; the hardware's logarithm is within
    2^-21 of itself, with two more roundings of it."""
    l, _, lp, _, live, at = wide(logits, targets)
    z = torch.where(live[:, None], logits.double(), 0.0)
    m = z.amax(1, keepdim=True)
    p = lp.exp()
    away = torch.where(p > 0, (z - m).abs(), 0.0)
    log_s = (torch.logsumexp(z - m, 1, keepdim=True)).abs()
    rel = (p * (2.0 ** -21 + 4 * E * away)).sum(1, keepdim=True) + ref._deep(z.shape[1]) * E
    dlog = rel + (2.0 ** -21 + 4 * E) * log_s
    dl = torch.where(live, dlog[:, 0] + 2 * E * l.abs(), 0.0)
    return l, dl, lp, dlog + 2.0 ** -21 + 4 * E * torch.where(p > 0, lp.abs(), 0.0), live, at


wide = ref.scores


@pytest.fixture
def near(monkeypatch):
    monkeypatch.setattr(ref, "scores", _scores)


# (f16: steps of 8 at 1e4; bf16: of 2 at 300, of 128 at -3e4, where most of a row is one value)
OFFSETS = [(F32, 0.0), (F32, 1000.0), (F32, 3e4), (F32, -2e5), (F16, 1e4), (BF16, 300.0), (BF16, -3e4)]


def _shifted(c, offset):
    """The rows' logits moved and rounded; what is compared with log-probabilities moves along with them."""
    y = c["targets"]
    before = wide(torch.nan_to_num(c["logits"]), y)[0]
    c["logits"] = (c["logits"].float() + offset).to(c["logits"].dtype)
    moved = wide(torch.nan_to_num(c["logits"]), y)[0] - before
    if "old" in c:
        for k in ("old", "reference"):
            c[k] = (c[k].double() + moved).float()
    else:
        ends = c["offsets"].tolist()
        c["reference"] = (c["reference"].double() + torch.stack([moved[a:b].sum() for a, b in zip(ends, ends[1:])])).float()
    return c


@pytest.mark.parametrize("dtype,offset", OFFSETS)
@pytest.mark.parametrize("lengths,V", [([5, 0, 1, 9], 3), ([3, 2, 7, 1], 100), ([12, 7, 3, 30], 2049), ([3, 2, 4, 1], 50021)])
def test_preference(lengths, V, dtype, offset, near):
    dev = tl._dev()
    c = _shifted(tl._pairs(lengths, V, dtype, seed=V), offset)
    tl._check_prefer(c, tl._prefer(c, dev, smoothing=0.1), smoothing=0.1)
    tl._check_prefer(c, tl._prefer(c, dev, gradient=False))


# Parts of rows, and whole ones in registers, in LDS as well, and partly read again.
@pytest.mark.parametrize("dtype,offset", OFFSETS)
@pytest.mark.parametrize("n,V", [(5, 3), (33, 100), (40, 2049), (5, 50021), (300, 2000), (300, 20000), (40, 28000)])
def test_policy(n, V, dtype, offset, near):
    dev = tl._dev()
    c = _shifted(tl._tokens(n, V, dtype, seed=n + V, masked=0.1), offset)
    tl._check_policy(c, tl._policy(c, dev))
    tl._check_policy(c, tl._policy(c, dev, gradient=False, kl=0.0), kl=0.0)


@pytest.mark.parametrize("n,V,dtype", [(260, 40000, F32), (60, 60000, F32), (130, 90000, F32), (258, 130000, BF16)])
def test_policy_of_long_rows(n, V, dtype, near):
    dev = tl._dev()
    c = _shifted(tl._tokens(n, V, dtype, seed=n + V, masked=0.1), 3e4)
    tl._check_policy(c, tl._policy(c, dev))


def test_long_rows_from_their_lines(near):
    dev = tl._dev()
    n, V = 172, 50021
    c = _shifted(tl._pairs([60, 109], V, F32, seed=V), 3e4)
    tl._check_prefer(c, tl._prefer(c, dev))
    c = _shifted(tl._tokens(n, V, F32, seed=V, masked=0.1), 3e4)
    tl._check_policy(c, tl._policy(c, dev))


def test_infinite_logits_are_as_they_were(near):
    """Rows cut down to one element or a few, and rows of -inf alone (no number)."""
    dev = tl._dev()
    c = tl._tokens(4, 3000, F32, seed=7, masked=0.0)
    z, y = c["logits"], c["targets"]
    z[0, :] = float("-inf")
    z[0, int(y[0])] = 3e4
    z[1, 5:2000] = float("-inf")
    z[1, int(y[1])] = 1.0
    l = wide(z, y)[0]
    c["old"], c["reference"] = (l - 0.1).float(), (l + 0.3).float()
    tl._check_policy(c, tl._policy(c, dev))
    z[2, :] = float("-inf")
    for got in tl._policy(c, dev):
        assert bool(torch.isnan(got[2]).all()) and bool(torch.isfinite(got[[0, 1, 3]]).all())
