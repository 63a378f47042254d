"""Performance cases of the key holder's operators: what runs on decrypted rows between two encrypted projections.

A case is one call of kv_append, paged_attention, adapter_linear or adapter_backward, with everything a user's program
holds before it already made: the rows, the paged cache and its table, the adapters, the handles and the output buffers.
`run` computes it in plain torch (`own` false: elementary operations in 32 bits, rounded once) or with the library's
calls; `exact` gives the results in 64 bits, sequence by sequence and adapter by adapter.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ----------------------------------------------------------------------------
# The cases
# ----------------------------------------------------------------------------

def _append(name, n_tok, n_head, n_kv, d, rot, page, src, dst, interleaved=False, skip=0):
    return dict(name=name, op="append", n_tok=n_tok, n_head=n_head, n_kv=n_kv, d=d, rot=rot, page=page, src=src,
                dst=dst, interleaved=interleaved, skip=skip)


def _attend(name, n_seq, shortest, longest, n_head, n_kv, d, page, dtype, window=0, softcap=0.0, empty=0):
    return dict(name=name, op="attend", n_seq=n_seq, shortest=shortest, longest=longest, n_head=n_head, n_kv=n_kv, d=d,
                page=page, dtype=dtype, window=window, softcap=softcap, empty=empty)


def _adapt(name, op, n_tok, n_adapter, rank, d_in, d_out, dtype, runs, plain=0):
    """runs: the tokens come as that many requests, each a run of tokens with one adapter; plain: runs without one."""
    return dict(name=name, op=op, n_tok=n_tok, n_adapter=n_adapter, rank=rank, d_in=d_in, d_out=d_out, dtype=dtype,
                runs=runs, plain=plain)


def listed():
    return [
        # One decode step of eight sequences at the 768-wide projection (12 heads of 64), decrypted rows in 32 bits.
        _append("append_step", 8, 12, 12, 64, 64, 16, "f32", "bf16"),
        # A prompt at the 4096-wide projection, 32 query heads on 8 key heads.
        _append("append_prompt", 16384, 32, 8, 128, 128, 64, "bf16", "bf16"),
        # Ragged: odd counts, part of each head rotated in interleaved pairs, padding tokens that are not written.
        _append("append_odd", 1531, 15, 5, 80, 48, 24, "f32", "f16", True, 31),
        # One sequence's first tokens, 12 heads of 64: the smallest step, all latency.
        _attend("attend_one", 1, 300, 300, 12, 12, 64, 16, "f32"),
        # A serving batch of ragged lengths, 32 query heads on 8 key heads.
        _attend("attend_batch", 64, 100, 8192, 32, 8, 128, 16, "bf16"),
        # Two long documents: few rows over a long axis.
        _attend("attend_long", 2, 100000, 131072, 32, 8, 128, 64, "bf16"),
        # Odd groups and head size, pages of 24, a sliding window, capped scores, idle slots of length zero.
        _attend("attend_odd", 19, 37, 6000, 35, 7, 80, 24, "f16", 3000, 30.0, 2),
        # One token for each of sixteen requests, an adapter each, beside the 768-wide projection.
        _adapt("adapter_step", "adapt", 16, 16, 8, 768, 768, "bf16", 16),
        # A batch of prompts beside the 4096-wide projection.
        _adapt("adapter_prompt", "adapt", 8192, 8, 16, 4096, 4096, "bf16", 12, 1),
        # Mixed: prompts and single tokens together, odd widths and rank, some without an adapter.
        _adapt("adapter_mixed", "adapt", 613, 23, 20, 1000, 1373, "f32", 61, 5),
        # A training step beside the 768-wide projection, and one beside the 4096-wide one.
        _adapt("train_small", "train", 2048, 4, 8, 768, 768, "f32", 16),
        _adapt("train_large", "train", 8192, 4, 64, 4096, 4096, "bf16", 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attend", "attend", "adapt", "train"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op in ("append", "attend"):
            n_kv = rng.choice([1, 2, 4, 5, 8, 12])
            n_head = n_kv * rng.choice([1, 1, 2, 4, 5, 8])
            d = rng.choice([64, 64, 80, 96, 128, 128])
            page = rng.choice([8, 16, 24, 32, 64, 128])
        if op == "append":
            dst = dtype if rng.random() < 0.5 else rng.choice(["bf16", "f16", "f32"])
            n_tok = _log_int(rng, 1, 16384)
            c = _append("", n_tok, n_head, n_kv, d, rng.choice([d, d, d // 2, 0]), page, dtype, dst,
                        rng.random() < 0.3, rng.choice([0, 0, n_tok // 10]))
        elif op == "attend":
            longest = _log_int(rng, 1, 131072)
            n_seq = _log_int(rng, 1, 128)
            c = _attend("", n_seq, _log_int(rng, 1, longest), longest, n_head, n_kv, d, page, dtype,
                        rng.choice([0, 0, 0, _log_int(rng, 64, 8192)]), rng.choice([0.0, 0.0, 0.0, 20.0]),
                        rng.choice([0, 0, n_seq // 8]))
            padded = n_seq * longest * n_kv * d
            if padded > 1.1e9:
                continue
        else:
            n_tok = _log_int(rng, 1, 8192)
            n_adapter = _log_int(rng, 1, 64 if op == "adapt" else 8)
            width = lambda: rng.choice([768, 768, 1000, 1373, 2048, 4096, 4096])
            c = _adapt("", op, n_tok, n_adapter, rng.choice([4, 8, 16, 16, 20, 32, 64]), width(), width(), dtype,
                       min(n_tok, _log_int(rng, 1, 64 if op == "adapt" else 16)), rng.choice([0, 0, 1]))
        del c["name"]
        if work(c)["bytes"] <= 0.9e9:
            return c


def _lengths(c):
    """The sequences' lengths: spread over their range (over its logarithm), in a fixed shuffled order."""
    n, lo, hi = c["n_seq"], c["shortest"], c["longest"]
    out = [hi if n == 1 else int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    r = random.Random(n * 1000003 + hi)
    r.shuffle(out)
    for i in r.sample(range(n), c["empty"]):
        out[i] = 0
    return out


def _ids(c):
    """The adapter of each token: the requests' runs of uneven lengths, -1 for the runs without one."""
    n, runs = c["n_tok"], c["runs"]
    r = random.Random(n * 1000003 + runs)
    cuts = sorted(r.sample(range(1, n), runs - 1))
    which = [i % c["n_adapter"] for i in range(runs)]
    r.shuffle(which)
    for i in r.sample(range(runs), min(c["plain"], runs)):
        which[i] = -1
    out = []
    for i, (a, b) in enumerate(zip([0] + cuts, cuts + [n])):
        out += [which[i]] * (b - a)
    return out


def _size(name):
    return 4 if name == "f32" else 2


def work(c):
    """What the inputs and outputs hold, each read or written once, and the products of the definition."""
    if c["op"] == "append":
        heads = c["n_head"] + 2 * c["n_kv"]
        live = c["n_tok"] - c["skip"]
        row = c["d"] * (c["n_head"] * c["n_tok"] + 2 * c["n_kv"] * live)
        table = c["n_tok"] * c["rot"] * 4.0 + c["n_tok"] * 16.0
        return {"bytes": row * (_size(c["src"]) + _size(c["dst"])) + table, "flops": 3.0 * c["n_tok"] * heads * c["rot"]}
    if c["op"] == "attend":
        seen = float(sum(min(n, c["window"]) if c["window"] else n for n in _lengths(c)))
        rows = c["n_seq"] * c["n_head"]
        e = _size(c["dtype"])
        return {"bytes": 2 * seen * c["n_kv"] * c["d"] * e + 2 * rows * c["d"] * e + 4.0 * rows + 4 * seen / c["page"],
                "flops": 4 * seen * c["n_head"] * c["d"]}
    ids, e = _ids(c), _size(c["dtype"])
    live, used = sum(i >= 0 for i in ids), len({i for i in ids if i >= 0})
    if c["op"] == "adapt":
        elems = c["n_tok"] * 2 * c["d_out"] + live * c["d_in"] + used * c["rank"] * (c["d_in"] + c["d_out"])
        return {"bytes": float(elems * e + 4 * c["n_tok"]), "flops": 2.0 * live * c["rank"] * (c["d_in"] + c["d_out"])}
    elems = c["n_tok"] * 2 * c["d_in"] + live * (c["d_in"] + c["d_out"]) \
        + (used + c["n_adapter"]) * c["rank"] * (c["d_in"] + c["d_out"])
    return {"bytes": float(elems * e + 4 * c["n_tok"]),
            "flops": 2.0 * live * c["rank"] * (2 * c["d_out"] + 3 * c["d_in"])}


# ----------------------------------------------------------------------------
# Inputs, from the case and the seed alone
# ----------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": dict(case)}
    {"append": _prepare_append, "attend": _prepare_attend, "adapt": _prepare_adapt, "train": _prepare_adapt}[case["op"]](
        case, s, g)
    return s


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=g)


def _prepare_append(c, s, g):
    n, H, KV, d, page = c["n_tok"], c["n_head"], c["n_kv"], c["d"], c["page"]
    pages = n // page + 5
    # The rows of one fused projection: queries, keys and values side by side.
    rows = _randn(g, n, H + 2 * KV, d, dtype=TYPES[c["src"]])
    s["q"], s["k"], s["v"] = rows[:, :H], rows[:, H:H + KV], rows[:, H + KV:]
    s["k_cache"] = _randn(g, pages, page, KV, d, dtype=TYPES[c["dst"]])
    s["v_cache"] = _randn(g, pages, page, KV, d, dtype=TYPES[c["dst"]])
    s["q_out"] = torch.empty(n, H, d, dtype=TYPES[c["dst"]], device="cuda")
    # Consecutive tokens fill pages that lie anywhere; single tokens go to pages of their own sequences.
    order = torch.randperm(pages, generator=g, device="cuda")
    at = torch.arange(n, device="cuda") + 3
    slots = order[at // page] * page + at % page
    if c["skip"]:
        slots[torch.randperm(n, generator=g, device="cuda")[:c["skip"]]] = -1
    s["slots"] = slots
    s["positions"] = (torch.arange(n, device="cuda") % 4096 + 5).to(torch.int32)
    s["cos"] = s["sin"] = None
    if c["rot"]:
        p = torch.arange(4096 + 8, dtype=torch.float64, device="cuda")
        f = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
        s["cos"], s["sin"] = (p[:, None] * f).cos().float(), (p[:, None] * f).sin().float()


def _prepare_attend(c, s, g):
    n_seq, H, KV, d, page = c["n_seq"], c["n_head"], c["n_kv"], c["d"], c["page"]
    dt = TYPES[c["dtype"]]
    lengths = _lengths(c)
    held = [-(-n // page) for n in lengths]
    pages = sum(held) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((n_seq, max(1, -(-c["longest"] // page))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = order[at:at + h]
        at += h
    s["page_table"] = table
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["k_cache"] = _randn(g, pages, page, KV, d, dtype=dt)
    s["v_cache"] = _randn(g, pages, page, KV, d, dtype=dt)
    s["q"] = _randn(g, n_seq, H, d, dtype=dt, scale=2.0)
    s["scale"] = d ** -0.5
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(n_seq, H, dtype=torch.float32, device="cuda")
    if own:
        import paper_2609_35352_amd as fiona
        s["handle"] = fiona.Attention(dt, H, KV, d, page, n_seq, c["longest"])


def _prepare_adapt(c, s, g):
    n, nA, R, d_in, d_out = c["n_tok"], c["n_adapter"], c["rank"], c["d_in"], c["d_out"]
    dt = TYPES[c["dtype"]]
    s["ids"] = torch.tensor(_ids(c), dtype=torch.int32, device="cuda")
    s["x"] = _randn(g, n, d_in, dtype=dt)
    s["A"] = _randn(g, nA, R, d_in, dtype=dt, scale=d_in ** -0.5)
    s["B"] = _randn(g, nA, d_out, R, dtype=dt, scale=0.5)
    # Adapters of several ranks share one table of the largest; some have half of it.
    s["ranks"] = torch.tensor([R if i % 3 != 1 else (R + 1) // 2 for i in range(nA)], dtype=torch.int32, device="cuda")
    s["scaling"] = torch.rand(nA, generator=g, device="cuda") + 0.5
    if c["op"] == "adapt":
        s["base"] = _randn(g, n, d_out, dtype=dt)
        s["y"] = torch.empty_like(s["base"])
    else:
        s["dy"] = _randn(g, n, d_out, dtype=dt)
        s["dx_base"] = _randn(g, n, d_in, dtype=dt)
        s["dx"] = torch.empty_like(s["dx_base"])
        s["dA"], s["dB"] = torch.empty_like(s["A"]), torch.empty_like(s["B"])
    if own:
        import paper_2609_35352_amd as fiona
        s["handle"] = fiona.Adapters(dt, nA, R, d_in, d_out, n)


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    return {"append": _plain_append, "attend": _plain_attend, "adapt": _plain_adapt, "train": _plain_train}[op](s)


def _run_own(s, op):
    import paper_2609_35352_amd as fiona
    if op == "append":
        fiona.kv_append(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"], positions=s["positions"], cos=s["cos"],
                        sin=s["sin"], interleaved=s["case"]["interleaved"], q=s["q"], q_out=s["q_out"])
        return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"]}
    if op == "attend":
        fiona.paged_attention(s["handle"], s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["lengths"], s["out"],
                              scale=s["scale"], window=s["case"]["window"], softcap=s["case"]["softcap"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "adapt":
        fiona.adapter_linear(s["handle"], s["x"], s["ids"], s["A"], s["B"], s["base"], s["y"], ranks=s["ranks"],
                             scaling=s["scaling"])
        return {"y": s["y"]}
    fiona.adapter_backward(s["handle"], s["x"], s["ids"], s["A"], s["B"], s["dy"], s["dx_base"], s["dx"], s["dA"],
                           s["dB"], ranks=s["ranks"], scaling=s["scaling"])
    return {"dx": s["dx"], "dA": s["dA"], "dB": s["dB"]}


def _rotated(x, cos, sin, interleaved):
    if cos is None:
        return x
    h = cos.shape[-1]
    c, s, r = cos[:, None], sin[:, None], x[..., :2 * h]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :h], r[..., h:])
    u, v = a * c - b * s, a * s + b * c
    turned = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((turned, x[..., 2 * h:]), -1)


def _plain_append(s):
    c = s["case"]
    dst = TYPES[c["dst"]]
    cos = sin = None
    if c["rot"]:
        at = s["positions"].long()
        cos, sin = s["cos"][at], s["sin"][at]
    q = _rotated(s["q"].float(), cos, sin, c["interleaved"]).to(dst)
    k = _rotated(s["k"].float(), cos, sin, c["interleaved"]).to(dst)
    v = s["v"].float().to(dst)
    slots = s["slots"]
    if c["skip"]:
        keep = (slots >= 0).nonzero()[:, 0]
        slots, k, v = slots[keep], k[keep], v[keep]
    s["k_cache"].flatten(0, 1)[slots] = k
    s["v_cache"].flatten(0, 1)[slots] = v
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"]}


def _plain_attend(s):
    c = s["case"]
    n_seq, H, KV, d = c["n_seq"], c["n_head"], c["n_kv"], c["d"]
    table = s["page_table"].clamp(min=0).long()
    k = s["k_cache"][table].flatten(1, 2).permute(0, 2, 3, 1).float().contiguous()   # [n_seq, KV, d, keys]
    v = s["v_cache"][table].flatten(1, 2).permute(0, 2, 1, 3).float().contiguous()   # [n_seq, KV, keys, d]
    q = s["q"].float().view(n_seq, KV, H // KV, d) * s["scale"]
    score = torch.matmul(q, k)
    if c["softcap"]:
        score = c["softcap"] * torch.tanh(score / c["softcap"])
    at, n = torch.arange(score.shape[-1], device="cuda"), s["lengths"].long()[:, None]
    seen = at < n
    if c["window"]:
        seen = seen & (at >= n - c["window"])
    score = torch.where(seen[:, None, None], score, -math.inf)
    m = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = m + torch.log(total)
    return {"out": out.view(n_seq, H, d).to(TYPES[c["dtype"]]), "lse": lse.view(n_seq, H)}


def _scaled_mask(s):
    """[n_tok][n_adapter][rank]: the token's adapter's scaling within its rank, 0 elsewhere."""
    nA, R = s["A"].shape[:2]
    mine = s["ids"][:, None] == torch.arange(nA, device="cuda")
    inside = torch.arange(R, device="cuda") < s["ranks"][:, None]
    return torch.where(mine[:, :, None] & inside, s["scaling"][:, None], 0.0).flatten(1)


def _plain_adapt(s):
    A, B = s["A"].float().flatten(0, 1), s["B"].float().transpose(1, 2).flatten(0, 1)   # [nA R, d_in], [nA R, d_out]
    h = torch.matmul(s["x"].float(), A.t()) * _scaled_mask(s)
    return {"y": (s["base"].float() + torch.matmul(h, B)).to(s["y"].dtype)}


def _plain_train(s):
    nA, R, d_in = s["A"].shape
    dt = s["dx"].dtype
    A, B = s["A"].float().flatten(0, 1), s["B"].float().transpose(1, 2).flatten(0, 1)
    x, dy, mask = s["x"].float(), s["dy"].float(), _scaled_mask(s)
    h = torch.matmul(x, A.t()) * mask
    g = torch.matmul(dy, B.t()) * mask
    dx = s["dx_base"].float() + torch.matmul(g, A)
    dA = torch.matmul(g.t(), x).view(nA, R, d_in)
    dB = torch.matmul(dy.t(), h).view(-1, nA, R).transpose(0, 1).contiguous()
    return {"dx": dx.to(dt), "dA": dA.to(dt), "dB": dB.to(dt)}


# ----------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "adapt": _exact_adapt, "train": _exact_train}[case["op"]](
        case, s)


def _exact_append(c, s):
    def turn(x):
        y = x.double().clone()
        at = s["positions"].long()
        for i in range(c["rot"] // 2):
            lo, hi = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rot"] // 2)
            co, si = s["cos"][at, i].double()[:, None], s["sin"][at, i].double()[:, None]
            a, b = x[..., lo].double(), x[..., hi].double()
            y[..., lo] = a * co - b * si
            y[..., hi] = b * co + a * si
        return y

    out = {"q": turn(s["q"])}
    live = (s["slots"] >= 0).nonzero()[:, 0]
    for name, rows in (("k", turn(s["k"])), ("v", s["v"].double())):
        cache = s[name + "_cache"].double()
        cache[s["slots"][live] // c["page"], s["slots"][live] % c["page"]] = rows[live]
        out[name] = cache
    return out


def _exact_attend(c, s):
    H, KV, d, page = c["n_head"], c["n_kv"], c["d"], c["page"]
    out = torch.zeros(c["n_seq"], H, d, dtype=torch.float64, device="cuda")
    lse = torch.full((c["n_seq"], H), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lengths"].tolist()):
        first = max(0, n - c["window"]) if c["window"] else 0
        if n == first:
            continue
        j = torch.arange(first, n, device="cuda")
        p, r = s["page_table"][i, j // page].long(), j % page
        for h in range(KV):
            k, v = s["k_cache"][p, r, h].double(), s["v_cache"][p, r, h].double()
            group = slice(h * (H // KV), (h + 1) * (H // KV))
            z = s["q"][i, group].double() @ k.t().contiguous() * s["scale"]
            if c["softcap"]:
                z = torch.tanh(z / c["softcap"]) * c["softcap"]
            lse[i, group] = torch.logsumexp(z, -1)
            out[i, group] = torch.softmax(z, -1) @ v
    return {"out": out, "lse": lse}


def _exact_adapt(c, s):
    y = s["base"].double()
    for a in range(c["n_adapter"]):
        t, r = (s["ids"] == a).nonzero()[:, 0], int(s["ranks"][a])
        h = s["x"][t].double() @ s["A"][a, :r].double().t().contiguous()
        y[t] += s["scaling"][a].double() * (h @ s["B"][a, :, :r].double().t().contiguous())
    return {"y": y}


def _exact_train(c, s):
    dx = s["dx_base"].double()
    dA, dB = torch.zeros_like(s["A"], dtype=torch.float64), torch.zeros_like(s["B"], dtype=torch.float64)
    for a in range(c["n_adapter"]):
        t, r = (s["ids"] == a).nonzero()[:, 0], int(s["ranks"][a])
        A, B = s["A"][a, :r].double(), s["B"][a, :, :r].double()
        x, dy, k = s["x"][t].double(), s["dy"][t].double(), s["scaling"][a].double()
        g = k * (dy @ B)
        dx[t] += g @ A
        dA[a, :r] = g.t().contiguous() @ x
        dB[a, :, :r] = k * (dy.t().contiguous() @ (x @ A.t().contiguous()))
    return {"dx": dx, "dA": dA, "dB": dB}
