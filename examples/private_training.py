"""Private training, one layer: the projection runs on ciphertexts, everything that is trained stays at the key holder.

Two pairs of short answers train the key holder's adapter and norm on a preference.  A step normalises the hidden rows
(fiona_layer_norm), encrypts them, lets the server evaluate its projection to the logits on the ciphertexts
(fiona_hybrid_linear), decrypts, adds the adapter (fiona_adapter_linear) and takes the loss and its gradient
(fiona_preference_loss).  The gradient goes back through the server's transposed projection, again on ciphertexts, and
through the adapter (fiona_adapter_backward) and the norm (fiona_layer_norm_backward), and one optimiser step
(fiona_adamw_step) takes all four tensors on.  Every step's gradients are followed in float64 without encryption from the
same parameters; the program prints how far the two are apart.

    python examples/private_training.py

Diagonal packing: slot 64 t + s of a ciphertext belongs to token t, and input ciphertext i holds x_t[(s + i) mod d]
there, so that sum_i W[s][(s + i) mod d] x_t[(s + i) mod d] is row s of W x_t.
"""
from __future__ import annotations

import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np
import torch

import paper_2609_35352_amd as fiona
import synth
from oracle import ckks_toy

N, L = 1024, 2                       # ring and limbs: 512 slots
TOKENS, HIDDEN, VOCAB, RANK = 8, 32, 64, 4
OFFSETS = [0, 2, 4, 7, 8]            # two pairs: sequences of 2 and 2, 3 and 1 tokens
BETA, LR, EPS = 2.0, 1e-2, 1e-5


class Projection:
    """One matrix [up to 64][d] as the server holds it: plaintexts of its diagonals; sees ciphertexts only."""

    def __init__(self, toy, W, dev):
        rows, self.d = W.shape
        s, i = np.arange(512) % 64, np.arange(self.d)[:, None]
        value = lambda j: np.where(s < rows, W[np.minimum(s, rows - 1), (s + j) % self.d], 0.0)
        pts = np.stack([toy.encode_weight(value(j[0])) for j in i])
        u32 = lambda a: np.asarray(a, dtype=np.uint32)
        ctx = fiona.Ctx(N, L, toy.moduli)
        self.plan = fiona.Plan(ctx, self.d, 1, self.d, 0, u32([0, self.d]), u32(range(self.d)), u32(range(self.d)), u32([0, 0]),
                               u32([0]), u32([]), np.zeros(0, np.int8), u32([]))
        to = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a).view(dt)).to(dev)
        self.pt = to(pts.reshape(-1), np.int64)
        self.signs, self.scales = torch.zeros(1, dtype=torch.int8, device=dev), torch.zeros(1, dtype=torch.int64, device=dev)
        self.out = torch.empty(2 * L * N, dtype=torch.int64, device=dev)

    def apply(self, cts):
        fiona.hybrid_linear(self.plan, cts, self.pt, self.signs, self.scales, self.out)
        return self.out


class KeyHolder:
    """The secret key, the norm, the adapter and their optimiser."""

    def __init__(self, toy, forward, backward, hidden, targets, A, B, dev):
        self.toy, self.dev, self.forward, self.backward = toy, dev, forward, backward
        t = lambda a, dt=torch.float32: torch.tensor(a, dtype=dt, device=dev)
        self.hidden, self.targets, self.offsets = t(hidden), t(targets, torch.int32), t(OFFSETS, torch.int32)
        self.ids, self.reference = t([0] * TOKENS, torch.int32), None
        zeros = lambda *s: torch.zeros(*s, device=dev)
        self.params = {"weight": torch.ones(HIDDEN, device=dev), "bias": zeros(HIDDEN), "A": t(A)[None], "B": t(B)[None]}
        self.grads = {k: torch.empty_like(p) for k, p in self.params.items()}
        p, g = list(self.params.values()), list(self.grads.values())
        self.m, self.v = [torch.zeros_like(x) for x in p], [torch.zeros_like(x) for x in p]
        self.adapters = fiona.Adapters(torch.float32, 1, RANK, HIDDEN, VOCAB, TOKENS)
        self.norm = fiona.LayerNorm(torch.float32, HIDDEN, TOKENS)
        self.loss_of = fiona.TokenLoss(torch.float32, VOCAB, TOKENS, 2)
        self.optimiser = fiona.AdamW(p, g, self.m, self.v, weight_decay=[0.0, 0.0, 0.01, 0.01])
        self.steps, self.lr, self.at = torch.arange(1, 1001, dtype=torch.int32, device=dev), t([LR]), 0

    def through(self, projection, x):
        """The server's projection of rows x, encrypted on the way: scaled to one, as the toy's errors are absolute."""
        size = float(x.abs().max())
        rows, s = x.double().cpu().numpy() / size, np.arange(512)
        cts = np.stack([self.toy.encrypt(rows[s // 64, (s % 64 + i) % projection.d]) for i in range(projection.d)])
        ct = projection.apply(torch.from_numpy(cts.view(np.int64).reshape(-1)).to(self.dev))
        out = self.toy.decrypt(ct.cpu().numpy().view(np.uint64).reshape(2, L, N)).real.reshape(TOKENS, 64)
        return torch.tensor(out * size, dtype=torch.float32, device=self.dev)

    def step(self):
        """One step; returns the loss (its gradients stay in `grads`)."""
        p, g, dev = self.params, self.grads, self.dev
        rows = torch.empty_like(self.hidden)
        mean, rstd = torch.empty(TOKENS, device=dev), torch.empty(TOKENS, device=dev)
        fiona.layer_norm(self.hidden, p["weight"], p["bias"], rows, eps=EPS, mean=mean, rstd=rstd)
        logits = self.through(self.forward, rows)
        fiona.adapter_linear(self.adapters, rows, self.ids, p["A"], p["B"], logits, logits)
        loss, logps = torch.empty(2, device=dev), torch.empty(4, device=dev)
        if self.reference is None:       # what the adapter starts from is the reference
            fiona.preference_loss(self.loss_of, logits, self.targets, self.offsets, torch.zeros(4, device=dev), loss, logps)
            self.reference = logps.clone()
        fiona.preference_loss(self.loss_of, logits, self.targets, self.offsets, self.reference, loss, logps, logits, beta=BETA)
        past = self.through(self.backward, logits)[:, :HIDDEN].contiguous()
        fiona.adapter_backward(self.adapters, rows, self.ids, p["A"], p["B"], logits, past, past, g["A"], g["B"])
        fiona.layer_norm_backward(self.norm, past, self.hidden, p["weight"], mean, rstd, None, past, g["weight"], g["bias"])
        fiona.adamw_step(self.optimiser, self.lr, self.steps[self.at:self.at + 1])
        self.at += 1
        return float(loss.sum())


def plain_gradients(params, hidden, targets, W, reference):
    """The loss and its gradients in float64, without encryption."""
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in params.items()}
    x = torch.tensor(hidden, dtype=torch.float64)
    c = x - x.mean(1, keepdim=True)
    rows = c / (c.square().mean(1, keepdim=True) + EPS).sqrt() * p["weight"] + p["bias"]
    logits = rows @ torch.tensor(W).t() + rows @ p["A"][0].t() @ p["B"][0].t()
    logp = torch.log_softmax(logits, 1)[torch.arange(TOKENS), torch.tensor(targets)]
    sums = torch.stack([logp[a:b].sum() for a, b in zip(OFFSETS, OFFSETS[1:])])
    ratio = sums - reference.double().cpu()
    loss = -torch.nn.functional.logsigmoid(BETA * (ratio[0::2] - ratio[1::2])).mean()
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in p.items()}


def run(steps=4, seed=5):
    """The largest differences of the gradients (relative to each gradient's largest value) and of the loss over all steps."""
    dev = torch.device("cuda:0")
    rng = np.random.default_rng(seed)
    toy = ckks_toy.ToyCKKS(N, synth.ntt_primes(N, L), seed=seed)
    W = rng.normal(0, HIDDEN ** -0.5, (VOCAB, HIDDEN))
    hidden, targets = rng.normal(0.2, 1.0, (TOKENS, HIDDEN)), rng.integers(0, VOCAB, TOKENS)
    A, B = rng.normal(0, HIDDEN ** -0.5, (RANK, HIDDEN)), rng.normal(0, 0.1, (VOCAB, RANK))
    holder = KeyHolder(toy, Projection(toy, W, dev), Projection(toy, W.T.copy(), dev), hidden, targets, A, B, dev)
    worst, off = 0.0, 0.0
    for step in range(steps):
        before = {k: v.clone() for k, v in holder.params.items()}
        loss = holder.step()
        want, grads = plain_gradients(before, hidden, targets, W, holder.reference)
        apart = {k: float((holder.grads[k].double().cpu() - g).abs().max() / g.abs().max()) for k, g in grads.items()}
        worst, off = max(worst, *apart.values()), max(off, abs(loss - want))
        print("step %d: loss %.5f, off by %.1e; gradients off by %s of the largest" % (
            step, loss, abs(loss - want), ", ".join("%.1e (%s)" % (v, k) for k, v in apart.items())), flush=True)
    return worst, off


if __name__ == "__main__":
    if not torch.cuda.is_available():
        sys.exit("needs a GPU")
    run()
