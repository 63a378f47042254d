"""Private decoding, one attention layer: the projection runs on ciphertexts, the rest at the key holder.

Eight sequences decode together.  Every step the key holder encrypts the hidden rows (toy CKKS), the server evaluates
the fused query / key / value projection on the ciphertexts (fiona_hybrid_linear: diagonals as plaintexts, and one
ternary group of diagonals with a common scale), and the key holder decrypts the rows, adds its private adapters
(fiona_adapter_linear), rotates and appends keys and values to its paged cache (fiona_kv_append) and attends
(fiona_paged_attention).  The attention's rows are the next step's hidden rows.  Everything is followed in float64
without encryption; the program prints how far the two are apart.

    python examples/private_decode.py

Diagonal packing: slot 64 t + s of a ciphertext belongs to sequence t, and input ciphertext i holds
x_t[(s + i) mod 32] there, so that sum_i W[s][(s + i) mod 32] x_t[(s + i) mod 32] is row s of W x_t.
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

N, L = 1024, 2                                   # ring and limbs: 512 slots
SEQ, HIDDEN, HEADS, KV, D = 8, 32, 4, 2, 8       # sequences, width, query and key heads, head size
ROWS = (HEADS + 2 * KV) * D                      # rows of the fused projection: 64
RAW = 24                                         # diagonals as plaintexts; the other eight are one ternary group
PAGE, ADAPTERS, RANK = 4, 3, 4
DELTA_W = float(1 << ckks_toy.DELTA_W_BITS)


class Server:
    """The projection's weights and its plan; sees ciphertexts only."""

    def __init__(self, toy, W_raw, signs, scale, dev):
        ctx = fiona.Ctx(N, L, toy.moduli)
        s, i = np.arange(512) % 64, np.arange(RAW)[:, None]
        pts = np.stack([toy.encode_weight(W_raw[s, (s + j[0]) % HIDDEN]) for j in i])
        u32 = lambda a: np.asarray(a, dtype=np.uint32)
        self.plan = fiona.Plan(ctx, HIDDEN, 1, RAW, 1, u32([0, RAW]), u32(range(RAW)), u32(range(RAW)), u32([0, 1]),
                               u32([0, len(signs)]), u32(range(RAW, HIDDEN)), signs, u32([0]))
        to = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a).view(dt)).to(dev)
        self.pt, self.signs = to(pts.reshape(-1), np.int64), to(signs, np.int8)
        self.scale = to(np.array([scale], np.uint64), np.int64)
        self.out = torch.empty(2 * L * N, dtype=torch.int64, device=dev)

    def project(self, cts):
        fiona.hybrid_linear(self.plan, cts, self.pt, self.signs, self.scale, self.out)
        return self.out


class KeyHolder:
    """The secret key, the private adapters and the cache."""

    def __init__(self, toy, steps, A, B, scaling, ids, cos, sin, dev):
        self.toy, self.dev, self.step_at = toy, dev, 0
        t = lambda a, dt: torch.tensor(a, dtype=dt, device=dev)
        self.A, self.B, self.scaling, self.ids = t(A, torch.float32), t(B, torch.float32), t(scaling, torch.float32), t(ids, torch.int32)
        self.cos, self.sin = t(cos, torch.float32), t(sin, torch.float32)
        pages = -(-steps // PAGE)
        self.table = torch.randperm(SEQ * pages, device=dev).to(torch.int32).view(SEQ, pages)
        self.k_cache = torch.zeros(SEQ * pages, PAGE, KV, D, device=dev)
        self.v_cache = torch.zeros_like(self.k_cache)
        self.adapters = fiona.Adapters(torch.float32, ADAPTERS, RANK, HIDDEN, ROWS, SEQ, forward_only=True)
        self.attention = fiona.Attention(torch.float32, HEADS, KV, D, PAGE, SEQ, steps)

    def encrypt(self, x):
        s = np.arange(512)
        cts = np.stack([self.toy.encrypt(x[s // 64, (s % 64 + i) % HIDDEN]) for i in range(HIDDEN)])
        return torch.from_numpy(cts.view(np.int64).reshape(-1)).to(self.dev)

    def decode(self, x, ct):
        """The attention's rows [SEQ][HIDDEN] for hidden rows x and the encrypted projection ct of them."""
        ct = ct.cpu().numpy().view(np.uint64).reshape(2, L, N)
        rows = torch.tensor(self.toy.decrypt(ct).real.reshape(SEQ, ROWS), dtype=torch.float32, device=self.dev)
        hidden = torch.tensor(x, dtype=torch.float32, device=self.dev)
        fiona.adapter_linear(self.adapters, hidden, self.ids, self.A, self.B, rows, rows, scaling=self.scaling)
        qkv = rows.view(SEQ, HEADS + 2 * KV, D)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
        at = self.step_at
        slots = self.table[:, at // PAGE].long() * PAGE + at % PAGE
        positions = torch.full((SEQ,), at, dtype=torch.int32, device=self.dev)
        fiona.kv_append(k, v, slots, self.k_cache, self.v_cache, positions=positions, cos=self.cos, sin=self.sin, q=q, q_out=q)
        out = torch.empty(SEQ, HEADS, D, device=self.dev)
        lengths = torch.full((SEQ,), at + 1, dtype=torch.int32, device=self.dev)
        fiona.paged_attention(self.attention, q, self.k_cache, self.v_cache, self.table, lengths, out)
        self.step_at += 1
        return out.reshape(SEQ, HIDDEN).double().cpu().numpy()


class Plain:
    """The same layer in float64, without encryption."""

    def __init__(self, W, A, B, scaling, ids, cos, sin):
        self.W, self.A, self.B, self.scaling, self.ids, self.cos, self.sin = W, A, B, scaling, ids, cos, sin
        self.k, self.v = [], []

    def _turn(self, x, at):
        a, b = x[..., :D // 2], x[..., D // 2:]
        c, s = self.cos[at], self.sin[at]
        return np.concatenate((a * c - b * s, a * s + b * c), -1)

    def decode(self, x):
        rows = x @ self.W.T
        for t, a in enumerate(self.ids):
            if a >= 0:
                rows[t] += self.scaling[a] * (self.B[a] @ (self.A[a] @ x[t]))
        qkv = rows.reshape(SEQ, HEADS + 2 * KV, D)
        at = len(self.k)
        q = self._turn(qkv[:, :HEADS], at)
        self.k.append(self._turn(qkv[:, HEADS:HEADS + KV], at))
        self.v.append(qkv[:, HEADS + KV:])
        k, v = np.stack(self.k, 1), np.stack(self.v, 1)              # [SEQ][keys][KV][D]
        out = np.empty((SEQ, HEADS, D))
        for h in range(HEADS):
            s = np.einsum("td,tnd->tn", q[:, h], k[:, :, h * KV // HEADS]) * D ** -0.5
            p = np.exp(s - s.max(1, keepdims=True))
            out[:, h] = np.einsum("tn,tnd->td", p / p.sum(1, keepdims=True), v[:, :, h * KV // HEADS])
        return out.reshape(SEQ, HIDDEN)


def run(steps=5, seed=3):
    """The largest difference from the float64 layer, relative to its largest value, over all steps."""
    dev = torch.device("cuda:0")
    rng = np.random.default_rng(seed)
    toy = ckks_toy.ToyCKKS(N, synth.ntt_primes(N, L), seed=seed)
    W_raw = rng.normal(0, HIDDEN ** -0.5, (ROWS, HIDDEN))
    signs = rng.integers(-1, 2, HIDDEN - RAW).astype(np.int8)
    scale = int(rng.integers(1 << 17, 1 << 18))
    W = np.zeros((ROWS, HIDDEN))
    s = np.arange(ROWS)
    for i in range(HIDDEN):
        W[s, (s + i) % HIDDEN] = W_raw[s, (s + i) % HIDDEN] if i < RAW else scale / DELTA_W * signs[i - RAW]
    A, B = rng.normal(0, HIDDEN ** -0.5, (ADAPTERS, RANK, HIDDEN)), rng.normal(0, 0.3, (ADAPTERS, ROWS, RANK))
    scaling, ids = rng.uniform(0.5, 1.5, ADAPTERS), [0, 2, -1, 1, 0, 1, -1, 2]
    angle = np.arange(steps)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    cos, sin = np.cos(angle), np.sin(angle)
    server = Server(toy, W_raw, signs, scale, dev)
    holder = KeyHolder(toy, steps, A, B, scaling, ids, cos, sin, dev)
    plain = Plain(W, A, B, scaling, ids, cos, sin)
    x = y = rng.uniform(-1, 1, (SEQ, HIDDEN))
    worst = 0.0
    for step in range(steps):
        x = holder.decode(x, server.project(holder.encrypt(x)))
        y = plain.decode(y)
        worst = max(worst, float(np.abs(x - y).max() / np.abs(y).max()))
        print("step %d: largest value %.3f, off by %.2e of it" % (step, np.abs(y).max(), np.abs(x - y).max() / np.abs(y).max()),
              flush=True)
    return worst


if __name__ == "__main__":
    if not torch.cuda.is_available():
        sys.exit("needs a GPU")
    run()
