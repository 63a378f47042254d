"""Python binding of the MI355X hybrid weighted sum (include/fiona.h).

Argument marshalling only: every step of the computation runs in the HIP
kernels of ``libfiona.so``.  PyTorch supplies device memory and streams.  If
the library has not been built, importing works but every call raises.

    ctx  = Ctx(N, L, moduli)
    plan = Plan.from_layer(ctx, layer)          # or Plan(ctx, n_in=..., ...)
    hybrid_linear(plan, in_t, pt_t, sign_t, scale_t, out_t)

Tensors are device tensors of 8-byte elements (uint64 residues, stored in any
8-byte dtype) for in/pt/scale/out and int8 for the signs, laid out as the
header describes: in [n_in][2][L][N], pt n_pt rows of [L][N] at the plan's
pitch (default L*N), out [n_out][2][L][N].
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
import types

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfiona.so")

FIONA_PLAN_NO_SHARING = 1
FIONA_PLAN_HOST_ONLY = 2
FIONA_PLAN_NO_LDS_SUMS = 4
FIONA_PLAN_NO_PARTIAL_SHARING = 8
FIONA_PLAN_PER_CONTRIBUTION = 16
FIONA_PLAN_NO_OUTPUT_BURSTS = 32
FIONA_PLAN_CHECK_INPUTS = 64

FIONA_ERR_ARG = -1
FIONA_ERR_PRECONDITION = -9
FIONA_ERR_BOUNDS = -10

STATUS = {0: "FIONA_OK", -1: "FIONA_ERR_ARG", -2: "FIONA_ERR_PLAN", -3: "FIONA_ERR_UNSUPPORTED",
          -4: "FIONA_ERR_ALIGN", -5: "FIONA_ERR_ALIAS", -6: "FIONA_ERR_HIP", -7: "FIONA_ERR_NOMEM",
          -8: "FIONA_ERR_NODEVICE", -9: "FIONA_ERR_PRECONDITION", -10: "FIONA_ERR_BOUNDS"}


class FionaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, STATUS.get(status, "unknown"), status))


class _LayerDesc(ctypes.Structure):
    _fields_ = [("n_in", ctypes.c_uint32), ("n_out", ctypes.c_uint32), ("n_pt", ctypes.c_uint32),
                ("n_scale", ctypes.c_uint32),
                ("pm_off", ctypes.c_void_p), ("pm_input", ctypes.c_void_p), ("pm_pt", ctypes.c_void_p),
                ("grp_off", ctypes.c_void_p), ("grp_mem_off", ctypes.c_void_p),
                ("mem_input", ctypes.c_void_p), ("mem_sign", ctypes.c_void_p), ("grp_scale", ctypes.c_void_p),
                ("flags", ctypes.c_uint32), ("pt_pitch", ctypes.c_uint64)]


class _Stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in (
        "ct_terms", "n_pmult", "n_member", "n_member_nonzero", "n_use", "n_sum_distinct", "n_sum_resident",
        "pmult_per_contribution", "pmult_grouped", "addsub_unshared", "addsub_shared", "addsub_partial")] + \
        [(n, ctypes.c_uint32) for n in ("tile", "waves", "lds_bytes", "grid", "split_outputs", "segment_slots",
                                        "n_partial", "partial_levels", "output_rounds",
                                        "output_buffer_rows", "input_passes")]


_lib = None
_first_use = threading.RLock()


def lib():
    """The loaded HIP library; raises if it has not been built."""
    if _lib is None:
        _load()
    return _lib


def _load():
    global _lib
    with _first_use:
        if _lib is not None:
            return
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libfiona.so is not built (run __graft_entry__.build()); "
                               "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        L.fiona_ctx_create.restype = ctypes.c_int
        L.fiona_ctx_create.argtypes = [ctypes.c_uint32, ctypes.c_uint32, ctypes.c_void_p,
                                       ctypes.POINTER(ctypes.c_void_p)]
        L.fiona_ctx_destroy.restype = None
        L.fiona_ctx_destroy.argtypes = [ctypes.c_void_p]
        L.fiona_plan_create.restype = ctypes.c_int
        L.fiona_plan_create.argtypes = [ctypes.c_void_p, ctypes.POINTER(_LayerDesc),
                                        ctypes.POINTER(ctypes.c_void_p)]
        L.fiona_plan_destroy.restype = None
        L.fiona_plan_destroy.argtypes = [ctypes.c_void_p]
        L.fiona_plan_stats.restype = ctypes.c_int
        L.fiona_plan_stats.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Stats)]
        L.fiona_hybrid_linear.restype = ctypes.c_int
        L.fiona_hybrid_linear.argtypes = [ctypes.c_void_p] * 7
        L.fiona_pt_pitch_hint.restype = ctypes.c_uint64
        L.fiona_pt_pitch_hint.argtypes = [ctypes.c_void_p]
        L.fiona_status_string.restype = ctypes.c_char_p
        L.fiona_status_string.argtypes = [ctypes.c_int]
        _lib = L


def _check(rc: int, where: str):
    if rc != 0:
        raise FionaError(rc, where)


class Ctx:
    """RNS parameters: N coefficients, L limbs with moduli q_l < 2^50."""

    def __init__(self, N: int, L: int, moduli):
        self.N, self.L = int(N), int(L)
        self.moduli = [int(q) for q in moduli]
        arr = (ctypes.c_uint64 * len(self.moduli))(*self.moduli)
        h = ctypes.c_void_p()
        _check(lib().fiona_ctx_create(self.N, self.L, ctypes.cast(arr, ctypes.c_void_p), ctypes.byref(h)),
               "fiona_ctx_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def pt_pitch_hint(self) -> int:
        """fiona_pt_pitch_hint: a padded plaintext pitch (words) for this context."""
        return int(lib().fiona_pt_pitch_hint(self._h))

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().fiona_ctx_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _u32(a):
    return np.ascontiguousarray(a, dtype=np.uint32)


class Plan:
    """A compiled layer (fiona_plan_create)."""

    def __init__(self, ctx: Ctx, n_in, n_out, n_pt, n_scale, pm_off, pm_input, pm_pt, grp_off, grp_mem_off,
                 mem_input, mem_sign, grp_scale, flags: int = 0, pt_pitch: int = 0):
        self.ctx = ctx
        keep = [_u32(pm_off), _u32(pm_input), _u32(pm_pt), _u32(grp_off), _u32(grp_mem_off),
                _u32(mem_input), np.ascontiguousarray(mem_sign, dtype=np.int8), _u32(grp_scale)]

        def ptr(a):
            return a.ctypes.data if a.size else None

        d = _LayerDesc(int(n_in), int(n_out), int(n_pt), int(n_scale), *[ptr(a) for a in keep], int(flags),
                       int(pt_pitch))
        h = ctypes.c_void_p()
        _check(lib().fiona_plan_create(ctx.handle, ctypes.byref(d), ctypes.byref(h)), "fiona_plan_create")
        self._h = h
        self.n_in, self.n_out, self.n_pt, self.n_scale = int(n_in), int(n_out), int(n_pt), int(n_scale)
        self.n_member = int(keep[4][-1]) if keep[4].size else 0
        self.pt_pitch = int(pt_pitch) if pt_pitch else ctx.L * ctx.N

    @classmethod
    def from_layer(cls, ctx: Ctx, layer, flags: int = 0, pt_pitch: int = 0) -> "Plan":
        return cls(ctx, layer.n_in, layer.n_out, layer.n_pt, len(layer.scales), layer.pm_off, layer.pm_input,
                   layer.pm_pt, layer.grp_off, layer.grp_mem_off, layer.mem_input, layer.mem_sign,
                   layer.grp_scale, flags, pt_pitch)

    def pt_words(self) -> int:
        """Words the plaintext table spans under this plan's pitch."""
        return (self.n_pt - 1) * self.pt_pitch + self.ctx.L * self.ctx.N if self.n_pt else 0

    @property
    def handle(self):
        return self._h

    def stats(self) -> dict:
        s = _Stats()
        _check(lib().fiona_plan_stats(self._h, ctypes.byref(s)), "fiona_plan_stats")
        return {n: int(getattr(s, n)) for n, _ in _Stats._fields_}

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().fiona_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _dptr(t, name, elem_size):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.element_size() != elem_size:
        raise ValueError("%s must have %d-byte elements" % (name, elem_size))
    return t.data_ptr()


def _call_ptrs(plan: Plan, in_t, pt_t, sign_t, scale_t, out_t):
    """The device pointers of one call, after checking the tensors' sizes."""
    N, L = plan.ctx.N, plan.ctx.L
    sizes = [(in_t, "in_cts", plan.n_in * 2 * L * N), (pt_t, "pt_diags", plan.pt_words()),
             (out_t, "out_cts", plan.n_out * 2 * L * N), (sign_t, "ternary_groups", plan.n_member),
             (scale_t, "scales", plan.n_scale)]
    for t, name, n in sizes:
        if t is not None and t.numel() < n:
            raise ValueError("%s has %d elements, needs %d" % (name, t.numel(), n))
    return (_dptr(in_t, "in_cts", 8), _dptr(pt_t, "pt_diags", 8), _dptr(sign_t, "ternary_groups", 1),
            _dptr(scale_t, "scales", 8), _dptr(out_t, "out_cts", 8))


def hybrid_linear(plan: Plan, in_t, pt_t, sign_t, scale_t, out_t, stream=None) -> None:
    """fiona_hybrid_linear on torch device tensors (queued on ``stream``, default: current)."""
    _check(lib().fiona_hybrid_linear(plan.handle, *_call_ptrs(plan, in_t, pt_t, sign_t, scale_t, out_t),
                                     _stream_handle(stream)), "fiona_hybrid_linear")


class Rescaler:
    """NTT tables and workspace for the rescale epilogue (fiona_rescaler_create)."""

    def __init__(self, ctx: Ctx, max_ct: int, psi=None):
        L = lib()
        L.fiona_rescaler_create.restype = ctypes.c_int
        L.fiona_rescaler_create.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint32,
                                            ctypes.POINTER(ctypes.c_void_p)]
        L.fiona_rescaler_destroy.restype = None
        L.fiona_rescaler_destroy.argtypes = [ctypes.c_void_p]
        L.fiona_rescale.restype = ctypes.c_int
        L.fiona_rescale.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint32, ctypes.c_void_p,
                                    ctypes.c_void_p]
        self.ctx = ctx
        self.max_ct = int(max_ct)
        roots = None
        if psi is not None:
            roots = (ctypes.c_uint64 * ctx.L)(*[int(p) for p in psi])
        h = ctypes.c_void_p()
        _check(L.fiona_rescaler_create(ctx.handle, ctypes.cast(roots, ctypes.c_void_p) if roots else None,
                                       self.max_ct, ctypes.byref(h)), "fiona_rescaler_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().fiona_rescaler_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rescale(rescaler: Rescaler, in_t, n_ct: int, out_t, stream=None) -> None:
    """fiona_rescale on torch device tensors: in [n_ct][2][L][N] -> out [n_ct][2][L-1][N]."""
    import torch

    N, L = rescaler.ctx.N, rescaler.ctx.L
    if in_t.numel() < n_ct * 2 * L * N or out_t.numel() < n_ct * 2 * (L - 1) * N:
        raise ValueError("tensors too small for %d ciphertexts" % n_ct)
    if stream is None:
        stream = torch.cuda.current_stream()
    s = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    _check(lib().fiona_rescale(rescaler.handle, _dptr(in_t, "in_cts", 8), int(n_ct), _dptr(out_t, "out_cts", 8), s),
           "fiona_rescale")


class Rotator:
    """NTT tables of the data moduli and the special prime, and the workspace of
    the hoisted rotations (fiona_rotator_create)."""

    def __init__(self, ctx: Ctx, special_prime: int, max_rot: int, psi=None):
        L = lib()
        L.fiona_rotator_create.restype = ctypes.c_int
        L.fiona_rotator_create.argtypes = [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_uint32,
                                           ctypes.POINTER(ctypes.c_void_p)]
        L.fiona_rotator_destroy.restype = None
        L.fiona_rotator_destroy.argtypes = [ctypes.c_void_p]
        L.fiona_rotation_key_words.restype = ctypes.c_uint64
        L.fiona_rotation_key_words.argtypes = [ctypes.c_void_p]
        L.fiona_rotation_key_layout.restype = ctypes.c_int
        L.fiona_rotation_key_layout.argtypes = [ctypes.c_void_p, ctypes.c_uint32, ctypes.c_void_p, ctypes.c_void_p,
                                                ctypes.c_void_p]
        L.fiona_hoisted_rotate.restype = ctypes.c_int
        L.fiona_hoisted_rotate.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint32, ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        self.ctx = ctx
        self.P = int(special_prime)
        self.max_rot = int(max_rot)
        roots = None
        if psi is not None:
            roots = (ctypes.c_uint64 * (ctx.L + 1))(*[int(p) for p in psi])
        h = ctypes.c_void_p()
        _check(L.fiona_rotator_create(ctx.handle, self.P, ctypes.cast(roots, ctypes.c_void_p) if roots else None,
                                      self.max_rot, ctypes.byref(h)), "fiona_rotator_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def key_words(self) -> int:
        """Words of one rotation key: L * 2 * (L + 1) * N."""
        return int(lib().fiona_rotation_key_words(self._h))

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().fiona_rotator_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _stream_handle(stream):
    import torch

    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def rotation_key_layout(rotator: Rotator, galois: int, key_t, out_t, stream=None) -> None:
    """fiona_rotation_key_layout: a key [L][2][L+1][N] in natural NTT order -> the library's layout."""
    n = rotator.key_words()
    if key_t.numel() < n or out_t.numel() < n:
        raise ValueError("key tensors need %d words" % n)
    _check(lib().fiona_rotation_key_layout(rotator.handle, int(galois), _dptr(key_t, "key", 8),
                                           _dptr(out_t, "key_out", 8), _stream_handle(stream)),
           "fiona_rotation_key_layout")


def hoisted_rotate(rotator: Rotator, ct_t, galois, keys_t, out_t, stream=None) -> None:
    """fiona_hoisted_rotate: ct [2][L][N] -> out [len(galois)][2][L][N], keys [len(galois)] in the library layout."""
    N, L = rotator.ctx.N, rotator.ctx.L
    n_rot = len(galois)
    if ct_t.numel() < 2 * L * N or out_t.numel() < n_rot * 2 * L * N or keys_t.numel() < n_rot * rotator.key_words():
        raise ValueError("tensors too small for %d rotations" % n_rot)
    g = (ctypes.c_uint32 * max(1, n_rot))(*[int(x) for x in galois])
    _check(lib().fiona_hoisted_rotate(rotator.handle, _dptr(ct_t, "ct", 8), n_rot, ctypes.cast(g, ctypes.c_void_p),
                                      _dptr(keys_t, "keys", 8), _dptr(out_t, "out_cts", 8), _stream_handle(stream)),
           "fiona_hoisted_rotate")


def mac_microbench(blocks: int, chunks: int, sink_t, stream=None) -> int:
    """fiona_mac_microbench: the register-only raw-route arithmetic over
    blocks * 256 threads; returns the plaintext words it multiplies."""
    L = lib()
    L.fiona_mac_microbench.restype = ctypes.c_int
    L.fiona_mac_microbench.argtypes = [ctypes.c_uint32, ctypes.c_uint32, ctypes.c_void_p, ctypes.c_void_p]
    L.fiona_mac_microbench_words.restype = ctypes.c_uint64
    L.fiona_mac_microbench_words.argtypes = [ctypes.c_uint32, ctypes.c_uint32]
    if sink_t.numel() < blocks * 256:
        raise ValueError("sink holds fewer than blocks * 256 words")
    _check(L.fiona_mac_microbench(int(blocks), int(chunks), _dptr(sink_t, "sink", 8), _stream_handle(stream)),
           "fiona_mac_microbench")
    return int(L.fiona_mac_microbench_words(int(blocks), int(chunks)))


def check_ntt_offsets(op: str, N: int, L: int, moduli, capacity: int, n_call: int, out_shrink: int = 0):
    """fiona_check_ntt_offsets: host replay of every memory access of one
    rescale (op "rescale", L moduli) or one rotation call (op "rotate", L data
    moduli then the special prime).  Returns (status, first violation or "")."""
    L_ = lib()
    L_.fiona_check_ntt_offsets.restype = ctypes.c_int
    L_.fiona_check_ntt_offsets.argtypes = [ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_void_p,
                                           ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_char_p,
                                           ctypes.c_size_t]
    mods = (ctypes.c_uint64 * len(moduli))(*[int(q) for q in moduli])
    msg = ctypes.create_string_buffer(512)
    rc = L_.fiona_check_ntt_offsets({"rescale": 0, "rotate": 1}[op], int(N), int(L), ctypes.cast(mods, ctypes.c_void_p),
                                    int(capacity), int(n_call), int(out_shrink), msg, 512)
    return rc, msg.value.decode()


def stream_read(src_t, blocks: int, sink_t, stream=None) -> int:
    """fiona_stream_read over all of src_t (8-byte elements, an even count);
    returns the bytes read."""
    L_ = lib()
    L_.fiona_stream_read.restype = ctypes.c_int
    L_.fiona_stream_read.argtypes = [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_void_p,
                                     ctypes.c_void_p]
    if sink_t.numel() < blocks:
        raise ValueError("sink holds fewer than blocks words")
    _check(L_.fiona_stream_read(_dptr(src_t, "src", 8), src_t.numel(), int(blocks), _dptr(sink_t, "sink", 8),
                                _stream_handle(stream)), "fiona_stream_read")
    return src_t.numel() * 8


def stream_copy(src_t, dst_t, blocks: int, stream=None) -> int:
    """fiona_stream_copy of all of src_t into dst_t; returns the bytes moved (read + written)."""
    L_ = lib()
    L_.fiona_stream_copy.restype = ctypes.c_int
    L_.fiona_stream_copy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32,
                                     ctypes.c_void_p]
    if dst_t.numel() < src_t.numel():
        raise ValueError("dst is smaller than src")
    _check(L_.fiona_stream_copy(_dptr(src_t, "src", 8), _dptr(dst_t, "dst", 8), src_t.numel(), int(blocks),
                                _stream_handle(stream)), "fiona_stream_copy")
    return 2 * src_t.numel() * 8


def stream_write(dst_t, blocks: int, stream=None) -> int:
    """fiona_stream_write over all of dst_t (8-byte elements, an even count);
    returns the bytes written."""
    L_ = lib()
    L_.fiona_stream_write.restype = ctypes.c_int
    L_.fiona_stream_write.argtypes = [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_void_p]
    _check(L_.fiona_stream_write(_dptr(dst_t, "dst", 8), dst_t.numel(), int(blocks), _stream_handle(stream)),
           "fiona_stream_write")
    return dst_t.numel() * 8


def plan_check_inputs(plan: Plan, signs, scales, x=None, pt=None) -> int:
    """fiona_plan_check_inputs on host arrays (NumPy): signs int8 [n_member],
    scales uint64 [n_scale], x uint64 [n_in][2][L][N] or None, pt uint64 rows at
    the plan's pitch or None.  Returns the status (0, FIONA_ERR_PRECONDITION, ...)."""
    L_ = lib()
    L_.fiona_plan_check_inputs.restype = ctypes.c_int
    L_.fiona_plan_check_inputs.argtypes = [ctypes.c_void_p] * 5
    keep = [np.ascontiguousarray(signs, dtype=np.int8), np.ascontiguousarray(scales, dtype=np.uint64)]
    keep += [None if a is None else np.ascontiguousarray(a, dtype=np.uint64) for a in (x, pt)]
    ptrs = [None if a is None or not a.size else a.ctypes.data for a in keep]
    return int(L_.fiona_plan_check_inputs(plan.handle, *ptrs))


def hybrid_linear_static(plan: Plan, in_t, pt_t, sign_t, scale_t, out_t, stream=None) -> None:
    """fiona_hybrid_linear_static: hybrid_linear with its word blocks in the
    library's static per-device array (allocates nothing)."""
    L_ = lib()
    L_.fiona_hybrid_linear_static.restype = ctypes.c_int
    L_.fiona_hybrid_linear_static.argtypes = [ctypes.c_void_p] * 7
    _check(L_.fiona_hybrid_linear_static(plan.handle, *_call_ptrs(plan, in_t, pt_t, sign_t, scale_t, out_t),
                                         _stream_handle(stream)), "fiona_hybrid_linear_static")


# ----------------------------------------------------------------------------
# The key holder's operators (include/fiona.h): attention over a paged cache and
# low-rank adapters on the decrypted rows between two encrypted projections.
#
#     kv_append(k, v, slots, k_cache, v_cache, positions=p, cos=c, sin=s, q=q, q_out=q_out)
#     att = Attention(dtype, n_head, n_kv, head_dim, page_size, max_seq, max_length)
#     paged_attention(att, q, k_cache, v_cache, page_table, lengths, out)
#     ad = Adapters(dtype, n_adapter, max_rank, d_in, d_out, max_tokens)
#     adapter_linear(ad, x, ids, A, B, base, y)
#     adapter_backward(ad, x, ids, A, B, dy, dx_base, dx, dA, dB)
#
# The training step around them: a norm between projections, losses on the logits with
# their gradients, and the optimiser.
#
#     layer_norm(x, weight, bias, y, residual=r, total=s, mean=mean, rstd=rstd)
#     ln = LayerNorm(dtype, width, max_rows)
#     layer_norm_backward(ln, dy, s, weight, mean, rstd, dx_base, dx, dweight, dbias)
#     tl = TokenLoss(dtype, vocab, max_tokens, max_pairs)
#     preference_loss(tl, logits, targets, offsets, reference, loss, logps, dlogits)
#     policy_loss(tl, logits, targets, old, advantages, loss, logps, dlogits)
#     opt = AdamW(params, grads, m, v)
#     adamw_step(opt, lr, step)
#
# Tensors are float32, float16 or bfloat16 tensors of the current device whose last
# axis is contiguous; the other axes may have any stride.  Nothing is recorded for
# autograd: tensors that require a gradient are refused in grad mode, tensors with a
# forward-mode tangent always, and what a call writes counts as modified in place.
# ----------------------------------------------------------------------------

# The header's structs, fields in order with native alignment; packed in one go, as a
# decode step's calls are as short as a few microseconds.
_KV_CACHE = struct.Struct("@5I2P6Q")
_APPEND_ARGS = struct.Struct("@6I4P8Q4P")
_ATTENTION_DESC = struct.Struct("@7I")
_ATTENTION_ARGS = struct.Struct("@3I2f3P5Q2P")
_ADAPTERS_DESC = struct.Struct("@7I")
_ADAPTER_ARGS = struct.Struct("@I6PQ2P2Q5P3Q")
_NORM_ARGS = struct.Struct("@4If8P4Q")
_NORM_DESC = struct.Struct("@4I")
_NORM_BACKWARD_ARGS = struct.Struct("@I9P4Q")
_TOKEN_LOSS_DESC = struct.Struct("@4I")
_PREFERENCE_ARGS = struct.Struct("@2I2f2P2Q6P")
_POLICY_ARGS = struct.Struct("@I3f2P2Q7P")
_ADAMW_TENSOR = struct.Struct("@7PQd")
_ADAMW_DESC = struct.Struct("@4I3dP")

_DTYPES = {}   # torch dtype -> fiona_type
_raw_stream, _device_now, _modified, _forward = [], [], [], []
_INT = {}      # bytes -> torch dtype, and "f32"


def _lm_lib():
    L = lib()
    if _DTYPES:
        return L
    with _first_use:
        import torch

        p = ctypes.c_void_p
        for name, args in (("fiona_kv_append", [p] * 3), ("fiona_attention_create", [p, ctypes.POINTER(p)]),
                           ("fiona_paged_attention", [p] * 4), ("fiona_adapters_create", [p, ctypes.POINTER(p)]),
                           ("fiona_adapter_linear", [p] * 3), ("fiona_adapter_backward", [p] * 3),
                           ("fiona_layer_norm", [p] * 2), ("fiona_norm_create", [p, ctypes.POINTER(p)]),
                           ("fiona_layer_norm_backward", [p] * 3), ("fiona_token_loss_create", [p, ctypes.POINTER(p)]),
                           ("fiona_preference_loss", [p] * 3), ("fiona_policy_loss", [p] * 3),
                           ("fiona_adamw_create", [p, ctypes.POINTER(p)]), ("fiona_adamw_step", [p] * 5)):
            getattr(L, name).restype, getattr(L, name).argtypes = ctypes.c_int, args
        for name in ("fiona_attention_destroy", "fiona_adapters_destroy", "fiona_norm_destroy", "fiona_token_loss_destroy",
                     "fiona_adamw_destroy"):
            getattr(L, name).restype, getattr(L, name).argtypes = None, [p]
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # (without the stream object: 2 us a call)
        _raw_stream.append(raw or (lambda dev: torch.cuda.current_stream(dev).cuda_stream))
        _modified.append(torch.autograd.graph.increment_version)   # (a tensor or several)
        fw = torch.autograd.forward_ad   # (without its level: every call asks)
        _forward.append(fw if hasattr(fw, "_current_level") else types.SimpleNamespace(_current_level=0, unpack_dual=fw.unpack_dual))
        _device_now.append(getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device)
        _INT.update({4: torch.int32, 8: torch.int64, "f32": torch.float32})
        _DTYPES.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})   # (last: who finds a type finds all else)
    return L


def _stream_of(stream, dev: int) -> int:
    """The stream's handle; by default the current stream of the tensors' device, which has to be the current one:
    that is where a launch goes, whatever its pointers are."""
    if _device_now[0]() != dev:
        raise ValueError("the tensors are on device %d, the current device is %d" % (dev, _device_now[0]()))
    if stream is None:
        return _raw_stream[0](dev)
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError("the stream is on device %d, the tensors are on device %d" % (stream.device_index, dev))
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _type_code(dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        _lm_lib()
        code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError("%s is not float32, float16 or bfloat16" % (dtype,))
    return code


def _no_tangents(arguments):
    """Refuses tensors that carry a forward-mode tangent, in grad mode and outside it: no call computes those of its results.
    (Asked for where a dual level is open; nothing carries one elsewhere.)"""
    import torch

    for name, t in arguments.items():
        if isinstance(t, torch.Tensor) and _forward[0].unpack_dual(t).tangent is not None:
            raise ValueError("%s carries a tangent, which this call does not follow (its primal or detach() where that is meant)" % name)


def _refuse(t, name, dtype, shape, dev, packed=False):
    """Raises for what is wrong with t; returns where nothing is, for a tensor with requires_grad outside grad mode."""
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.get_device() != dev:
        raise ValueError("%s is on device %d, not on %d" % (name, t.get_device(), dev))
    if t.dtype is not dtype:
        raise ValueError("%s must be %s, is %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, has %s" % (name, tuple(shape), tuple(t.shape)))
    if packed and not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if not packed and t.stride()[-1] != 1 and shape[-1] > 1:
        raise ValueError("%s: its last axis must be contiguous" % name)
    import torch

    if torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, which this call does not record (torch.no_grad() or detach() where that "
                         "is meant)" % name)


def _rows(t, name, dtype, shape, dev):
    """The strides of a tensor whose last axis is contiguous, after checking type, shape and device."""
    st = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or dev < 0 or (st[-1] != 1 and shape[-1] > 1) \
            or t.requires_grad:
        _refuse(t, name, dtype, shape, dev)
    return st


def _packed(t, name, dtype, shape, dev):
    """The address of a contiguous tensor, after the same checks."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or dev < 0 or not t.is_contiguous() \
            or t.requires_grad:
        _refuse(t, name, dtype, shape, dev, True)
    return t.data_ptr()


def _cache_desc(k_cache, v_cache):
    """(fiona_kv_cache, dtype, device, n_kv, head_dim)"""
    dtype, shape, dev = k_cache.dtype, k_cache.shape, k_cache.get_device()
    if len(shape) != 4:
        raise ValueError("k_cache must have shape [n_pages][page_size][n_kv][head_dim]")
    code = _type_code(dtype)
    ks, vs = _rows(k_cache, "k_cache", dtype, shape, dev), _rows(v_cache, "v_cache", dtype, shape, dev)
    return _KV_CACHE.pack(code, *shape, k_cache.data_ptr(), v_cache.data_ptr(), *ks[:3], *vs[:3]), dtype, dev, shape[2], \
        shape[3]


def kv_append(k, v, slots, k_cache, v_cache, positions=None, cos=None, sin=None, interleaved: bool = False, q=None,
              q_out=None, stream=None) -> None:
    """fiona_kv_append: k, v [n_tok][n_kv][d] into the caches [n_pages][page_size][n_kv][d] at slots (int64
    [n_tok]; outside the cache: not written), keys rotated at positions (int32 [n_tok]) with cos, sin float32
    [n_pos][rot_dim / 2], and q [n_tok][n_head][d] rotated into q_out (the caches' type)."""
    cache, dtype, dev, n_kv, d = _cache_desc(k_cache, v_cache)
    n, rows = k.shape[0], k.dtype
    code = _type_code(rows)
    ks, vs = _rows(k, "k", rows, (n, n_kv, d), dev), _rows(v, "v", rows, (n, n_kv, d), dev)
    at = _packed(slots, "slots", _INT[8], (n,), dev)
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    H, qp, qop, qs, qos = 0, 0, 0, (0, 0), (0, 0)
    if q is not None:
        H = q.shape[1]
        qs, qos = _rows(q, "q", rows, (n, H, d), dev), _rows(q_out, "q_out", dtype, (n, H, d), dev)
        qp, qop = q.data_ptr(), q_out.data_ptr()
    n_pos, rot, pp, cp, sp = 0, 0, 0, 0, 0
    if cos is not None or sin is not None:
        if cos is None or sin is None or positions is None:
            raise ValueError("positions, cos and sin go together")
        shape = cos.shape
        if len(shape) != 2:
            raise ValueError("cos must have shape [n_pos][rot_dim / 2]")
        n_pos, rot = shape[0], 2 * shape[1]
        f32 = _INT["f32"]
        cp, sp = _packed(cos, "cos", f32, shape, dev), _packed(sin, "sin", f32, shape, dev)
        pp = _packed(positions, "positions", _INT[4], (n,), dev)
    args = _APPEND_ARGS.pack(n, H, code, rot, n_pos, 1 if interleaved else 0, k.data_ptr(), v.data_ptr(), qp, qop,
                             ks[0], ks[1], vs[0], vs[1], qs[0], qs[1], qos[0], qos[1], at, pp, cp, sp)
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_kv_append(cache, args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_kv_append")
    _modified[0]((k_cache, v_cache) if q_out is None else (k_cache, v_cache, q_out))


class Attention:
    """The workspace of paged_attention (fiona_attention_create)."""

    def __init__(self, dtype, n_head: int, n_kv: int, head_dim: int, page_size: int, max_seq: int, max_length: int):
        self.dtype = dtype
        self.n_head, self.n_kv, self.head_dim, self.max_seq = int(n_head), int(n_kv), int(head_dim), int(max_seq)
        d = _ATTENTION_DESC.pack(_type_code(dtype), self.n_head, self.n_kv, self.head_dim, int(page_size), self.max_seq,
                                 int(max_length))
        h = ctypes.c_void_p()
        _check(_lm_lib().fiona_attention_create(d, ctypes.byref(h)), "fiona_attention_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().fiona_attention_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def paged_attention(att: Attention, q, k_cache, v_cache, page_table, lengths, out, scale=None, window: int = 0,
                    softcap: float = 0.0, lse=None, stream=None) -> None:
    """fiona_paged_attention: q [n_seq][n_head][d] over the caches [n_pages][page_size][n_kv][d], page_table int32
    [n_seq][table_width], lengths int32 [n_seq] -> out [n_seq][n_head][d] and lse float32 [n_seq][n_head].
    scale: default head_dim ** -0.5."""
    cache, _, dev, _, _ = _cache_desc(k_cache, v_cache)
    n = q.shape[0]
    shape = (n, att.n_head, att.head_dim)
    qs, os_ = _rows(q, "q", att.dtype, shape, dev), _rows(out, "out", att.dtype, shape, dev)
    width = page_table.shape[-1]
    ts = _rows(page_table, "page_table", _INT[4], (n, width), dev)
    lp = _packed(lse, "lse", _INT["f32"], (n, att.n_head), dev) if lse is not None else 0
    args = _ATTENTION_ARGS.pack(n, width, int(window), float(scale) if scale is not None else att.head_dim ** -0.5,
                                float(softcap), q.data_ptr(), out.data_ptr(), lp, qs[0], qs[1], os_[0], os_[1],
                                ts[0], page_table.data_ptr(), _packed(lengths, "lengths", _INT[4], (n,), dev))
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_paged_attention(att.handle, cache, args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_paged_attention")
    _modified[0](out if lse is None else (out, lse))


class Adapters:
    """The workspace of adapter_linear and adapter_backward (fiona_adapters_create)."""

    def __init__(self, dtype, n_adapter: int, max_rank: int, d_in: int, d_out: int, max_tokens: int,
                 forward_only: bool = False):
        self.dtype = dtype
        self.n_adapter, self.max_rank, self.d_in, self.d_out = int(n_adapter), int(max_rank), int(d_in), int(d_out)
        d = _ADAPTERS_DESC.pack(_type_code(dtype), self.n_adapter, self.max_rank, self.d_in, self.d_out, int(max_tokens),
                                1 if forward_only else 0)
        h = ctypes.c_void_p()
        _check(_lm_lib().fiona_adapters_create(d, ctypes.byref(h)), "fiona_adapters_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().fiona_adapters_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _adapter_args(ad: Adapters, x, ids, A, B, ranks, scaling):
    """(the shared fields' values, n_tok, device)"""
    n, dev, dt = x.shape[0], x.get_device(), ad.dtype
    xs = _rows(x, "x", dt, (n, ad.d_in), dev)
    return (n, x.data_ptr(), _packed(A, "A", dt, (ad.n_adapter, ad.max_rank, ad.d_in), dev),
            _packed(B, "B", dt, (ad.n_adapter, ad.d_out, ad.max_rank), dev), _packed(ids, "ids", _INT[4], (n,), dev),
            _packed(ranks, "ranks", _INT[4], (ad.n_adapter,), dev) if ranks is not None else 0,
            _packed(scaling, "scaling", _INT["f32"], (ad.n_adapter,), dev) if scaling is not None else 0, xs[0]), n, dev


def adapter_linear(ad: Adapters, x, ids, A, B, base, y, ranks=None, scaling=None, stream=None) -> None:
    """fiona_adapter_linear: y [n_tok][d_out] = base (or None: zero) plus each token's adapter's part of
    x [n_tok][d_in]; ids int32 [n_tok] (outside the table: none), A [n_adapter][max_rank][d_in],
    B [n_adapter][d_out][max_rank], ranks int32 [n_adapter], scaling float32 [n_adapter].  y may be base."""
    head, n, dev = _adapter_args(ad, x, ids, A, B, ranks, scaling)
    shape = (n, ad.d_out)
    bp, bs = (base.data_ptr(), _rows(base, "base", ad.dtype, shape, dev)[0]) if base is not None else (0, 0)
    ys = _rows(y, "y", ad.dtype, shape, dev)
    args = _ADAPTER_ARGS.pack(*head, bp, y.data_ptr(), bs, ys[0], 0, 0, 0, 0, 0, 0, 0, 0)
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_adapter_linear(ad.handle, args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_adapter_linear")
    _modified[0](y)


def adapter_backward(ad: Adapters, x, ids, A, B, dy, dx_base, dx, dA, dB, ranks=None, scaling=None, stream=None) -> None:
    """fiona_adapter_backward: dx [n_tok][d_in] = dx_base (or None: zero) plus the adapters' part, and dA, dB
    (shaped as A and B) from dy [n_tok][d_out].  dx may be dx_base."""
    head, n, dev = _adapter_args(ad, x, ids, A, B, ranks, scaling)
    dt = ad.dtype
    gs = _rows(dy, "dy", dt, (n, ad.d_out), dev)
    bp, bs = (dx_base.data_ptr(), _rows(dx_base, "dx_base", dt, (n, ad.d_in), dev)[0]) if dx_base is not None else (0, 0)
    xs = _rows(dx, "dx", dt, (n, ad.d_in), dev)
    args = _ADAPTER_ARGS.pack(*head, 0, 0, 0, 0, dy.data_ptr(), bp, dx.data_ptr(),
                              _packed(dA, "dA", dt, (ad.n_adapter, ad.max_rank, ad.d_in), dev),
                              _packed(dB, "dB", dt, (ad.n_adapter, ad.d_out, ad.max_rank), dev), gs[0], bs, xs[0])
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_adapter_backward(ad.handle, args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_adapter_backward")
    _modified[0]((dx, dA, dB))


def _shared(t, name, dtype, dev):
    """The address of one value that a call reads on the device."""
    return _packed(t, name, dtype, (1,), dev)


def layer_norm(x, weight, bias, y, eps: float = 1e-5, residual=None, total=None, mean=None, rstd=None, stream=None) -> None:
    """fiona_layer_norm: y [n][d] = the norm of x [n][d], or of x + residual, which total receives; weight, bias [d] (x's
    type or float32, or None: one and zero); mean, rstd float32 [n].  y or total may be x or residual."""
    shape, dt, dev = x.shape, x.dtype, x.get_device()
    if len(shape) != 2:
        raise ValueError("x must have shape [n][width]")
    code = _type_code(dt)
    n, d = shape
    f32 = _INT["f32"]
    w = weight if weight is not None else bias
    wt = dt if w is None or w.dtype is dt else f32
    xs, ys = _rows(x, "x", dt, shape, dev), _rows(y, "y", dt, shape, dev)
    rp = rs = tp = ts = 0
    if residual is not None:
        rp, rs = residual.data_ptr(), _rows(residual, "residual", dt, shape, dev)[0]
    if total is not None:
        tp, ts = total.data_ptr(), _rows(total, "total", dt, shape, dev)[0]
    args = _NORM_ARGS.pack(n, d, code, code if wt is dt else 0, eps, x.data_ptr(), rp,
                           _packed(weight, "weight", wt, (d,), dev) if weight is not None else 0,
                           _packed(bias, "bias", wt, (d,), dev) if bias is not None else 0, y.data_ptr(), tp,
                           _packed(mean, "mean", f32, (n,), dev) if mean is not None else 0,
                           _packed(rstd, "rstd", f32, (n,), dev) if rstd is not None else 0, xs[0], rs, ys[0], ts)
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_layer_norm(args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_layer_norm")
    _modified[0]([t for t in (y, total, mean, rstd) if t is not None])


class _Handle:
    """A handle of the library's, freed with the object."""

    _destroy = ""

    def _create(self, create, desc):
        h = ctypes.c_void_p()
        _check(getattr(_lm_lib(), create)(desc, ctypes.byref(h)), create)
        self._h = h

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            getattr(lib(), self._destroy)(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LayerNorm(_Handle):
    """The workspace of layer_norm_backward (fiona_norm_create).  weight_dtype: dtype (default) or float32."""

    _destroy = "fiona_norm_destroy"

    def __init__(self, dtype, width: int, max_rows: int, weight_dtype=None):
        self.dtype, self.width, self.max_rows = dtype, int(width), int(max_rows)
        self.weight_dtype = dtype if weight_dtype is None else weight_dtype
        self._create("fiona_norm_create", _NORM_DESC.pack(_type_code(dtype), _type_code(self.weight_dtype), self.width,
                                                          self.max_rows))


def layer_norm_backward(ln: LayerNorm, dy, x, weight, mean, rstd, dx_base, dx, dweight=None, dbias=None, stream=None) -> None:
    """fiona_layer_norm_backward: dx [n][d] = dx_base (or None: zero) plus the gradient through the norm of x (layer_norm's
    total, where it had a residual) from dy [n][d]; dweight, dbias [d].  dx may be dx_base, dy or x."""
    n, dev, dt, wt, f32 = x.shape[0], x.get_device(), ln.dtype, ln.weight_dtype, _INT["f32"]
    shape, row = (n, ln.width), (ln.width,)
    gs, xs, ds = _rows(dy, "dy", dt, shape, dev), _rows(x, "x", dt, shape, dev), _rows(dx, "dx", dt, shape, dev)
    bp = bs = 0
    if dx_base is not None:
        bp, bs = dx_base.data_ptr(), _rows(dx_base, "dx_base", dt, shape, dev)[0]
    args = _NORM_BACKWARD_ARGS.pack(n, dy.data_ptr(), x.data_ptr(),
                                    _packed(weight, "weight", wt, row, dev) if weight is not None else 0,
                                    _packed(mean, "mean", f32, (n,), dev), _packed(rstd, "rstd", f32, (n,), dev), bp, dx.data_ptr(),
                                    _packed(dweight, "dweight", wt, row, dev) if dweight is not None else 0,
                                    _packed(dbias, "dbias", wt, row, dev) if dbias is not None else 0, gs[0], xs[0], bs, ds[0])
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_layer_norm_backward(ln.handle, args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_layer_norm_backward")
    _modified[0]([t for t in (dx, dweight, dbias) if t is not None])


class TokenLoss(_Handle):
    """The workspace of preference_loss and policy_loss (fiona_token_loss_create)."""

    _destroy = "fiona_token_loss_destroy"

    def __init__(self, dtype, vocab: int, max_tokens: int, max_pairs: int = 0):
        self.dtype, self.vocab, self.max_tokens, self.max_pairs = dtype, int(vocab), int(max_tokens), int(max_pairs)
        self._create("fiona_token_loss_create", _TOKEN_LOSS_DESC.pack(_type_code(dtype), self.vocab, self.max_tokens,
                                                                      self.max_pairs))


def preference_loss(tl: TokenLoss, logits, targets, offsets, reference, loss, logps, dlogits=None, beta: float = 0.1,
                    label_smoothing: float = 0.0, weights=None, stream=None) -> None:
    """fiona_preference_loss: logits [n_tok][vocab], targets int32 [n_tok] (outside the vocabulary: not counted), offsets int32
    [2 n_pair + 1], reference float32 [2 n_pair] -> loss float32 [n_pair], logps float32 [2 n_pair] and dlogits
    [n_tok][vocab] (None: not wanted; it may be logits).  weights float32 [n_pair]: default 1 / n_pair."""
    n, p, dev, i32, f32 = logits.shape[0], loss.shape[0], logits.get_device(), _INT[4], _INT["f32"]
    shape = (n, tl.vocab)
    zs = _rows(logits, "logits", tl.dtype, shape, dev)
    dp = ds = 0
    if dlogits is not None:
        dp, ds = dlogits.data_ptr(), _rows(dlogits, "dlogits", tl.dtype, shape, dev)[0]
    args = _PREFERENCE_ARGS.pack(n, p, beta, label_smoothing, logits.data_ptr(), dp, zs[0], ds,
                                 _packed(targets, "targets", i32, (n,), dev), _packed(offsets, "offsets", i32, (2 * p + 1,), dev),
                                 _packed(reference, "reference", f32, (2 * p,), dev),
                                 _packed(weights, "weights", f32, (p,), dev) if weights is not None else 0,
                                 _packed(loss, "loss", f32, (p,), dev), _packed(logps, "logps", f32, (2 * p,), dev))
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_preference_loss(tl.handle, args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_preference_loss")
    _modified[0]((loss, logps) if dlogits is None else (loss, logps, dlogits))


def policy_loss(tl: TokenLoss, logits, targets, old, advantages, loss, logps, dlogits=None, reference=None,
                clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0, weights=None, stream=None) -> None:
    """fiona_policy_loss: logits [n_tok][vocab], targets int32 [n_tok] (outside the vocabulary: not counted), old, advantages
    and, with kl > 0, reference float32 [n_tok] -> loss, logps float32 [n_tok] and dlogits [n_tok][vocab] (None: not
    wanted; it may be logits).  weights float32 [n_tok]: default 1 / n_tok."""
    n, dev, f32 = logits.shape[0], logits.get_device(), _INT["f32"]
    shape, each = (n, tl.vocab), (n,)
    zs = _rows(logits, "logits", tl.dtype, shape, dev)
    dp = ds = 0
    if dlogits is not None:
        dp, ds = dlogits.data_ptr(), _rows(dlogits, "dlogits", tl.dtype, shape, dev)[0]
    args = _POLICY_ARGS.pack(n, clip_low, clip_high, kl, logits.data_ptr(), dp, zs[0], ds,
                             _packed(targets, "targets", _INT[4], each, dev), _packed(old, "old", f32, each, dev),
                             _packed(advantages, "advantages", f32, each, dev),
                             _packed(reference, "reference", f32, each, dev) if reference is not None else 0,
                             _packed(weights, "weights", f32, each, dev) if weights is not None else 0,
                             _packed(loss, "loss", f32, each, dev), _packed(logps, "logps", f32, each, dev))
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_policy_loss(tl.handle, args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_policy_loss")
    _modified[0]((loss, logps) if dlogits is None else (loss, logps, dlogits))


class AdamW(_Handle):
    """An optimiser over many tensors (fiona_adamw_create), whose memory it keeps: lists of contiguous tensors of the same
    shape at the same place.  params, grads: float32, float16 or bfloat16; masters: float32, beside 16-bit parameters; m, v: float32,
    or float8_e4m3fn with m_scales, v_scales float32 [ceil(n / 256)] (v then holds the root).  weight_decay: one for all or
    a list.  Parameters may require a gradient: a step is not recorded."""

    _destroy = "fiona_adamw_destroy"

    def __init__(self, params, grads, m, v, masters=None, m_scales=None, v_scales=None, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.01, seed: int = 0):
        import torch

        _lm_lib()
        lists = {"params": params, "grads": grads, "m": m, "v": v, "masters": masters, "m_scales": m_scales, "v_scales": v_scales}
        lists = {k: list(t) for k, t in lists.items() if t is not None}
        if _forward[0]._current_level >= 0:
            _no_tangents({"%s[%d]" % (k, i): x for k, t in lists.items() for i, x in enumerate(t)})
        # What a step writes, tensors that share a version counter (views of one) once.
        roots = {id(b): b for b in (_root(x) for k in lists if k != "grads" for x in lists[k] if x is not None)}
        lists["params"] = [x.detach() for x in lists["params"]]
        n = len(lists["params"])
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        for name, t in list(lists.items()) + [("weight_decay", decay)]:
            if len(t) != n:
                raise ValueError("%s has %d entries, params %d" % (name, len(t), n))
        self.dtype = lists["params"][0].dtype if n else torch.float32
        code, f32 = _type_code(self.dtype), torch.float32
        small = n > 0 and lists["m"][0].dtype is torch.float8_e4m3fn
        if small != ("m_scales" in lists) or small != ("v_scales" in lists):
            raise ValueError("m_scales and v_scales go with states of 8 bits")
        self.device = lists["params"][0].get_device() if n else None
        packed = []
        for i in range(n):
            shape, count = lists["params"][i].shape, lists["params"][i].numel()
            kinds = [("params", self.dtype, shape), ("grads", self.dtype, shape), ("masters", f32, shape),
                     ("m", torch.float8_e4m3fn if small else f32, shape), ("v", torch.float8_e4m3fn if small else f32, shape),
                     ("m_scales", f32, (-(-count // 256),)), ("v_scales", f32, (-(-count // 256),))]
            at = []
            for name, dtype, want in kinds:
                t = lists[name][i] if name in lists else None
                at.append(_packed(t, "%s[%d]" % (name, i), dtype, want, self.device) if t is not None else 0)
            packed.append(_ADAMW_TENSOR.pack(*at, count, decay[i]))
        table = ctypes.create_string_buffer(b"".join(packed), max(1, n * _ADAMW_TENSOR.size))
        if n:
            _stream_of(None, self.device)      # (the current device is the tensors')
        self._create("fiona_adamw_create", _ADAMW_DESC.pack(code, 8 if small else 32, n, int(seed) & 0xFFFFFFFF, betas[0], betas[1], eps,
                                                            ctypes.addressof(table)))
        # Aliases: their memory stays, whatever becomes of the tensors given.
        self._tensors = {k: [x if x is None else x.detach() for x in t] for k, t in lists.items()}
        self._written = [b.detach() for b in roots.values()]


def _root(t):
    while t._base is not None:
        t = t._base
    return t


def adamw_step(opt: AdamW, lr, step, grad_scale=None, stream=None) -> None:
    """fiona_adamw_step: one step over the handle's tensors; lr float32 [1], step int32 [1] (from 1 on) and grad_scale float32
    [1] (default: one) are read on the device."""
    dev = lr.get_device() if opt.device is None else opt.device
    args = (_shared(lr, "lr", _INT["f32"], dev), _shared(step, "step", _INT[4], dev),
            _shared(grad_scale, "grad_scale", _INT["f32"], dev) if grad_scale is not None else 0)
    if _forward[0]._current_level >= 0:
        _no_tangents(locals())
    rc = lib().fiona_adamw_step(opt.handle, *args, _stream_of(stream, dev))
    if rc:
        raise FionaError(rc, "fiona_adamw_step")
    _modified[0](opt._written)
