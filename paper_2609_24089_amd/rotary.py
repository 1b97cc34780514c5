"""Heads of an attention from a projection's output: norms of queries and keys for each head and the rotation by
position in one pass, with the change of layout (the attn_rotary_* calls of include/flashbob.h).

`rotate_heads` is the differentiable layer, with first and second derivatives on the HIP path (without norms it is
linear, and differentiable any number of times; third derivatives of the norms raise NotImplementedError).
`rotary_attention` is it and `scored_attention`, a layer from the projections to the output.

Queries q [B, H, N, d] and keys k [B, Hkv, N, d] may have any strides whose last is 1; a projection's [B, N, H, d] is
passed as its transpose(1, 2).  (Where data or strides are not multiples of 16 bytes the layer copies them first.)
The results are contiguous.  With a weight [d] (fp32 or bf16) each head vector x becomes w x / sqrt(mean(x^2) + eps)
first.  `rotary` is a pair (freqs, axes): freqs fp64 [pairs], the radians a position, which have no gradient, and axes
int32 [pairs], the axis of the positions that turns each pair (`rotary_frequencies` makes the usual ones); positions are
int32 [axes, B, N], or [B, N] with one axis.  The pairs, a multiple of 8, are those of the first 2 pairs elements: (i, i +
pairs) or, interleaved, (2 i, 2 i + 1); further elements are not rotated.  Angles are formed in fp64.
"""
import ctypes

import torch

from . import (BOB_BF16, BOB_F32, _call, _differentiated, _dtype_code, _fast, _has_tangent, _p, _stream,
               _uncompiled, load_library)
from .score import scored_attention

HEAD_DIMS = (32, 64, 128, 256)


class AttnHeads(ctypes.Structure):
    """attn_heads of include/flashbob.h."""
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("stride_b", "stride_h", "stride_n")]


class AttnRotary(ctypes.Structure):
    """attn_rotary of include/flashbob.h."""
    _fields_ = [("positions", ctypes.c_void_p), ("freqs", ctypes.c_void_p), ("axes", ctypes.c_void_p),
                ("num_axes", ctypes.c_int32), ("pairs", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("weight_dtype", ctypes.c_int32),
                ("eps", ctypes.c_float)]


def _declare(lib):
    """Argument types of the attn_rotary_* calls."""
    i32, i64, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    heads, rotary = ctypes.POINTER(AttnHeads), ctypes.POINTER(AttnRotary)
    shape = [i32] + [i64] * 5
    lib.attn_rotary_fwd.argtypes = shape + [i32, rotary] + [heads] * 4 + [vp]
    lib.attn_rotary_bwd.argtypes = shape + [rotary] + [heads] * 6 + [vp] * 3 + [i64, vp]
    lib.attn_rotary_bwd2.argtypes = shape + [rotary] + [heads] * 6 + [vp] * 2 + [heads] * 4 + [vp] * 3 + [i64, vp]
    for name in ("fwd", "bwd", "bwd2"):
        getattr(lib, "attn_rotary_" + name).restype = i32
    lib.attn_rotary_workspace_bytes.argtypes = shape + [rotary]
    lib.attn_rotary_workspace_bytes.restype = i64


def rotary_frequencies(dims, base=10000.0, sections=None, apart=False, device=None):
    """The rotary pair (freqs, axes) for `dims` rotated elements: pair i of the dims / 2 turns by base^(-2 i / dims)
    radians a position.  sections: how many consecutive pairs each axis of the positions has, (t, h, w) for a video's
    frames, rows and columns; None: one axis.  apart: every axis has frequencies of its own, falling from 1 over its
    section, instead of its section of one series."""
    dims = int(dims)
    if dims < 16 or dims % 16 != 0:
        raise ValueError("dims must be a positive multiple of 16")
    pairs = dims // 2
    sections = (pairs,) if sections is None else tuple(int(n) for n in sections)
    if min(sections) < 0 or sum(sections) != pairs:
        raise ValueError(f"sections must be counts of pairs that sum to dims / 2 = {pairs}")
    if not float(base) > 0:
        raise ValueError("base must be positive")
    own = [-i / n for n in sections for i in range(n)] if apart else [-i / pairs for i in range(pairs)]
    freqs = torch.tensor([float(base) ** x for x in own], dtype=torch.float64, device=device)
    axes = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], dtype=torch.int32, device=device)
    return freqs, axes


def _aligned(t):
    unit = 16 // t.element_size()
    return (t.data_ptr() % 16 == 0 and (t.shape[3] == 1 or t.stride(3) == 1) and
            all(s % unit == 0 for s in t.stride()[:3]))


def _heads(t):
    """t's attn_heads by reference, or None."""
    return None if t is None else ctypes.byref(AttnHeads(t.data_ptr(), *t.stride()[:3]))


def _tokens_first(x):
    """Whether the heads of a token lie together in x."""
    return x.stride(1) < x.stride(2)


def _empty(x, tokens_first):
    B, H, N, d = x.shape
    # x's own method: of its subclass
    return x.new_empty(B, N, H, d).transpose(1, 2) if tokens_first else x.new_empty(B, H, N, d)


def _like(x):
    """An output for gradients of x, in x's order of heads and tokens."""
    return _empty(x, _tokens_first(x))


class _Rotary:
    """Checked shapes of one call and its attn_rotary."""

    def __init__(self, q, k, positions, freqs, axes, q_weight, k_weight, eps, interleaved, stream=None):
        self.stream = stream
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("heads must be [B, H, N, d]")
        B, H, N, d = q.shape
        if (k.shape[0], k.shape[2], k.shape[3]) != (B, N, d) or k.dtype != q.dtype or k.device != q.device:
            raise ValueError("the keys must match the queries in B, N, d, dtype and device")
        if d not in HEAD_DIMS:
            raise ValueError(f"the head dim must be one of {HEAD_DIMS}, not {d}")
        if not q.is_cuda:
            raise ValueError("heads must be on the ROCm device")
        self.code, self.like = _dtype_code(q), q
        pairs = freqs.numel()
        if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous() or freqs.device != q.device or \
                pairs % 8 != 0 or 2 * pairs > d:
            raise ValueError("freqs must be a contiguous fp64 [pairs] tensor on the device of the heads, with a multiple "
                             "of 8 pairs of the head dim")
        if axes is not None and (axes.dtype != torch.int32 or axes.shape != freqs.shape or not axes.is_contiguous() or
                                 axes.device != q.device):
            raise ValueError("axes must be a contiguous int32 [pairs] tensor on the device of the heads, or None")
        if positions.dim() == 2:
            positions = positions[None]
        num = positions.shape[0]
        if positions.dtype != torch.int32 or positions.dim() != 3 or tuple(positions.shape[1:]) != (B, N) or num < 1 or \
                not positions.is_contiguous() or positions.device != q.device:
            raise ValueError("positions must be a contiguous int32 [axes, B, N] (or [B, N]) tensor on the device of the "
                             "heads")
        if num > 1 and axes is None:
            raise ValueError("positions of several axes need the axes of the pairs")
        weights = [w for w in (q_weight, k_weight) if w is not None]
        for w in weights:
            if w.dtype not in (torch.float32, torch.bfloat16) or w.dtype != weights[0].dtype:
                raise TypeError("weights must be torch.bfloat16 or torch.float32, both the same")
            if tuple(w.shape) != (d,) or not w.is_contiguous() or w.device != q.device:
                raise ValueError("weights must be contiguous [d] tensors on the device of the heads")
        if weights and not 0 <= float(eps) < float("inf"):
            raise ValueError("eps must not be negative")
        if not 0 <= B * N <= 1 << 31 or H + k.shape[1] > 65535:
            raise ValueError("at most 2^31 tokens and 65535 heads")
        self.shape = (self.code, B, H, k.shape[1], N, d)
        self.keep = [w if w is None or w.data_ptr() % 16 == 0 else self.copied(w) for w in (q_weight, k_weight)]
        ptr = [None if w is None else w.data_ptr() for w in self.keep]
        self.rotary = AttnRotary(positions.data_ptr(), freqs.data_ptr(), None if axes is None else axes.data_ptr(), num,
                                 pairs, int(bool(interleaved)), *ptr,
                                 BOB_BF16 if weights and weights[0].dtype == torch.bfloat16 else BOB_F32, float(eps))
        self.ref = ctypes.byref(self.rotary)

    def copied(self, t):
        """A copy that the kernels can read, made on the current stream."""
        if self.stream is not None:
            raise ValueError("on a stream of the caller's, data and strides must be multiples of 16 bytes")
        t = t.contiguous()
        return t if t.data_ptr() % 16 == 0 else t.clone()

    def workspace(self):
        """(workspace, its pointer, bytes), kept from reuse until the kernels on the stream are done."""
        n = load_library().attn_rotary_workspace_bytes(*self.shape, self.ref)
        if n <= 0:
            return None, None, 0
        ws = torch.empty(n, dtype=torch.uint8, device=self.like.device)
        if self.stream is not None:
            ws.record_stream(self.stream)
        return ws, _p(ws), n

    def side(self, name, t, like):
        """A tensor of head vectors like `like`, copied if the kernels cannot read it where it lies."""
        if t is None:
            return None
        if t.shape != like.shape or t.dtype != like.dtype or t.device != like.device:
            raise ValueError(f"{name} must have the shape, dtype and device of its heads")
        return t if _aligned(t) else self.copied(t)

    def into(self, name, t, like):
        """An output of the caller's."""
        if t.shape != like.shape or t.dtype != like.dtype or t.device != like.device or not _aligned(t) or \
                any(s == 0 and n > 1 for s, n in zip(t.stride(), t.shape)):
            raise ValueError(f"{name} must have the shape, dtype and device of its heads, a last stride of 1, and data and "
                             "strides in multiples of 16 bytes")
        return t

    def gradient(self, name, t, weight):
        """An output of the caller's for a weight's gradient."""
        if t is not None and (weight is None or t.shape != weight.shape or t.dtype != weight.dtype or
                              t.device != weight.device or not t.is_contiguous()):
            raise ValueError(f"{name} must be like its weight")

    def vector(self, name, t, weight):
        """A cotangent like a weight."""
        if t is None:
            return None
        if weight is None:
            raise ValueError(f"{name} needs a weight")
        if t.shape != weight.shape or t.dtype != weight.dtype or t.device != weight.device:
            raise ValueError(f"{name} must be like the weight")
        return t if t.is_contiguous() and t.data_ptr() % 16 == 0 else self.copied(t)


def _ptr(t):
    return None if t is None else t.data_ptr()


def attn_rotary_fwd(Q, K, positions, freqs, axes=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                    inverse=False, out=None, stream=None):
    """Forward: returns (Qr, Kr), contiguous unless they are given in `out` (any strides in multiples of 16 bytes: a
    cache's slots).  inverse rotates back, without weights alone."""
    p = _Rotary(Q, K, positions, freqs, axes, q_weight, k_weight, eps, interleaved, stream)
    if inverse and (q_weight is not None or k_weight is not None):
        raise ValueError("inverse takes no weights")
    Q, K = p.side("Q", Q, Q), p.side("K", K, K)
    if out is None:
        out = [_empty(x, False) for x in (Q, K)]
    Qr, Kr = p.into("Qr", out[0], Q), p.into("Kr", out[1], K)
    _call(Q, load_library().attn_rotary_fwd, *p.shape, int(bool(inverse)), p.ref, _heads(Q), _heads(K), _heads(Qr),
          _heads(Kr), _stream(stream, Q))
    return Qr, Kr


def attn_rotary_bwd(Q, K, dQr, dKr, positions, freqs, axes=None, q_weight=None, k_weight=None, eps=1e-6,
                    interleaved=False, want_weights=True, out=None, stream=None):
    """Backward: returns (dQ, dK, dWq, dWk); dQ and dK in the order of Q's and K's strides; a weight's gradient is None
    without the weight or with want_weights=False."""
    p = _Rotary(Q, K, positions, freqs, axes, q_weight, k_weight, eps, interleaved, stream)
    order = (Q, K)
    Q, K, dQr, dKr = p.side("Q", Q, Q), p.side("K", K, K), p.side("dQr", dQr, Q), p.side("dKr", dKr, K)
    if out is None:
        out = [_like(x) for x in order] + [None if w is None or not want_weights else torch.empty_like(w)
                                           for w in (q_weight, k_weight)]
    dQ, dK, dWq, dWk = out
    p.into("dQ", dQ, Q), p.into("dK", dK, K)
    p.gradient("dWq", dWq, q_weight), p.gradient("dWk", dWk, k_weight)
    st = _stream(stream, Q)
    ws, wp, n = p.workspace() if dWq is not None or dWk is not None else (None, None, 0)
    _call(Q, load_library().attn_rotary_bwd, *p.shape, p.ref, _heads(Q), _heads(K), _heads(dQr), _heads(dKr),
          _heads(dQ), _heads(dK), _ptr(dWq), _ptr(dWk), wp, n, st)
    return dQ, dK, dWq, dWk


def attn_rotary_bwd2(Q, K, dQr, dKr, gdQ, gdK, positions, freqs, axes=None, q_weight=None, k_weight=None, eps=1e-6,
                     interleaved=False, gdWq=None, gdWk=None, want_weights=True, stream=None):
    """Backward of the backward, for cotangents gdQ, gdK, gdWq, gdWk (each may be None: 0) on its results: returns
    (Qt, Kt, dQrt, dKrt, Wqt, Wkt), None for what is 0 without a weight and for weights that are not wanted."""
    p = _Rotary(Q, K, positions, freqs, axes, q_weight, k_weight, eps, interleaved, stream)
    order = (Q, K)
    Q, K, dQr, dKr = p.side("Q", Q, Q), p.side("K", K, K), p.side("dQr", dQr, Q), p.side("dKr", dKr, K)
    gdQ, gdK = p.side("gdQ", gdQ, Q), p.side("gdK", gdK, K)
    gdWq, gdWk = p.vector("gdWq", gdWq, q_weight), p.vector("gdWk", gdWk, k_weight)
    Qt, Kt = (None if w is None else _like(x) for x, w in zip(order, (q_weight, k_weight)))
    dQrt, dKrt = (_empty(x, False) for x in (Q, K))
    Wqt, Wkt = (None if w is None or not want_weights else torch.empty_like(w) for w in (q_weight, k_weight))
    st = _stream(stream, Q)
    ws, wp, n = p.workspace() if Wqt is not None or Wkt is not None else (None, None, 0)
    _call(Q, load_library().attn_rotary_bwd2, *p.shape, p.ref, _heads(Q), _heads(K), _heads(dQr), _heads(dKr),
          _heads(gdQ), _heads(gdK), _ptr(gdWq), _ptr(gdWk), _heads(Qt), _heads(Kt), _heads(dQrt), _heads(dKrt),
          _ptr(Wqt), _ptr(Wkt), wp, n, st)
    return Qt, Kt, dQrt, dKrt, Wqt, Wkt


class _RotateFn(torch.autograd.Function):
    """The rotation alone: linear, and its own transpose but for the sign of the angles.  A gradient comes in the order
    (`tokens_first`) of what it is the gradient of."""

    @staticmethod
    def forward(ctx, q, k, positions, freqs, axes, interleaved, inverse, tokens_first):
        ctx.save_for_backward(positions, freqs, axes)
        ctx.options = interleaved, not inverse, tuple(_tokens_first(x) for x in (q, k))
        out = [_empty(x, first) for x, first in zip((q, k), tokens_first)]
        return tuple(attn_rotary_fwd(q, k, positions, freqs, axes, interleaved=interleaved, inverse=inverse, out=out))

    @staticmethod
    def backward(ctx, gq, gk):
        return (*_RotateFn.apply(gq, gk, *ctx.saved_tensors, *ctx.options),) + (None,) * 6


class _RotaryFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, freqs, axes, eps, interleaved):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, freqs, axes)
        ctx.options = eps, interleaved
        return attn_rotary_fwd(q, k, positions, freqs, axes, q_weight, k_weight, eps, interleaved)

    @staticmethod
    def backward(ctx, gq, gk):
        q, k, q_weight, k_weight, *more = ctx.saved_tensors
        want = ctx.needs_input_grad[2] or ctx.needs_input_grad[3]
        return (*_RotaryBackwardFn.apply(q, k, q_weight, k_weight, gq, gk, *more, *ctx.options, want),) + (None,) * 5


class _RotaryBackwardFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, gq, gk, positions, freqs, axes, eps, interleaved, want):
        ctx.save_for_backward(q, k, q_weight, k_weight, gq, gk, positions, freqs, axes)
        ctx.set_materialize_grads(False)
        ctx.options = eps, interleaved
        return attn_rotary_bwd(q, k, gq, gk, positions, freqs, axes, q_weight, k_weight, eps, interleaved,
                               want_weights=want)

    @staticmethod
    def backward(ctx, uq, uk, uwq, uwk):
        q, k, q_weight, k_weight, gq, gk, *more = ctx.saved_tensors
        want = ctx.needs_input_grad[2] or ctx.needs_input_grad[3]
        Qt, Kt, gqt, gkt, Wqt, Wkt = attn_rotary_bwd2(q, k, gq, gk, uq, uk, *more, q_weight, k_weight, *ctx.options,
                                                      gdWq=uwq, gdWk=uwk, want_weights=want)
        out = (Qt, Kt, Wqt, Wkt, gqt, gkt)
        if _differentiated(uq, uk, uwq, uwk):
            out = _RotarySecondFn.apply(*out, q, k, q_weight, k_weight, gq, gk, uq, uk, uwq, uwk)
        return (*out,) + (None,) * 6


class _RotarySecondFn(torch.autograd.Function):
    """The second backward's results, tied to what they depend on: asking for a
    third derivative has to fail, not to leave out these terms."""

    @staticmethod
    def forward(ctx, Qt, Kt, Wqt, Wkt, gqt, gkt, *depends):
        return Qt, Kt, Wqt, Wkt, gqt, gkt

    @staticmethod
    def backward(ctx, *g):
        raise NotImplementedError("third derivatives of rotate_heads with norms are not built")


def rotate_heads(q, k, positions, rotary, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    """The queries and keys of an attention, normalised per head (with a weight) and rotated by position: returns
    contiguous (q [B, H, N, d], k [B, Hkv, N, d]), with first and second derivatives for q, k and the weights on the HIP
    path.  The rotary pair and positions are as at the head of this file."""
    freqs, axes = rotary
    if torch.compiler.is_compiling():
        return _uncompiled(rotate_heads, q, k, positions, rotary, q_weight, k_weight, eps, interleaved)
    # the same functions in C++ (csrc/torch_binding.cpp); None for calls it does not take
    y = _fast().rotate_heads(q, k, positions, freqs, axes, q_weight, k_weight, float(eps), bool(interleaved))
    if y is not None:
        return y
    _Rotary(q, k, positions, freqs, axes, q_weight, k_weight, eps, interleaved)
    if freqs.requires_grad and torch.is_grad_enabled() or _has_tangent(freqs):
        raise ValueError("freqs have no gradient; detach them")
    if q_weight is None and k_weight is None:
        return _RotateFn.apply(q, k, positions, freqs, axes, bool(interleaved), False, (False, False))
    return _RotaryFn.apply(q, k, q_weight, k_weight, positions, freqs, axes, float(eps), bool(interleaved))


def rotary_attention(q, k, v, positions, rotary, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, scale=None,
                     causal=False, cap=None, slopes=None, spans=None, kv_lens=None, q_lens=None):
    """scored_attention of the queries and keys that rotate_heads makes of q [B, H, N, d] and k [B, Hkv, N, d], to the
    values v [B, Hkv, N, d] (each in any strides, as a projection leaves them)."""
    q, k = rotate_heads(q, k, positions, rotary, q_weight, k_weight, eps, interleaved)
    return scored_attention(q, k, v.contiguous(), scale, causal, cap, slopes, spans, kv_lens, q_lens)
