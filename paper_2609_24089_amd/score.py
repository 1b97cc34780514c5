"""Attention over capped scores, with a bias that falls with distance, and masks by spans of
positions: packed documents and prefixes (the attn_score_* calls of include/flashbob.h).

`scored_attention` is the differentiable layer, with first and second derivatives on the HIP path as
`cross_attention` and `biased_attention` have them (third ones raise NotImplementedError); the
attn_score_* functions are the entry points one by one, under the C names.

Matrices, valid lengths (kv_lens, q_lens), positions past a cache (q_starts), the causal mask and rows
without a valid key are as in ext.py.  With s = scale q.k the scores are

  cap tanh(s / cap) - slopes[h] |key position - query position|

cap: a positive number, or None: s itself.  slopes: fp32 [H] on the device, or None: no bias; they have
no gradient.  spans: int32 [B, Nk, 4] on the device (`attention_spans` makes them), or None: the causal
mask or none.  Position p's query sees the keys spans[b, p, 0] <= j < spans[b, p, 1] and its key is seen by the
queries of the positions spans[b, p, 2] <= i < spans[b, p, 3]; both have to tell the same mask.  Keys and
values that a mask hides have to be finite where kv_lens counts them.
"""
import ctypes

import torch

from . import (BOB_OK, _call, _check_mats, _check_rows, _differentiated, _dtype_code, _fast, _has_tangent, _p, _rows_empty,
               _stream, _uncompiled, load_library, status_string)
from .ext import AttnExtLaunch, _Problem, _ptr

ATTN_SCORE_FWD, ATTN_SCORE_BWD, ATTN_SCORE_PASS1, ATTN_SCORE_PASS2 = range(4)
MIN_CAP, MAX_CAP = 1e-6, 1e6


class AttnScore(ctypes.Structure):
    """attn_score of include/flashbob.h."""
    _fields_ = [("q_lens", ctypes.c_void_p), ("kv_lens", ctypes.c_void_p), ("q_starts", ctypes.c_void_p),
                ("spans", ctypes.c_void_p), ("slopes", ctypes.c_void_p), ("cap", ctypes.c_float)]


def _declare(lib):
    """Argument types of the attn_score_* calls."""
    i32, i64, f32, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
    score = ctypes.POINTER(AttnScore)
    shape = [i32] + [i64] * 6
    for name, pointers in (("fwd_lse", 6), ("bwd", 11), ("pass1_rows", 16), ("pass2_cols", 13)):
        fn = getattr(lib, "attn_score_" + name)
        fn.argtypes = shape + [f32, i32, score] + [vp] * pointers + [vp, i64, vp]
        fn.restype = i32
    lib.attn_score_workspace_bytes.argtypes = [i32] + shape + [i32, score]
    lib.attn_score_workspace_bytes.restype = i64
    lib.attn_score_layout.argtypes = [i32] + shape + [i32, score, ctypes.POINTER(AttnExtLaunch)]
    lib.attn_score_layout.restype = i32


def _whole(name, t, shapes, device):
    if t.dtype not in (torch.int32, torch.int64) or tuple(t.shape) not in shapes:
        raise ValueError(f"{name} must be an int32 or int64 tensor of shape {' or '.join(map(str, shapes))}")
    return t.to(device=device, dtype=torch.int64)


def attention_spans(B, N, documents=None, prefix_lens=None, device=None):
    """The causal mask of B sequences of N positions inside documents, behind prefixes, or both, as the spans of
    scored_attention: int32 [B, N, 4], made on `device` (default: that of the arguments) without a synchronisation,
    once for all layers of a model.

    documents: whole numbers [B, N], the document of every position.  A run of equal numbers is one document, whose
    positions see each other alone; a negative number is padding, which sees nothing and is seen by nothing.
    prefix_lens: whole numbers [B], or [B, N] (each document's number is that at its first position): so many leading
    positions of every document (of the sequence, without documents) see each other both ways."""
    B, N = int(B), int(N)
    if B < 0 or N < 0:
        raise ValueError("B and N must not be negative")
    if device is None:
        device = next((t.device for t in (documents, prefix_lens) if t is not None), None)
    at = torch.arange(N, device=device).expand(B, N)
    first, end = torch.zeros_like(at), torch.full_like(at, N)
    if documents is not None:
        documents = _whole("documents", documents, [(B, N)], device)
        new = documents[:, 1:] != documents[:, :-1]  # position p + 1 begins a document
        first[:, 1:] = torch.where(new, at[:, 1:], 0)
        first = first.cummax(1).values if N > 0 else first
        end[:, :-1] = torch.where(new, at[:, 1:], N)
        end = end.flip(1).cummin(1).values.flip(1) if N > 0 else end
    both = first
    if prefix_lens is not None:
        prefix_lens = _whole("prefix_lens", prefix_lens, [(B,), (B, N)], device)
        n = prefix_lens[:, None].expand(B, N) if prefix_lens.dim() == 1 else prefix_lens.gather(1, first)
        both = torch.minimum(first + n.clamp(0, N), end)
    spans = torch.stack([first, torch.maximum(at + 1, both), torch.where(at < both, first, at), end], 2)
    if documents is not None:
        spans = spans * (documents >= 0)[:, :, None]
    return spans.to(torch.int32)


def attn_score_layout(kernel, dtype, B, H, Hkv, Nq, Nk, d, causal=False, cap=None, slopes=False, spans=False,
                      device=None):
    """The AttnExtLaunch that kernel ATTN_EXT_FWD, ATTN_EXT_ROWS, ATTN_EXT_COLS, ATTN_EXT_PASS1 or ATTN_EXT_PASS2
    runs for this problem on `device` (default: the current device).  slopes, spans: whether there are any."""
    lib = load_library()
    code = _dtype_code(torch.empty(0, dtype=dtype))
    # the query reads the pointers' presence alone
    score, got = AttnScore(None, None, None, 16 if spans else None, 16 if slopes else None, cap or 0.0), AttnExtLaunch()
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        rc = lib.attn_score_layout(kernel, code, B, H, Hkv, Nq, Nk, d, int(bool(causal)), ctypes.byref(score),
                                   ctypes.byref(got))
    if rc != BOB_OK:
        raise RuntimeError(status_string(rc))
    return got


class _Score(_Problem):
    """Checked shapes of one call and its attn_score."""

    def __init__(self, qside, kside, scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts):
        super().__init__(qside, kside, scale, causal, None, kv_lens, q_lens, q_starts)
        q, k = qside[0], kside[0]
        (B, H), Nk = q.shape[:2], k.shape[2]
        if cap is not None and not MIN_CAP <= float(cap) <= MAX_CAP:
            raise ValueError(f"cap must be a number from {MIN_CAP} to {MAX_CAP}, or None")
        if slopes is not None:
            if slopes.dtype != torch.float32 or tuple(slopes.shape) != (H,) or not slopes.is_contiguous() or \
                    slopes.device != q.device:
                raise ValueError("slopes must be a contiguous fp32 [H] tensor on the device of the matrices")
            if slopes.requires_grad and torch.is_grad_enabled() or _has_tangent(slopes):
                raise ValueError("slopes have no gradient; detach them")
        if spans is not None:
            if spans.dtype != torch.int32 or tuple(spans.shape) != (B, Nk, 4) or not spans.is_contiguous() or \
                    spans.device != q.device:
                raise ValueError("spans must be a contiguous int32 [B, Nk, 4] tensor on the device of the matrices")
            if causal:
                raise ValueError("spans say which keys a query sees: causal must be False with them")
        self.score = AttnScore(_ptr(q_lens), _ptr(kv_lens), _ptr(q_starts), _ptr(spans), _ptr(slopes), float(cap or 0))
        self.options = (float(scale), int(bool(causal)), ctypes.byref(self.score))

    def space(self, call, stream):
        lib = load_library()
        return self.workspace(lambda *args: lib.attn_score_workspace_bytes(call, *args), stream)


def _check_rest(O, Orest):
    if Orest is not None:
        _check_mats(O, Orest)


def attn_score_fwd_lse(Q, K, V, scale, causal=False, cap=None, slopes=None, spans=None, kv_lens=None, q_lens=None,
                       q_starts=None, want_rest=False, out=None, stream=None):
    """Forward: returns (O, Orest, L).  Orest is what rounding O left, for the backward calls (None unless wanted)."""
    p = _Score((Q,), (K, V), scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts)
    if out is None:
        out = (torch.empty_like(Q), torch.empty_like(Q) if want_rest else None, _rows_empty(Q.shape, Q))
    O, Orest, L = out
    _check_mats(Q, O)
    _check_rest(Q, Orest)
    _check_rows(Q, L)
    st = _stream(stream, Q)
    ws, wp, n = p.space(ATTN_SCORE_FWD, stream)
    _call(Q, load_library().attn_score_fwd_lse, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(O), _ptr(Orest), _p(L),
          wp, n, st)
    return O, Orest, L


def attn_score_bwd(Q, K, V, O, Orest, dO, L, scale, causal=False, cap=None, slopes=None, spans=None, kv_lens=None,
                   q_lens=None, q_starts=None, out=None, stream=None):
    """First backward: returns (dQ, dK, dV, D).  Orest: the forward's, or None (0)."""
    p = _Score((Q, O, dO), (K, V), scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts)
    _check_rest(Q, Orest)
    _check_rows(Q, L)
    if out is None:
        out = (torch.empty_like(Q), torch.empty_like(K), torch.empty_like(K), _rows_empty(Q.shape, Q))
    dQ, dK, dV, D = out
    _check_mats(Q, dQ)
    _check_mats(K, dK, dV)
    _check_rows(Q, D)
    st = _stream(stream, Q)
    ws, wp, n = p.space(ATTN_SCORE_BWD, stream)
    _call(Q, load_library().attn_score_bwd, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(O), _ptr(Orest), _p(dO),
          _p(L), _p(dQ), _p(dK), _p(dV), _p(D), wp, n, st)
    return dQ, dK, dV, D


def attn_score_pass1_rows(Q, K, V, O, Orest, dO, gdQ, gdK, gdV, L, D, dQ, scale, causal=False, cap=None, slopes=None,
                          spans=None, kv_lens=None, q_lens=None, q_starts=None, out=None, stream=None):
    """BoB Pass 1: returns (Qt, dOt, alpha, E).  Orest: the forward's, or None (0)."""
    p = _Score((Q, O, dO, gdQ, dQ), (K, V, gdK, gdV), scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts)
    _check_rest(Q, Orest)
    _check_rows(Q, L, D)
    if out is None:
        out = (torch.empty_like(Q), torch.empty_like(Q), _rows_empty(Q.shape, Q), _rows_empty(Q.shape, Q))
    Qt, dOt, alpha, E = out
    _check_mats(Q, Qt, dOt)
    _check_rows(Q, alpha, E)
    st = _stream(stream, Q)
    ws, wp, n = p.space(ATTN_SCORE_PASS1, stream)
    _call(Q, load_library().attn_score_pass1_rows, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(O), _ptr(Orest),
          _p(dO), _p(gdQ), _p(gdK), _p(gdV), _p(L), _p(D), _p(dQ), _p(Qt), _p(dOt), _p(alpha), _p(E), wp, n, st)
    return Qt, dOt, alpha, E


def attn_score_pass2_cols(Q, K, V, dO, gdQ, gdK, gdV, L, D, alpha, E, scale, causal=False, cap=None, slopes=None,
                          spans=None, kv_lens=None, q_lens=None, q_starts=None, out=None, stream=None):
    """BoB Pass 2: returns (Kt, Vt)."""
    p = _Score((Q, dO, gdQ), (K, V, gdK, gdV), scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts)
    _check_rows(Q, L, D, alpha, E)
    if out is None:
        out = (torch.empty_like(K), torch.empty_like(K))
    Kt, Vt = out
    _check_mats(K, Kt, Vt)
    st = _stream(stream, Q)
    ws, wp, n = p.space(ATTN_SCORE_PASS2, stream)
    _call(Q, load_library().attn_score_pass2_cols, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(dO), _p(gdQ),
          _p(gdK), _p(gdV), _p(L), _p(D), _p(alpha), _p(E), _p(Kt), _p(Vt), wp, n, st)
    return Kt, Vt


class _ScoreFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, slopes, spans, kv_lens, q_lens, q_starts, scale, causal, cap):
        # fp32 outputs are as exact as their sums
        O, Orest, L = attn_score_fwd_lse(q, k, v, scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts,
                                         want_rest=q.dtype == torch.bfloat16)
        # O without its graph: the first backward passes no gradient on to it, and the engine
        # would run this node's backward on zeros for that
        ctx.save_for_backward(q, k, v, O.detach(), Orest, L, slopes, spans, kv_lens, q_lens, q_starts)
        ctx.options = scale, causal, cap
        return O

    @staticmethod
    def backward(ctx, dO):
        q, k, v, O, Orest, L, *more = ctx.saved_tensors
        dq, dk, dv = _ScoreBackwardFn.apply(q, k, v, O, Orest, L, dO.contiguous(), *more, *ctx.options)
        return (dq, dk, dv) + (None,) * 8


class _ScoreBackwardFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, O, Orest, L, dO, slopes, spans, kv_lens, q_lens, q_starts, scale, causal, cap):
        more = (slopes, spans, kv_lens, q_lens, q_starts)
        dq, dk, dv, D = attn_score_bwd(q, k, v, O, Orest, dO, L, scale, causal, cap, *more)
        ctx.save_for_backward(q, k, v, O, Orest, L, dO, D, dq.detach(), *more)
        ctx.set_materialize_grads(False)
        ctx.options = scale, causal, cap
        return dq, dk, dv

    @staticmethod
    def backward(ctx, gdq, gdk, gdv):
        q, k, v, O, Orest, L, dO, D, dq, *more = ctx.saved_tensors
        more = (*ctx.options, *more)
        cot = [torch.zeros_like(x) if g is None else g.contiguous() for g, x in ((gdq, q), (gdk, k), (gdv, v))]
        Qt, dOt, alpha, E = attn_score_pass1_rows(q, k, v, O, Orest, dO, *cot, L, D, dq, *more)
        Kt, Vt = attn_score_pass2_cols(q, k, v, dO, *cot, L, D, alpha, E, *more)
        if _differentiated(gdq, gdk, gdv):
            Qt, Kt, Vt, dOt = _ScoreSecondFn.apply(Qt, Kt, Vt, dOt, q, k, v, dO, gdq, gdk, gdv)
        return (Qt, Kt, Vt, None, None, None, dOt) + (None,) * 8


class _ScoreSecondFn(torch.autograd.Function):
    """The second backward's results, tied to what they depend on: asking for a
    third derivative has to fail, not to leave out these terms."""

    @staticmethod
    def forward(ctx, Qt, Kt, Vt, dOt, *depends):
        return Qt, Kt, Vt, dOt

    @staticmethod
    def backward(ctx, *g):
        raise NotImplementedError("third derivatives of scored_attention are not built")


def scored_attention(q, k, v, scale=None, causal=False, cap=None, slopes=None, spans=None, kv_lens=None, q_lens=None,
                     q_starts=None):
    """Attention of the queries q [B, H, Nq, d] to k, v [B, Hkv, Nk, d] over capped scores (cap), with a bias that
    falls with distance (slopes), under the causal mask or spans (`attention_spans`), each optional; first and
    second derivatives for q, k and v on the HIP path.  kv_lens, q_lens: the valid rows of each padded batch entry.
    q_starts: the position of the first query row of each entry, for the continuation of sequences whose keys and
    values lie in a cache of kv_lens rows.  scale defaults to 1/sqrt(d)."""
    if scale is None:
        scale = q.shape[-1] ** -0.5
    if torch.compiler.is_compiling():
        return _uncompiled(scored_attention, q, k, v, scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts)
    if cap is None or cap:
        # the same functions in C++ (csrc/torch_binding.cpp); None for calls it does not take
        O = _fast().scored_attention(q, k, v, float(scale), bool(causal), float(cap or 0), slopes, spans, kv_lens, q_lens,
                                     q_starts)
        if O is not None:
            return O
    _Score((q,), (k, v), scale, causal, cap, slopes, spans, kv_lens, q_lens, q_starts)
    return _ScoreFn.apply(q, k, v, slopes, spans, kv_lens, q_lens, q_starts, float(scale), bool(causal), cap)
