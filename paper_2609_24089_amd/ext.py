"""Attention between sequences of two lengths, with an optional learned bias by
buckets of relative position (the attn_ext_* calls of include/flashbob.h).

`cross_attention` and `biased_attention` are the differentiable layers, with
first and second derivatives on the HIP path as `attention` has them (third
ones are not built and raise NotImplementedError); the attn_ext_* functions are the entry points one by one, under the C names.

Query-side tensors are [B, H, Nq, d], key-side ones [B, Hkv, Nk, d] (H a
multiple of Hkv), contiguous bf16 or fp32 on the ROCm device.  Per batch entry
b, query row i has position q_starts[b] + i and key row j position j; row i is
valid for i < q_lens[b], key j for j < kv_lens[b] and, under the causal mask,
j <= q_starts[b] + i.  The lengths and positions are int32 [B] tensors on the
device (None: all rows valid, positions from 0).  A row without a valid key has
O = 0 and L = -inf, and neither it nor a padded row or key has a gradient; what
padded rows hold is never read.

bias is a pair (table, buckets): the scores gain
table[buckets[clamp(j - (q_starts[b] + i), -R, R) + R], h], with table
[num_buckets, H] in fp32 or bf16 and buckets int32 [2 R + 1] on the device
(`relative_buckets` makes the usual ones).  An entry of -2^24 or less (-inf, -1e9)
masks its bucket's keys.
"""
import ctypes

import torch

from . import (BOB_BF16, BOB_F32, BOB_OK, _call, _check_mats, _check_rows, _dtype_code, _fast, _p, _rows_empty,
               _stream, load_library, status_string)

MAX_DISTANCE = 1024
MAX_BUCKETS = 1 << 16


class AttnExt(ctypes.Structure):
    """attn_ext of include/flashbob.h."""
    _fields_ = [("q_lens", ctypes.c_void_p), ("kv_lens", ctypes.c_void_p), ("q_starts", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("buckets", ctypes.c_void_p), ("table_dtype", ctypes.c_int32),
                ("num_buckets", ctypes.c_int32), ("max_distance", ctypes.c_int32)]


ATTN_EXT_FWD, ATTN_EXT_ROWS, ATTN_EXT_COLS, ATTN_EXT_PASS1, ATTN_EXT_PASS2 = range(5)


class AttnExtLaunch(ctypes.Structure):
    """attn_ext_launch of include/flashbob.h."""
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "wave_sets", "parts", "folded", "resident")]

    def __repr__(self):
        return "AttnExtLaunch(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


def _declare(lib):
    """Argument types of the attn_ext_* calls."""
    i32, i64, f32, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
    ext = ctypes.POINTER(AttnExt)
    shape = [i32] + [i64] * 6
    lib.attn_ext_fwd_lse.argtypes = shape + [f32, i32, ext] + [vp] * 5 + [vp, i64, vp]
    lib.attn_ext_bwd.argtypes = shape + [f32, i32, ext] + [vp] * 11 + [vp, i64, vp]
    lib.attn_ext_pass1_rows.argtypes = shape + [f32, i32, ext] + [vp] * 16 + [vp, i64, vp]
    lib.attn_ext_pass2_cols.argtypes = shape + [f32, i32, ext] + [vp] * 15 + [vp, i64, vp]
    for name in ("fwd_lse", "bwd", "pass1_rows", "pass2_cols"):
        getattr(lib, "attn_ext_" + name).restype = i32
    for name in ("fwd", "bwd", "pass1", "pass2"):
        fn = getattr(lib, f"attn_ext_{name}_workspace_bytes")
        fn.argtypes = shape + [i32, ext]
        fn.restype = i64
    lib.attn_ext_layout.argtypes = [i32] + shape + [i32, ext, ctypes.POINTER(AttnExtLaunch)]
    lib.attn_ext_layout.restype = i32


def relative_buckets(num_buckets, max_distance, bidirectional=True, device=None):
    """The bucket of every step of position (key minus query) from -max_distance
    to max_distance: int32 [2 max_distance + 1] for biased_attention.

    Bidirectional, keys before the query use the first half of the buckets and
    keys after it the second; else keys after the query share the bucket of
    step 0 and all buckets serve the keys before it.  Of a side's n buckets the
    first n // 2 are single distances and the others share distances whose
    borders grow by a constant factor: distance x >= e = n // 2 has bucket e + k
    for the largest k < n - e with (x / e)^(n - e) >= (max_distance / e)^k,
    compared in whole numbers.  From max_distance on every key has the last."""
    num_buckets, R = int(num_buckets), int(max_distance)
    n = num_buckets // 2 if bidirectional else num_buckets
    e = n // 2
    if e < 1 or num_buckets > MAX_BUCKETS or (bidirectional and num_buckets % 2 != 0):
        raise ValueError(f"num_buckets must be an even number of at least 4 (2 if one-sided) and at most {MAX_BUCKETS}")
    if not e < R <= MAX_DISTANCE:
        raise ValueError(f"max_distance must exceed the {e} single distances and be at most {MAX_DISTANCE}")
    side, k = [], 0
    for x in range(R + 1):
        while x >= e and k < n - e - 1 and x ** (n - e) * e ** (k + 1) >= R ** (k + 1) * e ** (n - e):
            k += 1
        side.append(x if x < e else e + k)
    after = [n + c for c in side] if bidirectional else [side[0]] * (R + 1)
    return torch.tensor(side[:0:-1] + side[:1] + after[1:], dtype=torch.int32, device=device)


def attn_ext_layout(kernel, dtype, B, H, Hkv, Nq, Nk, d, causal=False, bias=None, device=None):
    """The AttnExtLaunch that kernel ATTN_EXT_FWD, ATTN_EXT_ROWS, ATTN_EXT_COLS,
    ATTN_EXT_PASS1 or ATTN_EXT_PASS2 runs for this problem on `device` (default:
    the current device).  bias: (num_buckets, max_distance) of its table, or None."""
    lib = load_library()
    code = _dtype_code(torch.empty(0, dtype=dtype))
    ext, got = AttnExt(), AttnExtLaunch()
    if bias is not None:  # the query reads the pointers' presence alone
        ext.table = ext.buckets = 16
        ext.table_dtype, ext.num_buckets, ext.max_distance = BOB_F32, *bias
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        rc = lib.attn_ext_layout(kernel, code, B, H, Hkv, Nq, Nk, d, int(bool(causal)), ctypes.byref(ext),
                                 ctypes.byref(got))
    if rc != BOB_OK:
        raise RuntimeError(status_string(rc))
    return got


def _check_lens(name, t, B, like):
    if t is None:
        return
    if t.dtype != torch.int32 or tuple(t.shape) != (B,) or not t.is_contiguous() or t.device != like.device:
        raise ValueError(f"{name} must be a contiguous int32 [B] tensor on the device of the matrices")


def _check_table(t, like_shape, like):
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported table dtype {t.dtype}; expected torch.bfloat16 or torch.float32")
    if tuple(t.shape) != tuple(like_shape) or not t.is_contiguous() or t.device != like.device:
        raise ValueError("a bias table (and its cotangent) must be contiguous [num_buckets, H] on the device of the "
                         "matrices")


def _ptr(t):
    return None if t is None else t.data_ptr()


class _Problem:
    """Checked shapes of one call and its attn_ext."""

    def __init__(self, qside, kside, scale, causal, bias, kv_lens, q_lens, q_starts):
        q, k = qside[0], kside[0]
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("matrices must be [B, H, N, d]")
        B, H, Nq, d = q.shape
        kB, Hkv, Nk, kd = k.shape
        if (kB, kd) != (B, d) or k.dtype != q.dtype or k.device != q.device:
            raise ValueError("key/value-side matrices must match the query side in B, d, dtype and device")
        if (Hkv == 0 and H != 0) or (Hkv > 0 and H % Hkv != 0):
            raise ValueError(f"the query heads ({H}) must be a multiple of the key/value heads ({Hkv})")
        _check_mats(*qside)
        _check_mats(*kside)
        for name, t in (("kv_lens", kv_lens), ("q_lens", q_lens), ("q_starts", q_starts)):
            _check_lens(name, t, B, q)
        self.code, self.like = _dtype_code(q), q
        self.ext = AttnExt(_ptr(q_lens), _ptr(kv_lens), _ptr(q_starts))
        self.table = None
        if bias is not None:
            table, buckets = bias
            if table.dim() != 2 or not 1 <= table.shape[0] <= MAX_BUCKETS:
                raise ValueError(f"the bias table must be [num_buckets, H] with 1 to {MAX_BUCKETS} buckets")
            _check_table(table, (table.shape[0], H), q)
            R = (buckets.numel() - 1) // 2
            if (buckets.dtype != torch.int32 or buckets.dim() != 1 or buckets.numel() != 2 * R + 1 or
                    not 1 <= R <= MAX_DISTANCE or not buckets.is_contiguous() or buckets.device != q.device):
                raise ValueError(f"buckets must be a contiguous int32 [2 R + 1] tensor with R from 1 to {MAX_DISTANCE} "
                                 "on the device of the matrices")
            self.table = table
            self.ext.table, self.ext.buckets = _ptr(table), _ptr(buckets)
            self.ext.table_dtype = BOB_F32 if table.dtype == torch.float32 else BOB_BF16
            self.ext.num_buckets, self.ext.max_distance = table.shape[0], R
        self.shape = (self.code, B, H, Hkv, Nq, Nk, d)
        self.options = (float(scale), int(bool(causal)), ctypes.byref(self.ext))

    def workspace(self, query, stream):
        """(workspace, its pointer, bytes) of a call, kept from reuse until the
        kernels on `stream` are done."""
        with torch.cuda.device(self.like.device):
            n = query(*self.shape, self.options[1], self.options[2])
        if n <= 0:
            return None, None, 0
        ws = torch.empty(n, dtype=torch.uint8, device=self.like.device)
        if stream is not None:
            ws.record_stream(stream)
        return ws, _p(ws), n

    def cotangent(self, gT):
        """The pointer of a cotangent on the table's gradient."""
        if gT is None:
            return None
        if self.table is None:
            raise ValueError("a cotangent on the table's gradient needs a bias")
        if gT.dtype != self.table.dtype:
            raise ValueError("the cotangent on the table's gradient must have the table's dtype")
        _check_table(gT, self.table.shape, self.like)
        return _p(gT)


def _bias(bias):
    table, buckets = (None, None) if bias is None else bias
    return table, buckets


def attn_ext_fwd_lse(Q, K, V, scale, causal=False, bias=None, kv_lens=None, q_lens=None, q_starts=None, out=None,
                     stream=None):
    """Forward: returns (O, L)."""
    if out is None and stream is None:
        got = _fast().ext_fwd(Q, K, V, float(scale), bool(causal), *_bias(bias), kv_lens, q_lens, q_starts)
        if got is not None:
            return got
    p = _Problem((Q,), (K, V), scale, causal, bias, kv_lens, q_lens, q_starts)
    if out is None:
        out = (torch.empty_like(Q), _rows_empty(Q.shape, Q))
    O, L = out
    _check_mats(Q, O)
    _check_rows(Q.shape, L)
    lib = load_library()
    st = _stream(stream, Q)
    ws, wp, n = p.workspace(lib.attn_ext_fwd_workspace_bytes, stream)
    _call(Q, lib.attn_ext_fwd_lse, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(O), _p(L), wp, n, st)
    return O, L


def attn_ext_bwd(Q, K, V, O, dO, L, scale, causal=False, bias=None, kv_lens=None, q_lens=None, q_starts=None,
                 want_table=True, out=None, stream=None):
    """First backward: returns (dQ, dK, dV, D, dT); dT is None without a bias or
    with want_table=False."""
    if out is None and stream is None:
        got = _fast().ext_bwd(Q, K, V, O, dO, L, float(scale), bool(causal), *_bias(bias), kv_lens, q_lens, q_starts,
                              bool(want_table))
        if got is not None:
            return got
    p = _Problem((Q, O, dO), (K, V), scale, causal, bias, kv_lens, q_lens, q_starts)
    _check_rows(Q.shape, L)
    if out is None:
        out = (torch.empty_like(Q), torch.empty_like(K), torch.empty_like(K), _rows_empty(Q.shape, Q),
               torch.empty_like(p.table) if p.table is not None and want_table else None)
    dQ, dK, dV, D, dT = out
    _check_mats(Q, dQ)
    _check_mats(K, dK, dV)
    _check_rows(Q.shape, D)
    tp = p.cotangent(dT)
    lib = load_library()
    st = _stream(stream, Q)
    ws, wp, n = p.workspace(lib.attn_ext_bwd_workspace_bytes, stream)
    _call(Q, lib.attn_ext_bwd, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(O), _p(dO), _p(L), _p(dQ), _p(dK),
          _p(dV), _p(D), tp, wp, n, st)
    return dQ, dK, dV, D, dT


def attn_ext_pass1_rows(Q, K, V, O, dO, gdQ, gdK, gdV, L, D, dQ, scale, causal=False, bias=None, gdT=None,
                        kv_lens=None, q_lens=None, q_starts=None, out=None, stream=None):
    """BoB Pass 1: returns (Qt, dOt, alpha, E).  gdT: the cotangent on dT (None: 0)."""
    if out is None and stream is None:
        got = _fast().ext_pass1(Q, K, V, O, dO, gdQ, gdK, gdV, L, D, dQ, float(scale), bool(causal), *_bias(bias), gdT,
                                kv_lens, q_lens, q_starts)
        if got is not None:
            return got
    p = _Problem((Q, O, dO, gdQ, dQ), (K, V, gdK, gdV), scale, causal, bias, kv_lens, q_lens, q_starts)
    _check_rows(Q.shape, L, D)
    if out is None:
        out = (torch.empty_like(Q), torch.empty_like(Q), _rows_empty(Q.shape, Q), _rows_empty(Q.shape, Q))
    Qt, dOt, alpha, E = out
    _check_mats(Q, Qt, dOt)
    _check_rows(Q.shape, alpha, E)
    lib = load_library()
    st = _stream(stream, Q)
    ws, wp, n = p.workspace(lib.attn_ext_pass1_workspace_bytes, stream)
    _call(Q, lib.attn_ext_pass1_rows, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(O), _p(dO), _p(gdQ), _p(gdK),
          _p(gdV), p.cotangent(gdT), _p(L), _p(D), _p(dQ), _p(Qt), _p(dOt), _p(alpha), _p(E), wp, n, st)
    return Qt, dOt, alpha, E


def attn_ext_pass2_cols(Q, K, V, dO, gdQ, gdK, gdV, L, D, alpha, E, scale, causal=False, bias=None, gdT=None,
                        kv_lens=None, q_lens=None, q_starts=None, want_table=True, out=None, stream=None):
    """BoB Pass 2: returns (Kt, Vt, Tt); Tt is None without a bias or with
    want_table=False."""
    if out is None and stream is None:
        got = _fast().ext_pass2(Q, K, V, dO, gdQ, gdK, gdV, L, D, alpha, E, float(scale), bool(causal), *_bias(bias),
                                gdT, kv_lens, q_lens, q_starts, bool(want_table))
        if got is not None:
            return got
    p = _Problem((Q, dO, gdQ), (K, V, gdK, gdV), scale, causal, bias, kv_lens, q_lens, q_starts)
    _check_rows(Q.shape, L, D, alpha, E)
    if out is None:
        out = (torch.empty_like(K), torch.empty_like(K),
               torch.empty_like(p.table) if p.table is not None and want_table else None)
    Kt, Vt, Tt = out
    _check_mats(K, Kt, Vt)
    tp = p.cotangent(Tt)
    lib = load_library()
    st = _stream(stream, Q)
    ws, wp, n = p.workspace(lib.attn_ext_pass2_workspace_bytes, stream)
    _call(Q, lib.attn_ext_pass2_cols, *p.shape, *p.options, _p(Q), _p(K), _p(V), _p(dO), _p(gdQ), _p(gdK), _p(gdV),
          p.cotangent(gdT), _p(L), _p(D), _p(alpha), _p(E), _p(Kt), _p(Vt), tp, wp, n, st)
    return Kt, Vt, Tt


class _ExtFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, table, buckets, kv_lens, q_lens, q_starts, scale, causal):
        bias = None if table is None else (table, buckets)
        O, L = attn_ext_fwd_lse(q, k, v, scale, causal, bias, kv_lens, q_lens, q_starts)
        # O without its graph: the first backward passes no gradient on to it, and the engine
        # would run this node's backward on zeros for that
        ctx.save_for_backward(q, k, v, table, buckets, kv_lens, q_lens, q_starts, O.detach(), L)
        ctx.scale, ctx.causal = scale, causal
        return O

    @staticmethod
    def backward(ctx, dO):
        q, k, v, table, buckets, kv_lens, q_lens, q_starts, O, L = ctx.saved_tensors
        dq, dk, dv, dt = _ExtBackwardFn.apply(q, k, v, table, buckets, kv_lens, q_lens, q_starts, O, L,
                                              dO.contiguous(), ctx.scale, ctx.causal, ctx.needs_input_grad[3])
        return dq, dk, dv, dt, None, None, None, None, None, None


class _ExtBackwardFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, table, buckets, kv_lens, q_lens, q_starts, O, L, dO, scale, causal, want_table):
        bias = None if table is None else (table, buckets)
        dq, dk, dv, D, dt = attn_ext_bwd(q, k, v, O, dO, L, scale, causal, bias, kv_lens, q_lens, q_starts,
                                         want_table=want_table)
        ctx.save_for_backward(q, k, v, table, buckets, kv_lens, q_lens, q_starts, O, L, dO, D, dq.detach())
        ctx.set_materialize_grads(False)
        ctx.scale, ctx.causal = scale, causal
        return dq, dk, dv, dt

    @staticmethod
    def backward(ctx, gdq, gdk, gdv, gdt):
        q, k, v, table, buckets, kv_lens, q_lens, q_starts, O, L, dO, D, dq = ctx.saved_tensors
        cot = [torch.zeros_like(x) if g is None else g.contiguous() for g, x in ((gdq, q), (gdk, k), (gdv, v))]
        more = dict(bias=None if table is None else (table, buckets), gdT=None if gdt is None else gdt.contiguous(),
                    kv_lens=kv_lens, q_lens=q_lens, q_starts=q_starts)
        Qt, dOt, alpha, E = attn_ext_pass1_rows(q, k, v, O, dO, *cot, L, D, dq, ctx.scale, ctx.causal, **more)
        Kt, Vt, Tt = attn_ext_pass2_cols(q, k, v, dO, *cot, L, D, alpha, E, ctx.scale, ctx.causal,
                                         want_table=ctx.needs_input_grad[3], **more)
        if torch.is_grad_enabled():
            Qt, Kt, Vt, dOt, Tt = _ExtSecondFn.apply(Qt, Kt, Vt, dOt, Tt, q, k, v, table, dO, gdq, gdk, gdv, gdt)
        return Qt, Kt, Vt, Tt, None, None, None, None, None, None, dOt, None, None, None


class _ExtSecondFn(torch.autograd.Function):
    """The second backward's results, tied to what they depend on: asking for a
    third derivative has to fail, not to leave out these terms."""

    @staticmethod
    def forward(ctx, Qt, Kt, Vt, dOt, Tt, *depends):
        return Qt, Kt, Vt, dOt, Tt

    @staticmethod
    def backward(ctx, *g):
        raise NotImplementedError("third derivatives of cross_attention and biased_attention are not built")


def _layer(q, k, v, table, buckets, scale, causal, kv_lens, q_lens, q_starts):
    if scale is None:
        scale = q.shape[-1] ** -0.5
    if not torch.compiler.is_compiling():
        # the same functions in C++ (csrc/torch_binding.cpp); None for calls it does not take
        O = _fast().ext_attention(q, k, v, float(scale), bool(causal), table, buckets, kv_lens, q_lens, q_starts)
        if O is not None:
            return O
    bias = None if table is None else (table, buckets)
    _Problem((q,), (k, v), scale, causal, bias, kv_lens, q_lens, q_starts)
    return _ExtFn.apply(q, k, v, table, buckets, kv_lens, q_lens, q_starts, float(scale), bool(causal))


def cross_attention(q, k, v, scale=None, kv_lens=None, q_lens=None):
    """Attention of the queries q [B, H, Nq, d] to another sequence's keys and
    values k, v [B, Hkv, Nk, d], with first and second derivatives on the HIP
    path.  kv_lens, q_lens: the valid rows of each padded batch entry.  scale
    defaults to 1/sqrt(d)."""
    return _layer(q, k, v, None, None, scale, False, kv_lens, q_lens, None)


def biased_attention(q, k, v, table, buckets, scale=None, causal=False, kv_lens=None, q_lens=None, q_starts=None):
    """Attention with the learned bias table[buckets[...], h] by key position
    minus query position, with first and second derivatives on the HIP path for
    q, k, v and the table.  q_starts: the position of the first query row of
    each batch entry, for the continuation of sequences whose keys and values
    lie in a cache of kv_lens rows.  scale defaults to 1/sqrt(d)."""
    if table is None or buckets is None:
        raise ValueError("biased_attention needs a table and its buckets; cross_attention has no bias")
    return _layer(q, k, v, table, buckets, scale, causal, kv_lens, q_lens, q_starts)
