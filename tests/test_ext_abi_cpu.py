"""Refusals of the attention between sequences of two lengths, with no GPU: the C calls
check everything before any HIP call, the Python ones before the library."""
import ctypes
import os

import pytest
import torch

import paper_2609_24089_amd as fb
from paper_2609_24089_amd import ext as fx

ALIGNED, MISALIGNED = 1 << 20, (1 << 20) + 8   # never dereferenced
NPTR = {"fwd_lse": 5, "bwd": 11, "pass1_rows": 16, "pass2_cols": 15}
OPTIONAL = {"bwd": {10}, "pass1_rows": {8}, "pass2_cols": {7, 14}}   # dT; gdT; gdT, Tt
KEYS = {"fwd_lse": {1, 2}, "bwd": {1, 2, 7, 8}, "pass1_rows": {1, 2, 6, 7}, "pass2_cols": {1, 2, 5, 6, 12, 13}}
FNS = sorted(NPTR)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2609_24089_amd.build import build_library
        build_library()
    return fb.load_library()


def bias(table=ALIGNED, buckets=ALIGNED, dtype=fb.BOB_F32, num=32, far=128, lens=0):
    return fb.AttnExt(lens, lens, lens, table, buckets, dtype, num, far)


def call(lib, fn, dtype=fb.BOB_BF16, B=1, H=2, Hkv=1, Nq=16, Nk=20, d=64, scale=0.125, causal=0, ext=None, ptr=ALIGNED,
         bad=None, ws=ALIGNED, nbytes=1 << 50):
    """Optional pointers are NULL here unless `ext` has a bias, whose table they belong to."""
    ptrs = [ctypes.c_void_p(ptr) for _ in range(NPTR[fn])]
    if ext is None or not ext.table:
        for i in OPTIONAL.get(fn, ()):
            ptrs[i] = ctypes.c_void_p(0)
    for i, v in (bad or {}).items():
        ptrs[i] = ctypes.c_void_p(v)
    tail = [ctypes.c_void_p(ws), nbytes]
    return getattr(lib, "attn_ext_" + fn)(dtype, B, H, Hkv, Nq, Nk, d, ctypes.c_float(scale), causal,
                                          None if ext is None else ctypes.byref(ext), *ptrs, *tail, None)


@pytest.mark.parametrize("fn", FNS)
def test_bad_arguments(lib, fn):
    for kw in (dict(Nq=-1), dict(Nk=-1), dict(B=-1), dict(H=-1), dict(d=0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(dtype=5), dict(causal=2), dict(causal=-1), dict(H=4, Hkv=3),
               dict(H=4, Hkv=0), dict(H=4, Hkv=-2), dict(H=2, Hkv=4), dict(Nq=(1 << 30) + 1), dict(Nk=(1 << 30) + 1),
               dict(B=1 << 20, H=1 << 12), dict(B=1 << 10, Nk=1 << 28), dict(H=1 << 16, Hkv=1 << 16),
               dict(ptr=MISALIGNED), dict(ptr=0)):
        assert call(lib, fn, **kw) == fb.BOB_EINVAL, kw
    for kw in (dict(d=96), dict(d=16), dict(dtype=fb.BOB_F32, d=256)):
        assert call(lib, fn, **kw) == fb.BOB_EUNSUPPORTED, kw


@pytest.mark.parametrize("fn", FNS)
def test_bad_bias(lib, fn):
    for e in (bias(buckets=0), bias(dtype=7), bias(num=0), bias(num=(1 << 16) + 1), bias(far=0), bias(far=1025),
              bias(table=ALIGNED + 2), bias(buckets=ALIGNED + 2), bias(lens=ALIGNED + 1),
              bias(table=ALIGNED + 1, dtype=fb.BOB_BF16)):
        assert call(lib, fn, ext=e) == fb.BOB_EINVAL
    # a table's gradient or cotangent without a table, and one off its alignment
    for i in OPTIONAL.get(fn, ()):
        assert call(lib, fn, bad={i: ALIGNED}) == fb.BOB_EINVAL
        assert call(lib, fn, ext=bias(), bad={i: ALIGNED + 2}) == fb.BOB_EINVAL


@pytest.mark.parametrize("fn", FNS)
def test_every_pointer(lib, fn):
    for i in range(NPTR[fn]):
        for v in (0, MISALIGNED):
            if i in OPTIONAL.get(fn, ()):
                continue
            assert call(lib, fn, bad={i: v}) == fb.BOB_EINVAL, (i, v)


@pytest.mark.parametrize("fn", FNS)
def test_empty_problems(lib, fn):
    assert call(lib, fn, B=0, ptr=0, ws=0, nbytes=0) == fb.BOB_OK
    assert call(lib, fn, H=0, Hkv=0, ptr=0, ws=0, nbytes=0) == fb.BOB_OK
    assert call(lib, fn, Nq=0, Nk=0, ptr=0, ws=0, nbytes=0) == fb.BOB_OK
    assert call(lib, fn, B=0, d=80, ptr=0) == fb.BOB_EUNSUPPORTED
    # keys without queries still have gradients to clear, queries without keys an output
    bad = {i: 0 for i in range(NPTR[fn]) if i not in KEYS[fn]}
    if fn in ("bwd", "pass2_cols"):
        assert call(lib, fn, Nq=0, bad={i: 0 for i in KEYS[fn]}) == fb.BOB_EINVAL
    else:
        assert call(lib, fn, Nq=0, bad=bad) == fb.BOB_OK
    if fn != "pass2_cols":
        assert call(lib, fn, Nk=0, bad=bad) == fb.BOB_EINVAL


@pytest.mark.parametrize("fn", ["bwd", "pass2_cols"])
def test_workspace(lib, fn):
    """A bias needs room for the sums by step; with grouped heads also for each query head's part."""
    query = getattr(lib, f"attn_ext_{'bwd' if fn == 'bwd' else 'pass2'}_workspace_bytes")
    e = bias()
    need = query(fb.BOB_BF16, 1, 4, 2, 100, 300, 64, 0, ctypes.byref(e))
    parts = 2 * 2 * 1 * 2 * 300 * 64 * 4
    assert need > parts
    assert query(fb.BOB_BF16, 1, 4, 2, 100, 300, 64, 0, None) == 0
    assert query(fb.BOB_BF16, 1, 4, 3, 100, 300, 64, 0, ctypes.byref(e)) == 0
    kw = dict(H=4, Hkv=2, Nq=100, Nk=300, ext=e)
    for ws, n in ((0, need), (MISALIGNED, need), (ALIGNED, need - 1)):
        assert call(lib, fn, ws=ws, nbytes=n, **kw) == fb.BOB_EINVAL


def mats(Nq=8, Nk=12, H=4, Hkv=2, dtype=torch.bfloat16, B=2, d=64):
    return torch.zeros(B, H, Nq, d, dtype=dtype), torch.zeros(B, Hkv, Nk, d, dtype=dtype)


def test_python_refuses_shapes():
    q, k = mats()
    with pytest.raises(ValueError, match="ROCm device"):
        fb.cross_attention(q, k, k)
    with pytest.raises(ValueError, match="ROCm device"):
        fb.attn_ext_fwd_lse(q, k, k, 0.125)
    with pytest.raises(ValueError, match="must match the query side"):
        fb.cross_attention(q, k[:1], k[:1])
    with pytest.raises(ValueError, match="must match the query side"):
        fb.cross_attention(q, k.float(), k.float())
    with pytest.raises(ValueError, match="multiple of the key/value heads"):
        fb.cross_attention(q, torch.zeros(2, 3, 12, 64, dtype=q.dtype), torch.zeros(2, 3, 12, 64, dtype=q.dtype))
    with pytest.raises(ValueError, match="contiguous"):
        fb.cross_attention(q.transpose(1, 2).contiguous().transpose(1, 2), k, k)
    with pytest.raises(ValueError, match="must be \\[B, H, N, d\\]"):
        fb.cross_attention(q[0], k, k)
    with pytest.raises(ValueError, match="needs a table"):
        fb.biased_attention(q, k, k, None, None)


def on_meta(x):
    return x.to("meta")


def test_python_refuses_lengths_and_tables(monkeypatch):
    """The checks behind the device check, on host tensors with that one check off."""
    monkeypatch.setattr(fx, "_check_mats", lambda *ts: ts[0].shape)
    q, k = mats()
    table, buckets = torch.zeros(32, 4), fb.relative_buckets(32, 128)
    P = lambda **kw: fx._Problem((q,), (k, k), 0.1, False, kw.pop("bias", None), kw.get("kv_lens"),  # noqa: E731
                                 kw.get("q_lens"), kw.get("q_starts"))
    P(bias=(table, buckets), kv_lens=torch.zeros(2, dtype=torch.int32))
    for name in ("kv_lens", "q_lens", "q_starts"):
        for bad in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32),
                    torch.zeros(2, 1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)[::2],
                    on_meta(torch.zeros(2, dtype=torch.int32))):
            with pytest.raises(ValueError, match=name):
                P(**{name: bad})
    with pytest.raises(TypeError, match="table dtype"):
        P(bias=(table.half(), buckets))
    for bad in (torch.zeros(32, 3), torch.zeros(32, 8)[:, ::2], on_meta(table)):
        with pytest.raises(ValueError, match="bias table"):
            P(bias=(bad, buckets))
    with pytest.raises(ValueError, match="bias table"):
        P(bias=(torch.zeros(0, 4), buckets))
    for bad in (buckets.long(), buckets[:-1], buckets[:1], buckets[None], torch.zeros(2051, dtype=torch.int32),
                on_meta(buckets)):
        with pytest.raises(ValueError, match="buckets"):
            P(bias=(table, bad))
    p = P(bias=(table, buckets))
    assert p.cotangent(None) is None
    with pytest.raises(ValueError, match="dtype"):
        p.cotangent(table.bfloat16())
    with pytest.raises(ValueError, match="bias table"):
        p.cotangent(torch.zeros(31, 4))
    with pytest.raises(ValueError, match="needs a bias"):
        P().cotangent(table)
