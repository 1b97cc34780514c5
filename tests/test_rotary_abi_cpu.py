"""Refusals of the normalised, rotated heads, with no GPU: the C calls check everything before any
HIP call, the Python ones before the library.  And the frequencies that rotary_frequencies makes."""
import ctypes
import os

import pytest
import torch

import paper_2609_24089_amd as fb
from paper_2609_24089_amd import rotary as fr

ALIGNED, MISALIGNED = 1 << 20, (1 << 20) + 8   # never dereferenced
FNS = ("fwd", "bwd", "bwd2")
# tensors of head vectors, those that may be NULL without a weight, and those that always may
HEADS = {"fwd": 4, "bwd": 6, "bwd2": 10}
WEIGHTED = {"fwd": (), "bwd": (0, 1), "bwd2": (0, 1, 2, 3, 6, 7)}
OPTIONAL = {"fwd": (), "bwd": (), "bwd2": (4, 5)}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2609_24089_amd.build import build_library
        build_library()
    return fb.load_library()


def rotary(positions=ALIGNED, freqs=ALIGNED, axes=None, num_axes=1, pairs=16, interleaved=0, wq=None, wk=None,
           weight_dtype=fb.BOB_F32, eps=1e-6):
    return fr.AttnRotary(positions, freqs, axes, num_axes, pairs, interleaved, wq, wk, weight_dtype, eps)


def call(lib, fn, dtype=fb.BOB_BF16, B=1, H=2, Hkv=1, N=16, d=64, rot="default", heads=None, grads=(None, None),
         cots=(None, None), ws=ALIGNED, nbytes=1 << 50, inverse=0):
    """heads: {index: attn_heads or None} in the place of good ones."""
    r = rotary() if rot == "default" else rot
    hs = [fr.AttnHeads(ALIGNED, 1 << 12, 64, 128) for _ in range(HEADS[fn])]
    for i, h in (heads or {}).items():
        hs[i] = h
    hs = [None if h is None else ctypes.byref(h) for h in hs]
    vp = ctypes.c_void_p
    args = [dtype, B, H, Hkv, N, d] + ([inverse] if fn == "fwd" else []) + [None if r is None else ctypes.byref(r)]
    if fn == "fwd":
        return lib.attn_rotary_fwd(*args, *hs, None)
    tail = [vp(g) for g in grads] + [vp(ws), nbytes, None]
    if fn == "bwd":
        return lib.attn_rotary_bwd(*args, *hs, *tail)
    return lib.attn_rotary_bwd2(*args, *hs[:6], *[vp(c) for c in cots], *hs[6:], *tail)


NORMS = dict(wq=ALIGNED, wk=ALIGNED)


@pytest.mark.parametrize("fn", FNS)
def test_bad_arguments(lib, fn):
    for kw in (dict(B=-1), dict(H=-1), dict(Hkv=-1), dict(N=-1), dict(dtype=5), dict(rot=None), dict(H=65535, Hkv=1),
               dict(N=(1 << 30) + 1), dict(B=1 << 16, N=(1 << 15) + 1)):
        assert call(lib, fn, **kw) == fb.BOB_EINVAL, kw
    for kw in (dict(d=0), dict(d=48), dict(d=512)):
        assert call(lib, fn, **kw) == fb.BOB_EUNSUPPORTED, kw


@pytest.mark.parametrize("fn", FNS)
def test_bad_rotary(lib, fn):
    for r in (rotary(pairs=-8), rotary(pairs=12), rotary(pairs=40), rotary(interleaved=2), rotary(num_axes=0),
              rotary(num_axes=2), rotary(positions=None), rotary(freqs=None), rotary(positions=ALIGNED + 2),
              rotary(freqs=ALIGNED + 4), rotary(axes=ALIGNED + 2), rotary(weight_dtype=7, **NORMS),
              rotary(wq=MISALIGNED), rotary(wk=MISALIGNED), rotary(eps=-1e-9, **NORMS),
              rotary(eps=float("nan"), **NORMS), rotary(eps=float("inf"), **NORMS)):
        assert call(lib, fn, rot=r) == fb.BOB_EINVAL
    if fn == "fwd":  # back only where that is the inverse
        assert call(lib, fn, inverse=1, rot=rotary(**NORMS)) == fb.BOB_EINVAL
        assert call(lib, fn, inverse=2) == fb.BOB_EINVAL


@pytest.mark.parametrize("dtype", [fb.BOB_BF16, fb.BOB_F32])
@pytest.mark.parametrize("fn", FNS)
def test_every_tensor(lib, fn, dtype):
    unit = 8 if dtype == fb.BOB_BF16 else 4
    for i in range(HEADS[fn]):
        for bad in (fr.AttnHeads(MISALIGNED, 1 << 12, 64, 128), fr.AttnHeads(ALIGNED, (1 << 12) + unit // 2, 64, 128),
                    fr.AttnHeads(ALIGNED, 1 << 12, 64 + unit // 2, 128), fr.AttnHeads(ALIGNED, 1 << 12, 64, 128 - unit // 2)):
            assert call(lib, fn, dtype=dtype, heads={i: bad}, rot=rotary(**NORMS)) == fb.BOB_EINVAL, i
        if i not in OPTIONAL[fn]:
            for none in (None, fr.AttnHeads(None, 0, 0, 0)):
                assert call(lib, fn, dtype=dtype, heads={i: none}, rot=rotary(**NORMS)) == fb.BOB_EINVAL, i
                if i not in WEIGHTED[fn]:
                    assert call(lib, fn, dtype=dtype, heads={i: none}) == fb.BOB_EINVAL, i


@pytest.mark.parametrize("fn", ["bwd", "bwd2"])
def test_weights_gradients(lib, fn):
    need = lib.attn_rotary_workspace_bytes(fb.BOB_BF16, 1, 2, 1, 16, 64, ctypes.byref(rotary(**NORMS)))
    assert need > 0
    assert lib.attn_rotary_workspace_bytes(fb.BOB_BF16, 1, 2, 1, 16, 64, ctypes.byref(rotary())) == 0
    assert lib.attn_rotary_workspace_bytes(fb.BOB_BF16, 1, 2, 1, 16, 48, ctypes.byref(rotary(**NORMS))) == 0
    kw = dict(rot=rotary(**NORMS), grads=(ALIGNED, ALIGNED))
    for ws, n in ((0, need), (MISALIGNED, need), (ALIGNED, need - 1)):
        assert call(lib, fn, ws=ws, nbytes=n, **kw) == fb.BOB_EINVAL
    # a gradient without a weight, or off its type's alignment
    for i in range(2):
        grads = [None, None]
        grads[i] = ALIGNED
        assert call(lib, fn, grads=grads) == fb.BOB_EINVAL
        grads[i] = ALIGNED + 2
        assert call(lib, fn, rot=rotary(**NORMS), grads=grads) == fb.BOB_EINVAL
        if fn == "bwd2":
            cots = [None, None]
            cots[i] = ALIGNED
            assert call(lib, fn, cots=cots) == fb.BOB_EINVAL
            cots[i] = MISALIGNED
            assert call(lib, fn, rot=rotary(**NORMS), cots=cots) == fb.BOB_EINVAL


@pytest.mark.parametrize("fn", FNS)
def test_empty_problems(lib, fn):
    none = {i: None for i in range(HEADS[fn])}
    for kw in (dict(B=0), dict(N=0), dict(H=0, Hkv=0)):
        assert call(lib, fn, heads=none, **kw) == fb.BOB_OK
        assert call(lib, fn, heads=none, rot=rotary(None, None), **kw) == fb.BOB_OK
    assert call(lib, fn, B=0, d=48, heads=none) == fb.BOB_EUNSUPPORTED


def heads(H=4, Hkv=2, B=2, N=8, d=64, dtype=torch.bfloat16):
    return torch.zeros(B, H, N, d, dtype=dtype), torch.zeros(B, Hkv, N, d, dtype=dtype)


def test_python_refuses():
    q, k = heads()
    pos, rot = torch.zeros(2, 8, dtype=torch.int32), fb.rotary_frequencies(64)
    with pytest.raises(ValueError, match="ROCm device"):
        fb.rotate_heads(q, k, pos, rot)
    with pytest.raises(ValueError, match="must match the queries"):
        fb.rotate_heads(q, k[:1], pos, rot)
    with pytest.raises(ValueError, match="must match the queries"):
        fb.rotate_heads(q, k.float(), pos, rot)
    with pytest.raises(ValueError, match="\\[B, H, N, d\\]"):
        fb.rotate_heads(q[0], k, pos, rot)
    with pytest.raises(ValueError, match="head dim"):
        fb.rotate_heads(q[..., :48], k[..., :48], pos, rot)


def test_frequencies():
    freqs, axes = fb.rotary_frequencies(64)
    want = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    assert freqs.dtype == torch.float64 and (freqs / want - 1).abs().max() < 1e-14
    assert axes.dtype == torch.int32 and int(axes.sum()) == 0
    freqs, axes = fb.rotary_frequencies(128, 1e6, (16, 24, 24))
    assert (freqs / 1e6 ** (-torch.arange(64, dtype=torch.float64) / 64) - 1).abs().max() < 1e-14
    assert axes.tolist() == [0] * 16 + [1] * 24 + [2] * 24
    freqs, axes = fb.rotary_frequencies(64, 100.0, (16, 16), apart=True)
    one = 100.0 ** (-torch.arange(16, dtype=torch.float64) / 16)
    assert (freqs / torch.cat([one, one]) - 1).abs().max() < 1e-14
    for args in ((0,), (24,), (-16,), (64, 0.0), (64, float("nan")), (64, 1e4, (16, 15)), (64, 1e4, (40, -8))):
        with pytest.raises(ValueError):
            fb.rotary_frequencies(*args)
