"""Refusals of the attention over capped scores, distance biases and spans, with no GPU: the C calls
check everything before any HIP call, the Python ones before the library.  And the spans that
attention_spans makes, against the masks that they stand for."""
import ctypes
import os

import pytest
import torch

import paper_2609_24089_amd as fb
from paper_2609_24089_amd import ext as fx
from paper_2609_24089_amd import score as fs

ALIGNED, MISALIGNED = 1 << 20, (1 << 20) + 8   # never dereferenced
NPTR = {"fwd_lse": 6, "bwd": 11, "pass1_rows": 16, "pass2_cols": 13}
REST = {"fwd_lse": 4, "bwd": 4, "pass1_rows": 4}
KEYS = {"fwd_lse": {1, 2}, "bwd": {1, 2, 8, 9}, "pass1_rows": {1, 2, 7, 8}, "pass2_cols": {1, 2, 5, 6, 11, 12}}
FNS = sorted(NPTR)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2609_24089_amd.build import build_library
        build_library()
    return fb.load_library()


def options(lens=0, spans=0, slopes=0, cap=0.0):
    return fs.AttnScore(lens, lens, lens, spans, slopes, cap)


def call(lib, fn, dtype=fb.BOB_BF16, B=1, H=2, Hkv=1, Nq=16, Nk=20, d=64, scale=0.125, causal=0, score=None, ptr=ALIGNED,
         bad=None, ws=ALIGNED, nbytes=1 << 50):
    ptrs = [ctypes.c_void_p(ptr) for _ in range(NPTR[fn])]
    for i, v in (bad or {}).items():
        ptrs[i] = ctypes.c_void_p(v)
    return getattr(lib, "attn_score_" + fn)(dtype, B, H, Hkv, Nq, Nk, d, ctypes.c_float(scale), causal,
                                            None if score is None else ctypes.byref(score), *ptrs, ctypes.c_void_p(ws),
                                            nbytes, None)


@pytest.mark.parametrize("fn", FNS)
def test_bad_arguments(lib, fn):
    for kw in (dict(Nq=-1), dict(Nk=-1), dict(B=-1), dict(H=-1), dict(d=0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(dtype=5), dict(causal=2), dict(causal=-1), dict(H=4, Hkv=3),
               dict(H=4, Hkv=0), dict(H=2, Hkv=4), dict(Nq=(1 << 30) + 1), dict(Nk=(1 << 30) + 1),
               dict(B=1 << 20, H=1 << 12), dict(ptr=MISALIGNED), dict(ptr=0)):
        assert call(lib, fn, **kw) == fb.BOB_EINVAL, kw
    for kw in (dict(d=96), dict(d=16), dict(dtype=fb.BOB_F32, d=256)):
        assert call(lib, fn, **kw) == fb.BOB_EUNSUPPORTED, kw


@pytest.mark.parametrize("fn", FNS)
def test_bad_options(lib, fn):
    for s in (options(lens=ALIGNED + 1), options(spans=MISALIGNED), options(slopes=ALIGNED + 2), options(cap=-1.0),
              options(cap=float("nan")), options(cap=float("inf")), options(cap=9e-7), options(cap=1.1e6)):
        assert call(lib, fn, score=s) == fb.BOB_EINVAL, (s.spans, s.slopes, s.cap)
    assert call(lib, fn, score=options(spans=ALIGNED), causal=1) == fb.BOB_EINVAL
    assert call(lib, fn, score=options(cap=1.0), scale=1.1e6) == fb.BOB_EINVAL
    # more query heads that share a key/value head than their slopes have room for
    assert call(lib, fn, H=1025, Hkv=1, score=options(slopes=ALIGNED)) == fb.BOB_EINVAL


@pytest.mark.parametrize("fn", FNS)
def test_every_pointer(lib, fn):
    for i in range(NPTR[fn]):
        assert call(lib, fn, bad={i: MISALIGNED}) == fb.BOB_EINVAL, i
        if i != REST.get(fn):
            assert call(lib, fn, bad={i: 0}) == fb.BOB_EINVAL, i


@pytest.mark.parametrize("fn", FNS)
def test_empty_problems(lib, fn):
    for s in (None, options(ALIGNED, ALIGNED, ALIGNED, 30.0)):
        assert call(lib, fn, B=0, ptr=0, ws=0, nbytes=0, score=s) == fb.BOB_OK
        assert call(lib, fn, H=0, Hkv=0, ptr=0, ws=0, nbytes=0, score=s) == fb.BOB_OK
        assert call(lib, fn, Nq=0, Nk=0, ptr=0, ws=0, nbytes=0, score=s) == fb.BOB_OK
    assert call(lib, fn, B=0, d=80, ptr=0) == fb.BOB_EUNSUPPORTED
    # keys without queries still have gradients to clear, queries without keys an output
    bad = {i: 0 for i in range(NPTR[fn]) if i not in KEYS[fn]}
    if fn in ("bwd", "pass2_cols"):
        assert call(lib, fn, Nq=0, bad={i: 0 for i in KEYS[fn]}) == fb.BOB_EINVAL
    else:
        assert call(lib, fn, Nq=0, bad=bad) == fb.BOB_OK
    if fn != "pass2_cols":
        assert call(lib, fn, Nk=0, bad=bad) == fb.BOB_EINVAL


def test_workspace_and_layout_without_a_device(lib):
    got = fb.ext.AttnExtLaunch()
    ask = lambda kernel, s=None, **kw: lib.attn_score_layout(  # noqa: E731
        kernel, kw.get("dtype", fb.BOB_BF16), 1, 2, 1, 16, 20, kw.get("d", 64), 0, s and ctypes.byref(s),
        ctypes.byref(got))
    for kernel in (-1, 5):
        assert ask(kernel) == fb.BOB_EINVAL
    assert ask(0, d=80) == fb.BOB_EUNSUPPORTED
    assert ask(0, options(cap=-1.0)) == fb.BOB_EINVAL
    size = lambda which, H=2, Hkv=1, s=None: lib.attn_score_workspace_bytes(  # noqa: E731
        which, fb.BOB_BF16, 1, H, Hkv, 16, 20, 64, 0, s and ctypes.byref(s))
    for which in (-1, 4):
        assert size(which) == 0
    for which in range(4):
        assert size(which, H=4, Hkv=3) == 0 and size(which, s=options(cap=-1.0)) == 0


def mats(Nq=8, Nk=12, H=4, Hkv=2, dtype=torch.bfloat16, B=2, d=64):
    return torch.zeros(B, H, Nq, d, dtype=dtype), torch.zeros(B, Hkv, Nk, d, dtype=dtype)


def test_python_refuses_shapes():
    q, k = mats()
    with pytest.raises(ValueError, match="ROCm device"):
        fb.scored_attention(q, k, k)
    with pytest.raises(ValueError, match="ROCm device"):
        fb.attn_score_fwd_lse(q, k, k, 0.125)
    with pytest.raises(ValueError, match="must match the query side"):
        fb.scored_attention(q, k[:1], k[:1])
    with pytest.raises(ValueError, match="must match the query side"):
        fb.scored_attention(q, k.float(), k.float())
    with pytest.raises(ValueError, match="multiple of the key/value heads"):
        fb.scored_attention(q, torch.zeros(2, 3, 12, 64, dtype=q.dtype), torch.zeros(2, 3, 12, 64, dtype=q.dtype))
    with pytest.raises(ValueError, match="contiguous"):
        fb.scored_attention(q.transpose(1, 2).contiguous().transpose(1, 2), k, k)


def test_python_refuses_options(monkeypatch):
    """The checks behind the device check, on host tensors with that one check off."""
    monkeypatch.setattr(fx, "_check_mats", lambda *ts: ts[0].shape)
    q, k = mats()

    def problem(causal=False, cap=None, slopes=None, spans=None, kv_lens=None):
        return fs._Score((q,), (k, k), 0.1, causal, cap, slopes, spans, kv_lens, None, None)

    slopes, spans = torch.zeros(4), fb.attention_spans(2, 12)
    problem(cap=30, slopes=slopes, spans=spans, kv_lens=torch.zeros(2, dtype=torch.int32))
    for cap in (0, -1, 1e7, 1e-7, float("nan"), float("inf")):
        with pytest.raises(ValueError, match="cap"):
            problem(cap=cap)
    for bad in (torch.zeros(2), torch.zeros(4, dtype=torch.bfloat16), torch.zeros(4, 1), torch.zeros(8)[::2],
                torch.zeros(4, device="meta"), torch.zeros(4, requires_grad=True)):
        with pytest.raises(ValueError, match="slopes"):
            problem(slopes=bad)
    for bad in (spans.long(), spans[:1], spans[:, :8], spans[..., :2], spans.transpose(0, 1).contiguous().transpose(0, 1),
                spans.to("meta")):
        with pytest.raises(ValueError, match="spans"):
            problem(spans=bad)
    with pytest.raises(ValueError, match="causal"):
        problem(causal=True, spans=spans)


def seen(spans, keys_of_queries):
    """bool [B, N query positions, N key positions] from one of the two sides of spans."""
    B, N, _ = spans.shape
    at = torch.arange(N)
    if keys_of_queries:
        return (at >= spans[:, :, 0:1]) & (at < spans[:, :, 1:2])
    return ((at >= spans[:, :, 2:3]) & (at < spans[:, :, 3:4])).transpose(1, 2)


@pytest.mark.parametrize("seed", range(6))
def test_spans_tell_one_mask(seed):
    gen = torch.Generator().manual_seed(seed)
    B, N = 3, (1, 2, 7, 33, 64, 100)[seed]
    docs = torch.repeat_interleave(torch.randint(-1, 5, (B, N), generator=gen), torch.randint(1, 9, (N,), generator=gen),
                                   dim=1)[:, :N]
    prefix = torch.randint(-2, N + 3, (B, N), generator=gen)
    for documents, lens in ((None, None), (docs, None), (None, prefix[:, 0]), (docs, prefix), (docs.int(), prefix[:, 0])):
        spans = fb.attention_spans(B, N, documents, lens)
        assert spans.dtype == torch.int32 and spans.is_contiguous() and tuple(spans.shape) == (B, N, 4)
        want = torch.zeros(B, N, N, dtype=torch.bool)
        for b in range(B):
            first = 0
            while first < N:
                end = first + 1
                while end < N and (documents is None or documents[b, end] == documents[b, first]):
                    end += 1
                if documents is None or documents[b, first] >= 0:
                    n = 0 if lens is None else int(lens[b] if lens.dim() == 1 else lens[b, first])
                    for i in range(first, end):
                        for j in range(first, end):
                            want[b, i, j] = j <= i or (i < first + n and j < first + n)
                first = end
        assert torch.equal(seen(spans, True), want)
        assert torch.equal(seen(spans, False), want)


def test_spans_refuse():
    for kw in (dict(documents=torch.zeros(2, 7, dtype=torch.int32)), dict(documents=torch.zeros(2, 8)),
               dict(prefix_lens=torch.zeros(3, dtype=torch.int32)), dict(prefix_lens=torch.zeros(2))):
        with pytest.raises(ValueError):
            fb.attention_spans(2, 8, **kw)
    with pytest.raises(ValueError):
        fb.attention_spans(-1, 8)
    assert tuple(fb.attention_spans(0, 5).shape) == (0, 5, 4) and tuple(fb.attention_spans(2, 0).shape) == (2, 0, 4)
