"""The two-length kernels row by row: no single row, key or table column of any case may be off
by more than a small multiple of the bar that its whole output keeps (a norm over thousands of
rows does not see one that is lost), and two shapes that the cases lack: fp32 tokens with a
bias, and both backward passes past 2^31 elements.

A row's rounding error is a sum of its own products' errors, each a step of 2^-8 (fp32: of the
bar's 1000 2^-24) of its term, so over its own norm it differs from the whole output's error by
how far the terms' sizes stand from the row's: rows lie within eight times the output's mean of
that ratio, or below the head's mean row norm, which stands in for the norm of rows that cancel.
Heads that are 0 by cancellation in every row (dQ, dK and the like of an entry with one key: P = 1, dP = D) keep the
fp32 rounding of their terms: inner products of d terms of size up to 16, d 2^-20 in all, once an
element on the query side and once a query row on the key side.  A row that was lost or taken from elsewhere is off by its norm: 1 and more, against 8 x 5 x 2^-8."""
import numpy as np
import pytest
import torch

import paper_2609_24089_amd as fb
from oracle import ext_oracle
from tests.parity_util import say
from tests.test_gpu_ext import CASES, SCALARS, TABLES, bar, chain, make, reference

pytestmark = pytest.mark.gpu

WORST = 8


def rows_off(got, want, left=0.0):
    """The largest error of a row of [..., rows, d] over its norm or its head's mean row norm.  Heads
    that cancel in every row: no element above `left`."""
    off, size = np.linalg.norm(got - want, axis=-1), np.linalg.norm(want, axis=-1)
    some = np.maximum((size > 0).sum(-1, keepdims=True), 1)
    mean = np.sqrt((size ** 2).sum(-1, keepdims=True) / some)
    cancels = np.broadcast_to(mean < 1e-9, size.shape)
    assert np.abs(got[cancels]).max(initial=0.0) <= left, np.abs(got[cancels]).max()
    return float((off[~cancels] / np.maximum(size, mean)[~cancels]).max(initial=0.0))


def compare_rows(got, want, c, names):
    errs = {}
    for n in names:
        a, b = got[n].double().cpu().numpy(), want[n]
        assert a.shape == b.shape, n
        if n in SCALARS:
            if n == "L":
                assert np.array_equal(np.isneginf(a), np.isneginf(b))
                a, b = np.where(np.isneginf(a), 0, a), np.where(np.isneginf(b), 0, b)
            size = np.maximum(np.abs(b).max(-1, initial=1.0, keepdims=True), 1.0)
            errs[n] = float((np.abs(a - b) / size).max(initial=0.0))
        elif n in TABLES:
            errs[n] = rows_off(a.T, b.T, want["O"].shape[2] * want["O"].shape[-1] * 2.0 ** -20)
        else:
            terms = want["O"].shape[2] * want["O"].shape[1] // b.shape[1] if n in ("dK", "dV", "Kt", "Vt") else 1
            errs[n] = rows_off(a, b, terms * a.shape[-1] * 2.0 ** -20)
    say("   worst rows", {n: f"{e:.1e}" for n, e in errs.items()})
    for n, e in errs.items():
        assert e <= WORST * bar(n, c.get("dtype"), c.get("table_dtype", "f32")), (n, e)


@pytest.mark.parametrize("name", CASES)
def test_every_row(name):
    c = CASES[name]
    say(f"[ext rows] {name}")
    x = make(c, 61)
    got = chain({n: t.cuda() for n, t in x.items()}, c, c["d"] ** -0.5)
    torch.cuda.synchronize()
    want = reference(x, c, c["d"] ** -0.5)
    compare_rows(got, want, c, list(want))


@pytest.mark.parametrize("case", [
    dict(B=4, H=4, Hkv=4, Nq=1, Nk=500, d=64, q_starts=[499, 3, 0, 250], kv_lens=[500, 4, 1, 251]),
    dict(B=2, H=16, Hkv=2, Nq=1, Nk=300, d=128, q_starts=[299, 100], kv_lens=[300, 101]),
    dict(B=1, H=2, Hkv=2, Nq=1, Nk=6000, d=32, q_starts=[5999]),
    dict(B=3, H=8, Hkv=2, Nq=3, Nk=190, d=64, q_starts=[187, 0, 97], kv_lens=[190, 3, 100]),
], ids=lambda c: f"B{c['B']}H{c['H']}kv{c['Hkv']}Nq{c['Nq']}Nk{c['Nk']}d{c['d']}")
def test_f32_tokens_with_a_bias(case):
    c = dict(case, dtype="f32", bias=(32, 128), causal=True)
    say(f"[ext rows] {c}")
    x = make(c, 62)
    got = chain({n: t.cuda() for n, t in x.items()}, c, c["d"] ** -0.5)
    want = reference(x, c, c["d"] ** -0.5)
    compare_rows(got, want, c, list(want))


@pytest.mark.parametrize("side", ["keys", "queries"])
def test_backward_offsets_past_32_bits(side):
    """More than 2^31 elements on one side: the last entry's gradients and second gradients, whose
    rows lie behind them."""
    B, H, long, short, d = 33, 8, 65536, 40, 128
    assert B * H * long * d > 2 ** 31
    Nq, Nk = (short, long) if side == "keys" else (long, short)
    gen = torch.Generator(device="cuda").manual_seed(63)

    def mat(n):
        t = torch.zeros(B, H, n, d, dtype=torch.bfloat16, device="cuda")
        t[-1] = torch.randn(H, n, d, generator=gen, device="cuda").bfloat16()
        return t

    Q, dO, UQ, K, V, UK, UV = mat(Nq), mat(Nq), mat(Nq), mat(Nk), mat(Nk), mat(Nk), mat(Nk)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[-1] = 700     # the rows that count: the last entry's first 700 on the long side
    o = dict(kv_lens=lens) if side == "keys" else dict(q_lens=lens)
    O, L = fb.attn_ext_fwd_lse(Q, K, V, 0.1, **o)
    dQ, dK, dV, D, _ = fb.attn_ext_bwd(Q, K, V, O, dO, L, 0.1, **o)
    Qt, dOt, alpha, E = fb.attn_ext_pass1_rows(Q, K, V, O, dO, UQ, UK, UV, L, D, dQ, 0.1, **o)
    Kt, Vt, _ = fb.attn_ext_pass2_cols(Q, K, V, dO, UQ, UK, UV, L, D, alpha, E, 0.1, **o)
    n, m = (short, 700) if side == "keys" else (700, short)
    f = {k: t[-1:, :, :r].double().cpu().numpy() for k, t, r in (("Q", Q, n), ("K", K, m), ("V", V, m), ("dO", dO, n),
                                                               ("UQ", UQ, n), ("UK", UK, m), ("UV", UV, m))}
    want = ext_oracle.run(f["Q"], f["K"], f["V"], 0.1, dO=f["dO"], UQ=f["UQ"], UK=f["UK"], UV=f["UV"])
    got = dict(O=O, L=L, dQ=dQ, dK=dK, dV=dV, D=D, Qt=Qt, dOt=dOt, alpha=alpha, E=E, Kt=Kt, Vt=Vt)
    rows = {k: t[-1:, :, :(m if k in ("dK", "dV", "Kt", "Vt") else n)] for k, t in got.items()}
    compare_rows(rows, want, {}, list(want))
    for k, t in got.items():
        r = m if k in ("dK", "dV", "Kt", "Vt") else n
        # the padded rows and the empty entries; summed in pieces of one entry
        assert not any(bool(t[b].any()) for b in range(B - 1)) if k != "L" else torch.isneginf(t[:-1]).all(), k
        assert not t[-1, :, r:].any() if k != "L" else torch.isneginf(t[-1, :, r:]).all(), k
