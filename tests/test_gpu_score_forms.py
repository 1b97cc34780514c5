"""Every launch that the estimate makes of the kernels over capped scores, distance biases and spans, on
the smallest problem whose layout query names it: each block shape and number of wave sets, unsplit and
split into parts, with and without folded rows, a cap and grouped heads, under each mask, for every type
and head dim, row by row against float64 on the first, a middle and the last key/value head."""
import functools

import pytest
import torch

import paper_2609_24089_amd as fb
from tests.parity_util import say
from tests.test_gpu_ext_forms import COLS, DT, FORMS, FWD, KERNELS, OUTS, PASS2, ROWS
from tests.test_gpu_ext_rows import compare_rows
from tests.test_gpu_score import chain

pytestmark = pytest.mark.gpu

CAP = 4.0   # scores of normal queries and keys, about 1: tanh from its straight part to its bend


def built(kernel, dt, d, cap):
    """(rows of a workgroup, wave sets) of every kernel that is built."""
    if (kernel, dt, d) == (COLS, "bf16", 256):
        return {(128, 1), (32, 2), (16, 2)}
    if (kernel, dt, d) == (ROWS, "bf16", 64):
        return {(128, 2), (64, 1), (64, 4), (32, 8), (16, 8)}
    if (kernel, dt, d) == (PASS2, "bf16", 64) and cap:
        return {(64, 2), (64, 1), (32, 4), (16, 4)}
    return set(FORMS[kernel, dt, d])


@functools.cache
def problems(kernel, dt, d, cap):
    """The smallest problem of each launch: {(rows, sets, folded, split, grouped, mask): case}."""
    found = {}
    for mask in ("full", "causal", "spans"):
        for G in (1, 2, 8):
            for Hkv in (1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128):
                for Nq in (1, 3, 16, 24, 70, 101, 200, 301, 523, 777, 1101, 2100, 4099):
                    for Nk in {40, max(Nq, 24), 300, 1500, 5000} if mask == "full" else {Nq}:
                        H = Hkv * G
                        work = H * Nq * Nk * d
                        if H > 512 or work > 6e10 or Nk < 24:
                            continue
                        got = fb.attn_score_layout(kernel, DT[dt], 1, H, Hkv, Nq, Nk, d, mask == "causal", cap, True,
                                                   mask == "spans")
                        key = (got.rows, got.wave_sets, got.folded, got.parts > 1, G > 1, mask)
                        if key not in found or work < found[key][0]:
                            found[key] = (work, dict(B=1, H=H, Hkv=Hkv, Nq=Nq, Nk=Nk, d=d, dtype=dt, cap=cap,
                                                     causal=mask == "causal", mask=mask))
    return {key: c for key, (_, c) in found.items()}


def inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mat = lambda h, n: torch.randn(1, h, n, c["d"], generator=gen, device="cuda").to(DT[c["dtype"]])  # noqa: E731
    q, k = (c["H"], c["Nq"]), (c["Hkv"], c["Nk"])
    x = dict(Q=mat(*q), K=mat(*k), V=mat(*k), dO=mat(*q), UQ=mat(*q), UK=mat(*k), UV=mat(*k))
    lens = lambda n: torch.tensor([n], dtype=torch.int32, device="cuda")  # noqa: E731
    if c["mask"] == "full":
        x.update(kv_lens=lens(c["Nk"] - 3), q_lens=lens(max(1, c["Nq"] - 2)), q_starts=lens(max(0, c["Nk"] // 2 - c["Nq"])))
    if c["mask"] == "spans":
        N = c["Nk"]
        x["documents"] = (torch.arange(N, device="cuda") >= N // 3).long()[None] + 0
        x["documents"][:, N - 1] = -1
        x["prefix_lens"] = lens(N // 5)
    if seed % 2 == 0:
        x["slopes"] = 2.0 ** -torch.arange(1, c["H"] + 1, device="cuda").clamp(max=12).float()
    return x


def head(x, c, h, tau):
    """Every output of query head h in float64 on its valid rows; the key side's are the head's share."""
    n, m = (int(x[k][0]) if k in x else c[s] for k, s in (("q_lens", "Nq"), ("kv_lens", "Nk")))
    start = int(x["q_starts"][0]) if "q_starts" in x else 0
    kh = h // (c["H"] // c["Hkv"])
    q, do, uq = (x[k][0, h, :n].double() for k in ("Q", "dO", "UQ"))
    k, v, uk, uv = (x[k][0, kh, :m].double() for k in ("K", "V", "UK", "UV"))
    by = lambda a, b: torch.mm(a, b.t().contiguous())  # noqa: E731
    of = lambda a, b: torch.mm(a.t().contiguous(), b)  # noqa: E731
    rows, cols = start + torch.arange(n, device="cuda")[:, None], torch.arange(m, device="cuda")[None]
    s = tau * by(q, k)
    cap = c["cap"]
    t = torch.tanh(s / cap) if cap else torch.zeros_like(s)
    u = 1 - t * t
    z, F = cap * t if cap else s, u * tau * (by(uq, k) + by(q, uk))
    if "slopes" in x:
        z = z - x["slopes"][h].double() * (cols - rows).abs()
    valid = torch.ones_like(s, dtype=torch.bool)
    if c["mask"] == "causal":
        valid = cols <= rows
    elif c["mask"] == "spans":
        doc, first = x["documents"][0], torch.tensor([0, c["Nk"] // 3], device="cuda")
        same = (doc[:, None] == doc[None]) & (doc >= 0)[:, None]
        lead = torch.arange(c["Nk"], device="cuda") < first[doc.clamp(min=0)] + int(x["prefix_lens"][0])
        valid = same & ((cols <= rows) | (lead[:, None] & lead[None]))
    L = torch.logsumexp(z.masked_fill(~valid, float("-inf")), 1)
    P = torch.where(valid, torch.exp(z - L[:, None]), 0.0)
    mean = lambda y: (P * y).sum(1, keepdim=True)  # noqa: E731
    dP, C = by(do, v), by(do, uv)
    D, alpha = mean(dP), mean(F)
    dd = dP - D
    dS = P * dd * u
    w = C + F * dd - alpha * dP
    E = mean(w)
    St, Ph = P * (u * (w - E) - (2 / cap * t * dd * F if cap else 0)), P * (F - alpha)
    return dict(O=P @ v, L=L, dQ=tau * dS @ k, D=D[:, 0], dK=tau * of(dS, q), dV=of(P, do), alpha=alpha[:, 0], E=E[:, 0],
                Qt=tau * (St @ k + dS @ uk), dOt=P @ uv + Ph @ v, Kt=tau * (of(St, q) + of(dS, uq)), Vt=of(Ph, do)), n, m


def check(c, names, seed):
    x = inputs(c, seed)
    tau, G = c["d"] ** -0.5, c["H"] // c["Hkv"]
    got = chain(x, dict(c, **{k: True for k in ("documents", "prefix_lens") if k in x}), tau)
    torch.cuda.synchronize()
    for kh in sorted({0, c["Hkv"] // 2, c["Hkv"] - 1}):
        heads = range(kh * G, kh * G + G)
        refs = [head(x, c, h, tau) for h in heads]
        n, m = refs[0][1:]
        part, want = {}, {}
        for name in ("O",) + tuple(k for k in names if k != "O" and k in got):
            values = [r[0][name] for r in refs]
            if name in ("dK", "dV", "Kt", "Vt"):
                part[name], want[name] = got[name][:, kh:kh + 1, :m], sum(values)[None, None]
                assert not got[name][:, kh, m:].any(), name
            else:
                part[name], want[name] = got[name][:, heads, :n], torch.stack(values)[None]
                if name != "L":
                    assert not got[name][:, heads, n:].any(), name
        compare_rows(part, {k: t.cpu().numpy() for k, t in want.items()}, dict(dtype=c["dtype"]), list(want))


@pytest.mark.parametrize("cap", [None, CAP], ids=["plain", "cap"])
@pytest.mark.parametrize("kernel,dt,d", list(FORMS), ids=lambda v: KERNELS[v].replace(" ", "_") if v in range(5) else str(v))
def test_every_launch(kernel, dt, d, cap):
    found = problems(kernel, dt, d, cap)
    forms = {key[:2] for key in found}
    assert forms == built(kernel, dt, d, cap), forms ^ built(kernel, dt, d, cap)
    if kernel == FWD:
        assert any(key[2] for key in found)
    for i, (key, c) in enumerate(sorted(found.items())):
        say(f"[score forms] {KERNELS[kernel]} {dt} d{d} rows {key[0]} sets {key[1]} folded {key[2]} split {key[3]}: {c}")
        check(c, OUTS[kernel], 500 + i)
