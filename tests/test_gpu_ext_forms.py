"""Every launch that the two-length kernels' estimate makes, on the smallest problem whose layout
query names it: each block shape and number of wave sets, unsplit and split into parts, with and
without folded rows, a bias and grouped heads, for every type and head dim, row by row against
float64 on the first, a middle and the last key/value head."""
import functools

import pytest
import torch

import paper_2609_24089_amd as fb
from tests.parity_util import say
from tests.test_gpu_ext import chain
from tests.test_gpu_ext_rows import compare_rows

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FWD, ROWS, COLS, PASS1, PASS2 = range(5)
KERNELS = ["forward", "first backward rows", "first backward columns", "pass 1", "pass 2"]
# what each kernel writes; every kernel before it in the path has run in another or the same form
OUTS = {FWD: ("O", "L"), ROWS: ("dQ", "D"), COLS: ("dK", "dV", "dT"), PASS1: ("Qt", "dOt", "alpha", "E"),
        PASS2: ("Kt", "Vt", "Tt")}
# (rows of a workgroup, wave sets) of every kernel that is built
FORMS = {
    (FWD, "bf16", 32): [(128, 2), (128, 1), (64, 4), (32, 8), (16, 16)],
    (FWD, "bf16", 64): [(128, 2), (128, 1), (64, 4), (32, 8), (16, 8)],
    (FWD, "bf16", 128): [(128, 2), (128, 1), (64, 4), (32, 4), (16, 4)],
    (FWD, "bf16", 256): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (FWD, "f32", 32): [(64, 4), (64, 1), (32, 8), (16, 8)],
    (FWD, "f32", 64): [(64, 4), (64, 1), (32, 4), (16, 4)],
    (FWD, "f32", 128): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (ROWS, "bf16", 32): [(128, 2), (128, 1), (64, 4), (32, 8), (16, 16)],
    (ROWS, "bf16", 64): [(128, 2), (128, 1), (64, 4), (32, 8), (16, 8)],
    (ROWS, "bf16", 128): [(128, 2), (128, 1), (64, 4), (32, 4), (16, 4)],
    (ROWS, "bf16", 256): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (ROWS, "f32", 32): [(64, 4), (64, 1), (32, 8), (16, 8)],
    (ROWS, "f32", 64): [(64, 4), (64, 1), (32, 4), (16, 4)],
    (ROWS, "f32", 128): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (COLS, "bf16", 32): [(128, 2), (128, 1), (64, 4), (32, 8), (16, 16)],   # (16, 16) without a bias alone
    (COLS, "bf16", 64): [(128, 2), (128, 1), (64, 4), (32, 8), (16, 8)],
    (COLS, "bf16", 128): [(128, 2), (128, 1), (64, 2), (32, 4), (16, 4)],
    (COLS, "bf16", 256): [(128, 1), (64, 2), (32, 2), (16, 2)],
    (COLS, "f32", 32): [(64, 4), (64, 1), (32, 8), (16, 8)],
    (COLS, "f32", 64): [(64, 2), (64, 1), (32, 4), (16, 4)],
    (COLS, "f32", 128): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (PASS1, "bf16", 32): [(64, 2), (64, 1), (32, 4), (16, 8)],
    (PASS1, "bf16", 64): [(64, 2), (64, 1), (32, 4), (16, 4)],
    (PASS1, "bf16", 128): [(128, 1), (64, 2), (32, 2), (16, 2)],
    (PASS1, "bf16", 256): [(64, 1)],
    (PASS1, "f32", 32): [(64, 2), (64, 1), (32, 4), (16, 4)],
    (PASS1, "f32", 64): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (PASS1, "f32", 128): [(64, 1)],
    (PASS2, "bf16", 32): [(64, 1), (32, 4), (16, 8)],
    (PASS2, "bf16", 64): [(128, 2), (128, 1), (64, 2), (32, 4), (16, 4)],
    (PASS2, "bf16", 128): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (PASS2, "bf16", 256): [(64, 1)],
    (PASS2, "f32", 32): [(64, 2), (64, 1), (32, 4), (16, 4)],
    (PASS2, "f32", 64): [(64, 2), (64, 1), (32, 2), (16, 2)],
    (PASS2, "f32", 128): [(64, 1)],
}


@functools.cache
def problems(kernel, dt, d, bias):
    """The smallest problem of each launch: {(rows, sets, folded, split, grouped): case}."""
    found = {}
    for causal in (False, True):
        for G in (1, 2, 8):
            for Hkv in (1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128):
                for Nq in (1, 3, 16, 24, 70, 101, 200, 301, 523, 777, 1101, 2100, 4099):
                    for Nk in {Nq} if causal else {40, max(Nq, 24), 300, 1500, 5000}:
                        H = Hkv * G
                        work = H * Nq * Nk * d
                        if H > 512 or work > 6e10 or Nk < 24:
                            continue
                        got = fb.attn_ext_layout(kernel, DT[dt], 1, H, Hkv, Nq, Nk, d, causal, bias)
                        # with a bias each query head of a group has a column part of its own in any case
                        whole = G if bias and kernel in (COLS, PASS2) else 1
                        key = (got.rows, got.wave_sets, got.folded, got.parts > whole, G > 1)
                        if key not in found or work < found[key][0]:
                            found[key] = (work, dict(B=1, H=H, Hkv=Hkv, Nq=Nq, Nk=Nk, d=d, dtype=dt, causal=causal))
    return {key: c for key, (_, c) in found.items()}


def inputs(c, bias, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mat = lambda h, n: torch.randn(1, h, n, c["d"], generator=gen, device="cuda").to(DT[c["dtype"]])  # noqa: E731
    q, k = (c["H"], c["Nq"]), (c["Hkv"], c["Nk"])
    x = dict(Q=mat(*q), K=mat(*k), V=mat(*k), dO=mat(*q), UQ=mat(*q), UK=mat(*k), UV=mat(*k))
    lens = lambda n: torch.tensor([n], dtype=torch.int32, device="cuda")  # noqa: E731
    if not c["causal"]:
        x.update(kv_lens=lens(c["Nk"] - 3), q_lens=lens(max(1, c["Nq"] - 2)))
    if bias:
        x.update(table=torch.randn(bias[0], c["H"], generator=gen, device="cuda"),
                 UT=torch.randn(bias[0], c["H"], generator=gen, device="cuda"),
                 buckets=fb.relative_buckets(*bias, bidirectional=not c["causal"], device="cuda"))
        if not c["causal"]:
            x["q_starts"] = lens(max(0, c["Nk"] // 2 - c["Nq"] // 3))
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
    step = torch.arange(m, device="cuda")[None] - (start + torch.arange(n, device="cuda")[:, None])
    S, F = tau * by(q, k), tau * (by(uq, k) + by(q, uk))
    if "table" in x:
        R = (x["buckets"].numel() - 1) // 2
        bucket = x["buckets"].long()[step.clamp(-R, R) + R]
        S, F = S + x["table"][:, h].double()[bucket], F + x["UT"][:, h].double()[bucket]
    if c["causal"]:
        S = S.masked_fill(step > 0, float("-inf"))
    L = torch.logsumexp(S, 1)
    P = torch.exp(S - L[:, None])
    mean = lambda y: (P * y).sum(1, keepdim=True)  # noqa: E731
    dP, C = by(do, v), by(do, uv)
    D, alpha = mean(dP), mean(F)
    dS = P * (dP - D)
    Pt = C + F * (dP - D) - alpha * dP
    E = mean(Pt)
    St, Ph = P * (Pt - E), P * (F - alpha)
    out = dict(O=P @ v, L=L, dQ=tau * dS @ k, D=D[:, 0], dK=tau * of(dS, q), dV=of(P, do), alpha=alpha[:, 0], E=E[:, 0],
               Qt=tau * (St @ k + dS @ uk), dOt=P @ uv + Ph @ v, Kt=tau * (of(St, q) + of(dS, uq)), Vt=of(Ph, do))
    if "table" in x:
        near = step.abs() < R
        for name, t in (("dT", dS), ("Tt", St)):
            sums = torch.zeros(x["table"].shape[0], dtype=torch.float64, device="cuda")
            sums.index_add_(0, bucket[near], t[near])
            sums[x["buckets"][0].long()] += t[step <= -R].sum()
            sums[x["buckets"][-1].long()] += t[step >= R].sum()
            out[name] = sums
    return out, n, m


def check(c, bias, names, seed):
    x = inputs(c, bias, seed)
    tau, G = c["d"] ** -0.5, c["H"] // c["Hkv"]
    got = chain(x, c, tau)
    torch.cuda.synchronize()
    for kh in sorted({0, c["Hkv"] // 2, c["Hkv"] - 1}):
        heads = range(kh * G, kh * G + G)
        refs = [head(x, c, h, tau) for h in heads]
        n, m = refs[0][1:]
        part, want = {}, {}
        for name in ("O",) + tuple(names):
            if name not in got:
                continue
            values = [r[0][name] for r in refs]
            if name in ("dT", "Tt"):
                part[name], want[name] = got[name][:, heads], torch.stack(values, 1)
            elif name in ("dK", "dV", "Kt", "Vt"):
                part[name], want[name] = got[name][:, kh:kh + 1, :m], sum(values)[None, None]
                assert not got[name][:, kh, m:].any(), name
            else:
                part[name], want[name] = got[name][:, heads, :n], torch.stack(values)[None]
                if name != "L":
                    assert not got[name][:, heads, n:].any(), name
        compare_rows(part, {k: t.cpu().numpy() for k, t in want.items()}, dict(dtype=c["dtype"]), list(want))


@pytest.mark.parametrize("bias", [None, (32, 128)], ids=["plain", "bias"])
@pytest.mark.parametrize("kernel,dt,d", list(FORMS), ids=lambda v: KERNELS[v].replace(" ", "_") if v in range(5) else str(v))
def test_every_launch(kernel, dt, d, bias):
    found = problems(kernel, dt, d, bias)
    forms = {key[:2] for key in found}
    built = set(FORMS[kernel, dt, d])
    if (kernel, dt, d) == (COLS, "bf16", 32) and bias:
        built -= {(16, 16)}
    assert forms == built, forms ^ built
    # splits: of column blocks of grouped heads (with a bias beyond the group's heads), of any row
    # blocks, except where a block's sets divide so many tiles that no problem above has parts
    split = {key[4] for key in found if key[3]}
    assert True in split if kernel in (COLS, PASS2) else split or (kernel, dt, d) == (FWD, "bf16", 32), split
    if kernel == FWD:
        assert any(key[2] for key in found)
    for i, (key, c) in enumerate(sorted(found.items())):
        say(f"[ext forms] {KERNELS[kernel]} {dt} d{d} rows {key[0]} sets {key[1]} folded {key[2]} split {key[3]}: {c}")
        check(c, bias, OUTS[kernel], 300 + i)
