"""GPU parity of the attention between sequences of two lengths with a position bias,
against its float64 oracle: every output of the forward, the first backward and the two
BoB passes, at the lengths, masks and head layouts where they can go wrong.

Bars are on ||x - y||_F / ||y||_F per output and count roundings.  bf16 rounds to half a step
of 2^-8: the output itself and one factor of every product that the matrix instructions sum
(P, dS, ...) make two, O enters dQ and dK through D as a third; the second-order outputs sum
up to three such products, one of which cancels against another (five).  fp32 sums up to a
thousand terms in another order: at most 1000 2^-24 = 6e-5 each for the sum and for L.  Row
scalars, L and fp32 tables never leave fp32, also for bf16 matrices, whose products are exact:
they keep the fp32 bar.  alpha and E are sums of terms that cancel, held to that bar of the
terms' size (their row maximum over the problem)."""
import numpy as np
import pytest
import torch

from oracle import ext_oracle
from tests.parity_util import nrel, say

pytestmark = pytest.mark.gpu

BF, F32 = 2.0 ** -8, 1e-4
FIRST = ("O", "dQ", "dK", "dV")
SECOND = ("Qt", "Kt", "Vt", "dOt")
TABLES = ("dT", "Tt")
SCALARS = ("L", "D", "alpha", "E")


def bar(name, dtype, table_dtype):
    if name in SCALARS or (name in TABLES and table_dtype == "f32"):
        return F32
    if name in TABLES:
        return BF
    if dtype == "f32":
        return F32
    return {"O": 2, "dV": 2, "dQ": 3, "dK": 3}.get(name, 5) * BF


# id: B, H, Hkv, Nq, Nk, d, dtype and what else the case has
CASES = {
    # one row and one key, one row and a few, lengths around a tile, every head dim
    "one_pair": dict(B=1, H=1, Hkv=1, Nq=1, Nk=1, d=64),
    "one_query": dict(B=2, H=3, Hkv=3, Nq=1, Nk=77, d=32, kv_lens=[77, 33]),
    "one_key": dict(B=1, H=2, Hkv=1, Nq=70, Nk=1, d=64),
    "tile_edges": dict(B=3, H=2, Hkv=2, Nq=33, Nk=65, d=64, kv_lens=[32, 33, 64], q_lens=[1, 32, 33]),
    "d32": dict(B=1, H=4, Hkv=2, Nq=130, Nk=200, d=32),
    "d128": dict(B=2, H=2, Hkv=1, Nq=101, Nk=257, d=128, kv_lens=[257, 100]),
    "d256": dict(B=1, H=2, Hkv=2, Nq=67, Nk=131, d=256),
    "f32_d32": dict(B=1, H=2, Hkv=1, Nq=40, Nk=90, d=32, dtype="f32"),
    "f32_d64": dict(B=2, H=2, Hkv=2, Nq=65, Nk=129, d=64, dtype="f32", kv_lens=[129, 31], q_lens=[10, 65]),
    "f32_d128": dict(B=1, H=2, Hkv=2, Nq=70, Nk=50, d=128, dtype="f32"),
    # empty entries on either side, and lengths beyond the ends
    "empty_entries": dict(B=4, H=2, Hkv=1, Nq=40, Nk=50, d=64, kv_lens=[0, 50, -3, 99], q_lens=[40, 0, 40, 99]),
    # grids that fill the device: the whole block shapes
    "whole_d64": dict(B=4, H=24, Hkv=12, Nq=300, Nk=420, d=64, kv_lens=[420, 300, 65, 1]),
    "whole_d32_bias": dict(B=4, H=32, Hkv=32, Nq=290, Nk=290, d=32, bias=(32, 128), causal=True),
    "whole_d128_bias": dict(B=3, H=32, Hkv=32, Nq=260, Nk=260, d=128, bias=(32, 128), q_lens=[260, 100, 31],
                            kv_lens=[260, 100, 31]),
    "whole_d256_bias": dict(B=2, H=48, Hkv=48, Nq=200, Nk=200, d=256, bias=(16, 40)),
    "whole_f32_bias": dict(B=2, H=70, Hkv=70, Nq=140, Nk=140, d=64, dtype="f32", bias=(32, 128), causal=True),
    # the bias: one-sided and two-sided, beyond its distance, small and large distances, bf16 tables, grouped heads
    "bias": dict(B=1, H=2, Hkv=2, Nq=150, Nk=150, d=64, bias=(32, 128)),
    "bias_causal": dict(B=2, H=2, Hkv=2, Nq=333, Nk=333, d=64, bias=(32, 128), causal=True),
    "bias_far": dict(B=1, H=1, Hkv=1, Nq=700, Nk=700, d=64, bias=(16, 40)),
    "bias_near_only": dict(B=1, H=2, Hkv=2, Nq=100, Nk=130, d=64, bias=(64, 1024)),
    "bias_distance_2": dict(B=1, H=2, Hkv=2, Nq=200, Nk=150, d=32, bias=(4, 2)),
    "bias_bf16_table": dict(B=1, H=2, Hkv=2, Nq=90, Nk=90, d=128, bias=(32, 128), table_dtype="bf16", causal=True),
    "bias_grouped": dict(B=2, H=8, Hkv=2, Nq=120, Nk=120, d=64, bias=(32, 60), causal=True, q_lens=[120, 50],
                         kv_lens=[120, 50]),
    "bias_f32_grouped": dict(B=1, H=6, Hkv=2, Nq=65, Nk=97, d=32, dtype="f32", bias=(8, 20)),
    "bias_f32_d128": dict(B=1, H=2, Hkv=2, Nq=97, Nk=97, d=128, dtype="f32", bias=(32, 128), causal=True),
    "bias_d256": dict(B=1, H=2, Hkv=1, Nq=70, Nk=99, d=256, bias=(32, 128)),
    # a cache: positions past the first query's, rows before any key
    "cache_token": dict(B=4, H=4, Hkv=4, Nq=1, Nk=500, d=64, bias=(32, 128), causal=True, q_starts=[499, 3, 0, 250],
                        kv_lens=[500, 4, 1, 251]),
    "cache_token_grouped": dict(B=2, H=16, Hkv=2, Nq=1, Nk=300, d=128, bias=(32, 128), causal=True,
                                q_starts=[299, 100], kv_lens=[300, 101]),
    "cache_tokens_grouped": dict(B=2, H=24, Hkv=4, Nq=5, Nk=260, d=64, bias=(32, 100), causal=True,
                                 q_starts=[200, 17], kv_lens=[205, 22]),
    "cache_chunk": dict(B=2, H=2, Hkv=2, Nq=100, Nk=400, d=64, bias=(32, 128), causal=True, q_starts=[300, 40],
                        kv_lens=[400, 140]),
    "cross_tokens_grouped": dict(B=3, H=32, Hkv=4, Nq=3, Nk=190, d=64, kv_lens=[190, 7, 100]),
    "cross_token_grouped_f32": dict(B=2, H=20, Hkv=1, Nq=1, Nk=70, d=64, dtype="f32"),
    # more than 16 rows of a group as one matrix, in blocks of one to four waves a set
    "tokens_16_grouped": dict(B=8, H=32, Hkv=8, Nq=16, Nk=700, d=128, bias=(32, 128), causal=True,
                              q_starts=[684, 500, 31, 0, 3, 600, 64, 255], kv_lens=[700, 516, 47, 16, 19, 616, 80, 271],
                              q_lens=[16, 16, 1, 16, 0, 7, 16, 15]),
    "tokens_11_grouped": dict(B=6, H=30, Hkv=6, Nq=11, Nk=330, d=64, bias=(16, 40), q_starts=[300, 100, 0, 7, 50, 200]),
    "tokens_8_grouped_f32": dict(B=3, H=12, Hkv=3, Nq=8, Nk=200, d=64, dtype="f32", kv_lens=[200, 40, 1]),
    "tokens_12_grouped_d32": dict(B=16, H=64, Hkv=16, Nq=12, Nk=260, d=32),
    "tokens_9_grouped_d256": dict(B=2, H=16, Hkv=4, Nq=9, Nk=130, d=256, bias=(32, 128), q_lens=[9, 4]),
    "tokens_32_grouped": dict(B=3, H=12, Hkv=3, Nq=32, Nk=300, d=64, bias=(64, 90), causal=True, q_starts=[268, 0, 111],
                              kv_lens=[300, 32, 140], q_lens=[32, 32, 29]),
    "rows_33_grouped": dict(B=3, H=12, Hkv=3, Nq=33, Nk=300, d=64, bias=(64, 90), q_starts=[-10, 0, 111]),
    # the largest distance, with folded heads whose tables fit beside the rings and with more
    "far_token_grouped": dict(B=2, H=8, Hkv=2, Nq=1, Nk=1500, d=64, bias=(64, 1024), causal=True,
                              q_starts=[1499, 600], kv_lens=[1500, 601]),
    "far_token_16_heads": dict(B=1, H=32, Hkv=2, Nq=1, Nk=1300, d=128, bias=(64, 1024), causal=True, q_starts=[1299]),
    "far_d256": dict(B=1, H=2, Hkv=1, Nq=1100, Nk=40, d=256, bias=(64, 1024), q_starts=[-600]),
    # ragged batches of up to 64 entries are dealt out by length, larger ones in order
    "entries_64": dict(B=64, H=2, Hkv=2, Nq=40, Nk=70, d=64, kv_lens=[(37 * b) % 71 for b in range(64)],
                       q_lens=[(29 * b) % 41 for b in range(64)]),
    "entries_70": dict(B=70, H=8, Hkv=4, Nq=17, Nk=35, d=32, bias=(8, 20), kv_lens=[(11 * b) % 36 for b in range(70)],
                       q_lens=[(5 * b) % 18 for b in range(70)]),
    "rows_before_keys": dict(B=1, H=2, Hkv=2, Nq=80, Nk=60, d=64, bias=(32, 128), causal=True, q_starts=[-37]),
    "keys_behind": dict(B=1, H=2, Hkv=2, Nq=50, Nk=60, d=64, bias=(32, 128), q_starts=[100000]),
    # few rows against many keys, and few keys against many queries: blocks split over workgroups
    "split_token": dict(B=1, H=2, Hkv=2, Nq=1, Nk=6000, d=64, kv_lens=[5900]),
    "split_tokens_grouped": dict(B=3, H=8, Hkv=1, Nq=4, Nk=5000, d=128, bias=(32, 128), causal=True,
                                 q_starts=[4990, 20, 700], kv_lens=[4994, 24, 704]),
    "split_rows": dict(B=1, H=2, Hkv=1, Nq=40, Nk=5000, d=64),
    "split_rows_ragged": dict(B=3, H=1, Hkv=1, Nq=70, Nk=4100, d=128, kv_lens=[4100, 90, 0], q_lens=[70, 70, 20]),
    "split_rows_chunk": dict(B=2, H=1, Hkv=1, Nq=50, Nk=4000, d=64, bias=(32, 128), causal=True, q_starts=[3950, 0]),
    "split_rows_f32": dict(B=1, H=1, Hkv=1, Nq=33, Nk=3000, d=64, dtype="f32", bias=(32, 128)),
    "split_cols": dict(B=1, H=2, Hkv=2, Nq=6000, Nk=40, d=64, q_lens=[5800]),
    "split_cols_grouped": dict(B=1, H=8, Hkv=2, Nq=1100, Nk=100, d=128),
    "split_cols_bias": dict(B=1, H=4, Hkv=2, Nq=2100, Nk=64, d=32, bias=(32, 128)),
    "causal_no_bias": dict(B=2, H=2, Hkv=1, Nq=70, Nk=150, d=64, causal=True, q_starts=[80, 0]),
}


def make(c, seed):
    rng = np.random.default_rng(seed)
    dt = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    q = lambda: torch.tensor(rng.standard_normal((c["B"], c["H"], c["Nq"], c["d"])), dtype=torch.float32).to(dt)  # noqa: E731
    k = lambda: torch.tensor(rng.standard_normal((c["B"], c["Hkv"], c["Nk"], c["d"])), dtype=torch.float32).to(dt)  # noqa: E731
    x = dict(Q=q(), K=k(), V=k(), dO=q(), UQ=q(), UK=k(), UV=k())
    if "bias" in c:
        import paper_2609_24089_amd as fb
        num, far = c["bias"]
        tt = torch.bfloat16 if c.get("table_dtype") == "bf16" else torch.float32
        t = lambda: torch.tensor(rng.standard_normal((num, c["H"])), dtype=torch.float32).to(tt)  # noqa: E731
        x.update(table=t(), UT=t(), buckets=fb.relative_buckets(num, far, bidirectional=not c.get("causal", False)))
    for n in ("q_lens", "kv_lens", "q_starts"):
        if n in c:
            x[n] = torch.tensor(c[n], dtype=torch.int32)
    return x


def reference(x, c, tau, second=True):
    f = {n: t.double().numpy() if t.is_floating_point() else t.numpy() for n, t in x.items()}
    u = {n: f[n] for n in ("UQ", "UK", "UV", "UT") if n in f} if second else {}
    return ext_oracle.run(f["Q"], f["K"], f["V"], tau, causal=c.get("causal", False), table=f.get("table"),
                          buckets=f.get("buckets"), q_lens=f.get("q_lens"), kv_lens=f.get("kv_lens"),
                          q_starts=f.get("q_starts"), dO=f["dO"], **u)


def options(xd, c):
    return dict(causal=c.get("causal", False), bias=(xd["table"], xd["buckets"]) if "table" in xd else None,
                kv_lens=xd.get("kv_lens"), q_lens=xd.get("q_lens"), q_starts=xd.get("q_starts"))


def chain(xd, c, tau):
    """The four calls one by one."""
    import paper_2609_24089_amd as fb
    o = options(xd, c)
    Q, K, V, dO, U = xd["Q"], xd["K"], xd["V"], xd["dO"], [xd[n] for n in ("UQ", "UK", "UV")]
    O, L = fb.attn_ext_fwd_lse(Q, K, V, tau, **o)
    dQ, dK, dV, D, dT = fb.attn_ext_bwd(Q, K, V, O, dO, L, tau, **o)
    gT = xd.get("UT")
    Qt, dOt, alpha, E = fb.attn_ext_pass1_rows(Q, K, V, O, dO, *U, L, D, dQ, tau, gdT=gT, **o)
    Kt, Vt, Tt = fb.attn_ext_pass2_cols(Q, K, V, dO, *U, L, D, alpha, E, tau, gdT=gT, **o)
    out = dict(O=O, L=L, dQ=dQ, dK=dK, dV=dV, D=D, Qt=Qt, dOt=dOt, alpha=alpha, E=E, Kt=Kt, Vt=Vt)
    if dT is not None:
        out.update(dT=dT, Tt=Tt)
    return out


def compare(got, want, c, names):
    errs = {}
    for n in names:
        a, b = got[n].double().cpu().numpy(), want[n]
        assert a.shape == b.shape, n
        if n == "L":
            assert np.array_equal(np.isneginf(a), np.isneginf(b)), n
            a, b = np.where(np.isneginf(a), 0, a), np.where(np.isneginf(b), 0, b)
        assert np.all(np.isfinite(a)), n
        # what is 0 by cancellation (Qt of a row of one key: S~ = P (Pt - E) with P = 1, Pt = E)
        # keeps the fp32 rounding of its terms, inner products of d terms of size up to 16:
        # d 2^-20.  Empty and padded rows are exactly 0 (test_padding_is_never_read).
        assert np.abs(a[b == 0]).max(initial=0.0) <= c["d"] * 2.0 ** -20, n
        if n in ("alpha", "E", "D"):
            errs[n] = np.abs(a - b).max(initial=0.0) / max(np.abs(b).max(initial=0.0), 1.0)
        else:
            errs[n] = nrel(a, b) if np.linalg.norm(b) > 1e-12 else float(np.linalg.norm(a))
    say("   errs", {n: f"{e:.1e}" for n, e in errs.items()})
    for n, e in errs.items():
        assert e <= bar(n, c.get("dtype"), c.get("table_dtype", "f32")), (n, e)


@pytest.mark.parametrize("name", [n for n in CASES if n.startswith("split_")])
def test_split_cases_are_split(name):
    """The cases above need a workspace, without a bias for the parts' sums alone."""
    import ctypes
    import paper_2609_24089_amd as fb
    c = CASES[name]
    lib = fb.load_library()
    table = 1 << 20 if "bias" in c else 0
    e = fb.AttnExt(None, None, None, table, table, fb.BOB_F32, *c.get("bias", (0, 0)))
    args = (fb.BOB_F32 if c.get("dtype") == "f32" else fb.BOB_BF16, c["B"], c["H"], c["Hkv"], c["Nq"], c["Nk"], c["d"],
            int(c.get("causal", False)), ctypes.byref(e))
    n = {k: getattr(lib, f"attn_ext_{k}_workspace_bytes")(*args) for k in ("fwd", "bwd", "pass1", "pass2")}
    say("   bytes", n)
    if "cols" in name:
        assert n["pass2"] >= 2 * 2 * c["B"] * c["Hkv"] * c["Nk"] * c["d"] * 4
    if "token" in name:
        assert n["fwd"] >= 2 * c["B"] * c["H"] * c["Nq"] * c["d"] * 4
    if "rows" in name:
        assert n["pass1"] >= 2 * 3 * c["B"] * c["H"] * c["Nq"] * c["d"] * 4


@pytest.mark.parametrize("name", CASES)
def test_every_output(name):
    c = CASES[name]
    say(f"[ext] {name} {c}")
    x = make(c, 11)
    tau = c["d"] ** -0.5
    xd = {n: t.cuda() for n, t in x.items()}
    got = chain(xd, c, tau)
    torch.cuda.synchronize()
    want = reference(x, c, tau)
    compare(got, want, c, [n for n in want])


# ---------------------------------------------------------------------------
# The differentiable layers
# ---------------------------------------------------------------------------
def layer(xd, c, tau, q, k, v, table):
    import paper_2609_24089_amd as fb
    if "bias" in c:
        return fb.biased_attention(q, k, v, table, xd["buckets"], tau, causal=c.get("causal", False),
                                   kv_lens=xd.get("kv_lens"), q_lens=xd.get("q_lens"), q_starts=xd.get("q_starts"))
    return fb.cross_attention(q, k, v, tau, kv_lens=xd.get("kv_lens"), q_lens=xd.get("q_lens"))


def differentiate(xd, c, tau, fn=layer):
    """The layer's output, its gradients and the gradients of their product with the directions."""
    q, k, v, dO = (xd[n].clone().requires_grad_(True) for n in ("Q", "K", "V", "dO"))
    leaves = [q, k, v] + ([xd["table"].clone().requires_grad_(True)] if "bias" in c else [])
    O = fn(xd, c, tau, q, k, v, leaves[3] if "bias" in c else None)
    g = torch.autograd.grad(O, leaves, dO, create_graph=True)
    u = [xd[n] for n in ("UQ", "UK", "UV", "UT") if n in xd]
    h = torch.autograd.grad(g, [*leaves, dO], u)
    names = ["O", "dQ", "dK", "dV"] + ["dT"] * ("bias" in c) + ["Qt", "Kt", "Vt"] + ["Tt"] * ("bias" in c) + ["dOt"]
    return dict(zip(names, [t.detach() for t in (O, *g, *h)]))


LAYERS = ["split_rows_ragged", "split_cols_grouped", "split_cols_bias", "tile_edges", "f32_d64", "empty_entries", "bias_causal", "bias_grouped", "bias_bf16_table", "cache_chunk",
          "cross_tokens_grouped", "cache_tokens_grouped"]


@pytest.mark.parametrize("name", LAYERS)
def test_layers_equal_the_calls(name):
    """Bit for bit, through the native functions and through the Python ones."""
    import paper_2609_24089_amd as fb
    from paper_2609_24089_amd import ext
    c = CASES[name]
    xd = {n: t.cuda() for n, t in make(c, 12).items()}
    want = chain(xd, c, 0.15)
    got = differentiate(xd, c, 0.15)

    def in_python(xd, c, tau, q, k, v, table):
        return ext._ExtFn.apply(q, k, v, table, xd.get("buckets"), xd.get("kv_lens"), xd.get("q_lens"),
                                xd.get("q_starts"), tau, c.get("causal", False))

    slow = differentiate(xd, c, 0.15, in_python)
    for n, t in got.items():
        assert torch.equal(t, want[n]), n
        assert torch.equal(slow[n], want[n]), n
    with torch.no_grad():
        assert torch.equal(layer(xd, c, 0.15, xd["Q"], xd["K"], xd["V"], xd.get("table")), want["O"])
    again = chain(xd, c, 0.15)  # no atomics: the same bits twice
    for n, t in want.items():
        assert torch.equal(again[n], t), n
    # into outputs of the caller's, on a stream of the caller's: the calls without the native path
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, w = options(xd, c), {n: torch.empty_like(t) for n, t in want.items()}
    Q, K, V, dO, U = xd["Q"], xd["K"], xd["V"], xd["dO"], [xd[n] for n in ("UQ", "UK", "UV")]
    put = lambda *names: tuple(w.get(n) for n in names)  # noqa: E731
    torch.cuda.synchronize()
    fb.attn_ext_fwd_lse(Q, K, V, 0.15, out=put("O", "L"), stream=s, **o)
    fb.attn_ext_bwd(Q, K, V, w["O"], dO, w["L"], 0.15, out=put("dQ", "dK", "dV", "D", "dT"), stream=s, **o)
    fb.attn_ext_pass1_rows(Q, K, V, w["O"], dO, *U, w["L"], w["D"], w["dQ"], 0.15, gdT=xd.get("UT"),
                           out=put("Qt", "dOt", "alpha", "E"), stream=s, **o)
    fb.attn_ext_pass2_cols(Q, K, V, dO, *U, w["L"], w["D"], w["alpha"], w["E"], 0.15, gdT=xd.get("UT"),
                           out=put("Kt", "Vt", "Tt"), stream=s, **o)
    s.synchronize()
    for n, t in w.items():
        assert torch.equal(t, want[n]), n


def test_partial_gradients():
    """Some inputs without a gradient, a frozen table, and a table alone."""
    c = CASES["bias_grouped"]
    xd = {n: t.cuda() for n, t in make(c, 13).items()}
    want = chain(xd, c, 0.125)
    k = xd["K"].clone().requires_grad_(True)
    O = layer(xd, c, 0.125, xd["Q"], k, xd["V"], xd["table"])
    (g,) = torch.autograd.grad(O, k, xd["dO"], create_graph=True)
    assert torch.equal(g, want["dK"])
    (h,) = torch.autograd.grad(g, k, xd["UK"])
    zero = {**xd, "UQ": torch.zeros_like(xd["UQ"]), "UV": torch.zeros_like(xd["UV"]),
            "UT": torch.zeros_like(xd["UT"])}
    assert torch.equal(h, chain(zero, c, 0.125)["Kt"])
    t = xd["table"].clone().requires_grad_(True)
    O = layer(xd, c, 0.125, xd["Q"], xd["K"], xd["V"], t)
    (g,) = torch.autograd.grad(O, t, xd["dO"], create_graph=True)
    assert torch.equal(g, want["dT"])
    (h,) = torch.autograd.grad(g, t, xd["UT"])
    zero = {**xd, **{n: torch.zeros_like(xd[n]) for n in ("UQ", "UK", "UV")}}
    assert torch.equal(h, chain(zero, c, 0.125)["Tt"])


@pytest.mark.parametrize("name", ["tile_edges", "bias_grouped"])
def test_third_derivatives_are_refused(name):
    """The second gradients may be asked for with a graph; their own are refused, through the
    native functions and through the Python ones."""
    from paper_2609_24089_amd import ext
    c = CASES[name]
    xd = {n: t.cuda() for n, t in make(c, 14).items()}
    want = chain(xd, c, 0.125)

    def in_python(xd, c, tau, q, k, v, table):
        return ext._ExtFn.apply(q, k, v, table, xd.get("buckets"), xd.get("kv_lens"), xd.get("q_lens"),
                                xd.get("q_starts"), tau, c.get("causal", False))

    for fn in (layer, in_python):
        q, k, v = (xd[n].clone().requires_grad_(True) for n in ("Q", "K", "V"))
        leaves = [q, k, v] + ([xd["table"].clone().requires_grad_(True)] if "bias" in c else [])
        O = fn(xd, c, 0.125, q, k, v, leaves[3] if "bias" in c else None)
        g = torch.autograd.grad(O, leaves, xd["dO"], create_graph=True)
        u = [xd[n] for n in ("UQ", "UK", "UV", "UT") if n in xd]
        h = torch.autograd.grad(g, leaves, u, create_graph=True)
        for n, t in zip(("Qt", "Kt", "Vt", "Tt"), h):
            assert torch.equal(t, want[n]), n
            with pytest.raises(NotImplementedError, match="third derivatives"):
                torch.autograd.grad(t.float().square().sum(), leaves, retain_graph=True, allow_unused=True)


def test_two_streams_at_once():
    """The whole path on two streams at a time, each with its own inputs and workspaces."""
    jobs = []
    for name in ("split_cols_bias", "bias_grouped"):
        c = CASES[name]
        xd = {n: t.cuda() for n, t in make(c, 15).items()}
        jobs.append((c, xd, chain(xd, c, 0.125), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (c, xd, _, s) in enumerate(jobs):
            with torch.cuda.stream(s):
                got[i].append(chain(xd, c, 0.125))
    torch.cuda.synchronize()
    for runs, (_, _, want, _) in zip(got, jobs):
        for run in runs:
            for n, t in want.items():
                assert torch.equal(run[n], t), n


def test_gradient_against_differences():
    """The fp32 layer's gradients in every input against central differences of its output in
    float64 sums: with steps of 2^-7 the third-order term is about 1e-4 of the slope."""
    c = dict(B=1, H=2, Hkv=2, Nq=40, Nk=50, d=32, dtype="f32", bias=(8, 12))
    xd = {n: t.cuda() for n, t in make(c, 14).items()}
    w = xd["dO"].double()
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = chain(xd, c, 0.2)
    for name, out in (("Q", "dQ"), ("K", "dK"), ("V", "dV"), ("table", "dT")):
        u = torch.randn(xd[name].shape, generator=gen, device="cuda")
        ends = []
        for step in (2.0 ** -7, -2.0 ** -7):
            y = {**xd, name: xd[name] + step * u}
            O = layer(y, c, 0.2, y["Q"], y["K"], y["V"], y["table"])
            ends.append(float((O.double() * w).sum()))
        slope, exact = (ends[0] - ends[1]) * 2.0 ** 6, float((g[out].double() * u.double()).sum())
        say(f"   {name}: {slope:.6f} {exact:.6f}")
        assert abs(slope - exact) <= 2e-3 * max(1.0, abs(exact)), name


# ---------------------------------------------------------------------------
# Padding, masks, memory
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("name", ["split_rows_ragged", "split_cols", "split_tokens_grouped", "tile_edges", "empty_entries", "whole_d128_bias", "bias_grouped", "cache_chunk",
                                  "cross_tokens_grouped", "cache_token_grouped"])
def test_padding_is_never_read(name):
    """NaN and infinities in padded rows and keys change no output, and padded rows, padded
    keys and empty entries get exact zeros."""
    c = CASES[name]
    x = make(c, 15)
    xd = {n: t.cuda() for n, t in x.items()}
    ql = [min(max(n, 0), c["Nq"]) for n in c.get("q_lens", [c["Nq"]] * c["B"])]
    kl = [min(max(n, 0), c["Nk"]) for n in c.get("kv_lens", [c["Nk"]] * c["B"])]
    dirty = {n: t.clone() for n, t in xd.items()}
    for b in range(c["B"]):
        for n in ("Q", "dO", "UQ"):
            dirty[n][b, :, ql[b]:] = float("nan")
        for i, n in enumerate(("K", "V", "UK", "UV")):
            dirty[n][b, :, kl[b]:] = float("inf") if i % 2 else float("nan")
    want, got = chain(xd, c, 0.125), chain(dirty, c, 0.125)
    for n, t in want.items():
        assert torch.equal(got[n], t), n
    for b in range(c["B"]):
        for n in ("O", "dQ", "Qt", "dOt", "D", "alpha", "E"):
            assert not got[n][b, :, ql[b]:].any(), n
        for n in ("dK", "dV", "Kt", "Vt"):
            assert not got[n][b, :, kl[b]:].any(), n
        assert torch.isneginf(got["L"][b, :, ql[b]:]).all()


@pytest.mark.parametrize("low", [float("-inf"), torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min, -1e30])
def test_masked_buckets(low):
    """Table entries of the lowest values mask their keys; a row that sees nothing else is
    empty.  Causal with the buckets of steps 0..2 masked, the first three rows are."""
    c = dict(B=1, H=2, Hkv=2, Nq=100, Nk=100, d=64, bias=(8, 12), causal=True)
    x = make(c, 16)
    x["table"][:3, 1] = low          # head 1 alone: one-sided buckets 0, 1, 2 are steps 0, -1, -2
    want = reference(x, c, 0.125)
    xd = {n: t.cuda() for n, t in x.items()}
    got = chain(xd, c, 0.125)
    assert torch.isneginf(got["L"][0, 1, :3]).all() and not got["O"][0, 1, :3].any()
    assert not got["dT"][:3, 1].any() and not got["Tt"][:3, 1].any()
    compare(got, want, c, list(want))


def test_buckets_and_lengths_beyond_their_range():
    """Buckets outside 0..num_buckets - 1 count as the nearer end, also in the gradients."""
    c = dict(B=1, H=2, Hkv=2, Nq=70, Nk=70, d=64, bias=(8, 12))
    x = make(c, 17)
    x["buckets"][3], x["buckets"][-2] = -5, 1000
    want = reference(x, c, 0.125)
    got = chain({n: t.cuda() for n, t in x.items()}, c, 0.125)
    compare(got, want, c, list(want))


def test_no_queries_and_no_keys():
    import paper_2609_24089_amd as fb
    for Nq, Nk in ((0, 40), (30, 0), (0, 0)):
        c = dict(B=2, H=4, Hkv=2, Nq=Nq, Nk=Nk, d=64, bias=(8, 12))
        got = chain({n: t.cuda() for n, t in make(c, 18).items()}, c, 0.125)
        for n, t in got.items():
            assert torch.isneginf(t).all() if n == "L" else not t.any(), n
    c = dict(B=0, H=4, Hkv=2, Nq=5, Nk=6, d=64, bias=(8, 12))
    got = chain({n: t.cuda() for n, t in make(c, 18).items()}, c, 0.125)
    assert got["dT"].shape == (8, 4) and not got["dT"].any() and got["O"].shape == (0, 4, 5, 64)
    q, k = torch.zeros(2, 0, 5, 64, device="cuda"), torch.zeros(2, 0, 6, 64, device="cuda")
    assert fb.cross_attention(q, k, k).shape == q.shape


def test_extreme_scores():
    """Scores that grow late by hundreds (the forward's reference moves), tiny and huge ones,
    and a zero scale, against the oracle."""
    for tau, grow in ((0.125, 40.0), (0.0, 1.0), (30.0, 1.0)):
        c = dict(B=1, H=2, Hkv=2, Nq=90, Nk=400, d=64, bias=(8, 12))
        x = make(c, 19)
        ramp = torch.linspace(-grow, grow, 400)[:, None] if grow != 1.0 else 1.0
        x["K"] = (x["K"].float() * 0.1 + 0.05 * ramp).to(x["K"].dtype) if grow != 1.0 else x["K"]
        want = reference(x, c, tau, second=False)
        import paper_2609_24089_amd as fb
        xd = {n: t.cuda() for n, t in x.items()}
        o = options(xd, c)
        O, L = fb.attn_ext_fwd_lse(xd["Q"], xd["K"], xd["V"], tau, **o)
        assert nrel(O.double().cpu().numpy(), want["O"]) <= 2 * BF
        # L is relative to scores of size up to ~|tau| 8 * 64 * 5
        assert nrel(L.double().cpu().numpy(), want["L"]) <= 1e-5


def test_offsets_past_32_bits():
    """A key/value cache of more than 2^31 elements: the last entry's last keys."""
    import paper_2609_24089_amd as fb
    B, H, Nk, d = 33, 8, 65536, 128
    assert B * H * Nk * d > 2 ** 31
    k = torch.zeros(B, H, Nk, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    gen = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn(B, H, 1, d, generator=gen, device="cuda").bfloat16()
    n = 700
    k[-1, :, -n:] = torch.randn(H, n, d, generator=gen, device="cuda").bfloat16()
    v[-1, :, -n:] = torch.randn(H, n, d, generator=gen, device="cuda").bfloat16()
    k[-1, :, :-n] = 0
    starts = torch.full((B,), Nk - 1, dtype=torch.int32, device="cuda")
    lens = torch.full((B,), 1, dtype=torch.int32, device="cuda")
    lens[-1] = Nk
    table = torch.randn(32, H, generator=gen, device="cuda")
    buckets = fb.relative_buckets(32, 128, bidirectional=False, device="cuda")
    O = fb.biased_attention(q, k, v, table, buckets, 0.1, causal=True, kv_lens=lens, q_starts=starts)
    # the zero keys share the far bucket's score
    kt, vt = k[-1, :, -n:].double(), v[-1, :, -n:].double()
    step = torch.arange(Nk - n, Nk, device="cuda") - (Nk - 1)
    bias = table[buckets[step.clamp(-128, 128) + 128].long()].double().T
    S = 0.1 * (kt @ q[-1, :, 0].double()[:, :, None])[:, :, 0] + bias
    rest = table[31].double()
    top = torch.maximum(S.amax(1), rest)
    W = torch.exp(S - top[:, None])
    want = (W[:, :, None] * vt).sum(1) / (W.sum(1) + (Nk - n) * torch.exp(rest - top))[:, None]
    assert nrel(O[-1, :, 0].double().cpu().numpy(), want.cpu().numpy()) <= 2 * BF
    assert not O[:-1].any()


def test_two_captured_graphs_and_eager_calls_between():
    """A decoding step and a training step captured, replayed in turn on changing inputs with
    eager work between; each replay equals the eager result bit for bit."""
    ct, cg = CASES["cache_token"], CASES["bias_grouped"]
    xt = {n: t.cuda() for n, t in make(ct, 20).items()}
    xg = {n: t.cuda() for n, t in make(cg, 21).items()}

    def token():
        with torch.no_grad():
            return layer(xt, ct, 0.125, xt["Q"], xt["K"], xt["V"], xt["table"])

    leaves = [xg[n].requires_grad_(True) for n in ("Q", "K", "V", "table")]

    def train():
        O = layer(xg, cg, 0.125, *leaves[:3], leaves[3])
        return (O, *torch.autograd.grad(O, leaves, xg["dO"]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token(), train()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for fn in (token, train):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = fn()
        graphs.append(g)
        outs.append(o if isinstance(o, tuple) else (o,))
    gen = torch.Generator(device="cuda").manual_seed(5)
    for r in range(4):
        with torch.no_grad():
            for t in (xt["Q"], xt["K"], xg["Q"], xg["V"], xg["dO"]):
                t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
            xt["q_starts"].copy_(torch.tensor([499 - r, 3, r, 250], dtype=torch.int32))
        for g, o, fn in ((graphs[r % 2], outs[r % 2], (token, train)[r % 2]),
                         (graphs[1 - r % 2], outs[1 - r % 2], (token, train)[1 - r % 2])):
            g.replay()
            want = fn()
            torch.cuda.synchronize()
            for a, b in zip(o, want if isinstance(want, tuple) else (want,)):
                assert torch.equal(a, b), r


def test_an_encoder_decoder_step():
    """The operators as a model uses them: a padded encoder with a two-sided bias, a causal
    decoder with a one-sided one that attends to the encoder's states, a loss, its gradients
    and a Hessian-vector product; and the decoder's last token again from caches, which equals
    the whole pass's last row up to the rounding of its probabilities."""
    import paper_2609_24089_amd as fb
    torch.manual_seed(0)
    B, H, S, T, d = 2, 4, 70, 33, 64
    lens = torch.tensor([70, 41], dtype=torch.int32, device="cuda")
    w = {n: (torch.randn(d, d, device="cuda") / 8).requires_grad_(True)
         for n in ("eq", "ek", "ev", "dq", "dk", "dv", "cq", "ck", "cv")}
    te, td = (torch.randn(32, H, device="cuda", requires_grad=True) for _ in range(2))
    be, bd = fb.relative_buckets(32, 40, True, "cuda"), fb.relative_buckets(32, 40, False, "cuda")
    src, tgt = torch.randn(B, H, S, d, device="cuda"), torch.randn(B, H, T, d, device="cuda")

    def model():
        e = src + fb.biased_attention(src @ w["eq"], src @ w["ek"], src @ w["ev"], te, be, kv_lens=lens, q_lens=lens)
        s = tgt + fb.biased_attention(tgt @ w["dq"], tgt @ w["dk"], tgt @ w["dv"], td, bd, causal=True)
        y = s + fb.cross_attention(s @ w["cq"], e @ w["ck"], e @ w["cv"], kv_lens=lens)
        return e, s, y

    params = [*w.values(), te, td]
    e, s, y = model()
    loss = 0.5 * (y * y).mean()
    g = torch.autograd.grad(loss, params, create_graph=True)
    dirs = [torch.randn_like(p) for p in params]
    hv = torch.autograd.grad(sum((a * b).sum() for a, b in zip(g, dirs)), params)
    assert all(torch.isfinite(t).all() for t in (*g, *hv))
    # the same model with torch operations in float64.  The fp32 model rounds each of its ten
    # products and sums at 2^-24 of terms that cancel by at most a hundred: 1e-4
    def plain(q, k, v, table, buckets, causal, n):
        step = torch.arange(k.shape[2], device="cuda")[None] - torch.arange(q.shape[2], device="cuda")[:, None]
        S = q @ k.transpose(-1, -2) * d ** -0.5
        if table is not None:
            S = S + table[buckets[step.clamp(-40, 40) + 40].long()].permute(2, 0, 1)
        bad = torch.arange(k.shape[2], device="cuda") >= (lens if n else torch.full_like(lens, 10 ** 6))[:, None, None, None]
        bad = bad | (step > 0) if causal else bad.expand(S.shape)
        return torch.softmax(S.masked_fill(bad, float("-inf")), -1) @ v

    wide = [p.detach().double().requires_grad_(True) for p in params]
    W = dict(zip(w, wide))
    rows = (torch.arange(S, device="cuda") < lens[:, None])[:, None, :, None]
    src64, tgt64 = src.double(), tgt.double()
    e64 = src64 + rows * plain(src64 @ W["eq"], src64 @ W["ek"], src64 @ W["ev"], wide[-2], be, False, True)
    s64 = tgt64 + plain(tgt64 @ W["dq"], tgt64 @ W["dk"], tgt64 @ W["dv"], wide[-1], bd, True, False)
    y64 = s64 + plain(s64 @ W["cq"], e64 @ W["ck"], e64 @ W["cv"], None, None, False, True)
    g64 = torch.autograd.grad(0.5 * (y64 * y64).mean(), wide, create_graph=True)
    hv64 = torch.autograd.grad(sum((x * u.double()).sum() for x, u in zip(g64, dirs)), wide)
    errs = [float((x.double() - x64).norm() / x64.norm()) for x, x64 in zip((*g, *hv), (*g64, *hv64))]
    say("   gradients and products", [f"{x:.0e}" for x in errs])
    assert max(errs) <= 1e-4
    with torch.no_grad():
        last = torch.full((B,), T - 1, dtype=torch.int32, device="cuda")
        one = tgt[:, :, -1:].contiguous()
        s1 = one + fb.biased_attention(one @ w["dq"], tgt @ w["dk"], tgt @ w["dv"], td, bd, causal=True, q_starts=last)
        y1 = s1 + fb.cross_attention(s1 @ w["cq"], e @ w["ck"], e @ w["cv"], kv_lens=lens)
        assert nrel(y1.double().cpu().numpy(), y[:, :, -1:].detach().double().cpu().numpy()) <= 2e-5
