"""GPU parity of the attention over capped scores, distance biases and masks by document and prefix, against its
float64 oracle: every output of the forward, the first backward and the two BoB passes, at the lengths, masks and head
layouts where they can go wrong.

Bars are on ||x - y||_F / ||y||_F per output and count roundings, as those of the two-length calls: bf16 rounds to half
a step of 2^-8, the output itself and one factor of every product that the matrix instructions sum (P, dS, ...) make two,
O enters dQ and dK through D as a third; the second-order outputs sum up to three such products, one of which cancels
against another (five).  The cap adds no rounding to bf16: its factor 1 - tanh^2 goes into those operands before they are
rounded, and its tanh is off by 2^-23 of 1, a score of up to c = 50 by 6e-6.  fp32 sums up to a thousand terms in another
order: at most 1000 2^-24 = 6e-5 each for the sum and for L.  Row scalars and L never leave fp32, also for bf16 matrices.
alpha, E and D are sums of terms that cancel, held to that bar of the terms' size (their row maximum over the
problem)."""
import numpy as np
import pytest
import torch

from oracle import score_oracle
from tests.parity_util import nrel, say

pytestmark = pytest.mark.gpu

BF, F32 = 2.0 ** -8, 1e-4
SCALARS = ("L", "D", "alpha", "E")


def bar(name, dtype):
    if name in SCALARS or dtype == "f32":
        return F32
    return {"O": 2, "dV": 2, "dQ": 3, "dK": 3}.get(name, 5) * BF


def docs(*rows):
    """[B, N] documents from lengths; a negative length is padding."""
    out = []
    for lens in rows:
        out.append(sum(([-1] * -n if n < 0 else [i] * n for i, n in enumerate(lens)), []))
    return out


# id: B, H, Hkv, Nq, Nk, d, dtype and what else the case has
CASES = {
    # one row and one key, one row and a few, lengths around a tile, every head dim
    "one_pair": dict(B=1, H=1, Hkv=1, Nq=1, Nk=1, d=64, cap=5.0),
    "one_query": dict(B=2, H=3, Hkv=3, Nq=1, Nk=77, d=32, kv_lens=[77, 33], cap=2.0, slopes=True),
    "one_key": dict(B=1, H=2, Hkv=1, Nq=70, Nk=1, d=64, cap=2.0),
    "tile_edges": dict(B=3, H=2, Hkv=2, Nq=33, Nk=65, d=64, kv_lens=[32, 33, 64], q_lens=[1, 32, 33], slopes=True),
    "cap_d32": dict(B=1, H=4, Hkv=2, Nq=130, Nk=200, d=32, cap=3.0),
    "cap_d64": dict(B=2, H=4, Hkv=2, Nq=150, Nk=150, d=64, cap=1.0, causal=True),
    "cap_d128": dict(B=2, H=2, Hkv=1, Nq=101, Nk=257, d=128, kv_lens=[257, 100], cap=2.0),
    "cap_d256": dict(B=1, H=2, Hkv=2, Nq=67, Nk=131, d=256, cap=2.0, slopes=True),
    "plain": dict(B=1, H=2, Hkv=2, Nq=90, Nk=100, d=64),
    "loud": dict(B=1, H=2, Hkv=2, Nq=200, Nk=200, d=64, cap=20.0, causal=True, loud=20.0),
    "loud_f32": dict(B=1, H=2, Hkv=2, Nq=100, Nk=100, d=64, cap=5.0, causal=True, loud=10.0, dtype="f32"),
    "slopes_two_sided": dict(B=1, H=4, Hkv=4, Nq=150, Nk=170, d=64, slopes=True),
    "slopes_causal": dict(B=2, H=6, Hkv=2, Nq=333, Nk=333, d=64, slopes=True, causal=True),
    "slopes_d128": dict(B=1, H=4, Hkv=4, Nq=160, Nk=160, d=128, slopes=True, causal=True),
    "f32_d32": dict(B=1, H=2, Hkv=1, Nq=40, Nk=90, d=32, dtype="f32", cap=2.0),
    "f32_d64": dict(B=2, H=2, Hkv=2, Nq=65, Nk=129, d=64, dtype="f32", kv_lens=[129, 31], q_lens=[10, 65], slopes=True),
    "f32_d128": dict(B=1, H=2, Hkv=2, Nq=70, Nk=50, d=128, dtype="f32", cap=4.0, slopes=True),
    "f32_documents": dict(B=2, H=2, Hkv=1, Nq=97, Nk=97, d=64, dtype="f32", documents=docs([40, 57], [1, 95, 1]), cap=2.0),
    # empty entries on either side, and lengths beyond the ends
    "empty_entries": dict(B=4, H=2, Hkv=1, Nq=40, Nk=50, d=64, kv_lens=[0, 50, -3, 99], q_lens=[40, 0, 40, 99], cap=3.0),
    # documents: inside a tile, across tiles, single positions, padding in front, between and behind
    "documents": dict(B=2, H=2, Hkv=2, Nq=150, Nk=150, d=64, documents=docs([70, 30, 50], [-5, 3, 32, -10, 64, 1, -35])),
    "documents_cap": dict(B=2, H=4, Hkv=2, Nq=200, Nk=200, d=64, documents=docs([31, 1, 33, 64, 71], [200]), cap=2.0,
                          slopes=True),
    "documents_d128": dict(B=1, H=3, Hkv=3, Nq=260, Nk=260, d=128, documents=docs([100, 32, 65, 3, -60]), slopes=True),
    "documents_single": dict(B=1, H=2, Hkv=1, Nq=70, Nk=70, d=64, documents=docs([1] * 70), cap=2.0),
    "documents_none": dict(B=2, H=2, Hkv=1, Nq=70, Nk=70, d=64, documents=docs([-70], [-30, 40]), cap=2.0),
    "documents_prefix": dict(B=2, H=2, Hkv=2, Nq=210, Nk=210, d=64, documents=docs([90, 40, 80], [5, 10, 195]),
                             prefix_lens=[35, 8], cap=3.0),
    "documents_lens": dict(B=2, H=2, Hkv=1, Nq=100, Nk=100, d=32, documents=docs([60, 40], [20, 80]), kv_lens=[77, 100],
                           q_lens=[100, 33]),
    "prefix": dict(B=3, H=2, Hkv=2, Nq=180, Nk=180, d=64, prefix_lens=[70, 0, 500], kv_lens=[180, 100, 33],
                   q_lens=[180, 100, 33]),
    "prefix_d256": dict(B=1, H=2, Hkv=1, Nq=99, Nk=99, d=256, prefix_lens=[40], cap=2.0),
    # a cache: positions past the first query's, rows before any key, rows without a span
    "cache_token": dict(B=4, H=4, Hkv=4, Nq=1, Nk=500, d=64, causal=True, q_starts=[499, 3, 0, 250],
                        kv_lens=[500, 4, 1, 251], cap=2.0, slopes=True),
    "cache_token_grouped": dict(B=2, H=16, Hkv=2, Nq=1, Nk=300, d=128, causal=True, q_starts=[299, 100],
                                kv_lens=[300, 101], cap=3.0, slopes=True),
    "cache_tokens_grouped": dict(B=2, H=24, Hkv=4, Nq=5, Nk=260, d=64, causal=True, q_starts=[200, 17],
                                 kv_lens=[205, 22], slopes=True),
    "cache_chunk": dict(B=2, H=2, Hkv=2, Nq=100, Nk=400, d=64, causal=True, q_starts=[300, 40], kv_lens=[400, 140],
                        cap=2.0),
    "cache_documents": dict(B=2, H=4, Hkv=2, Nq=7, Nk=200, d=64, documents=docs([50, 150], [180, 20]),
                            q_starts=[193, 178], kv_lens=[200, 185], cap=2.0),
    "cache_spans_outside": dict(B=2, H=2, Hkv=1, Nq=40, Nk=60, d=64, documents=docs([30, 30], [60]), q_starts=[-9, 45]),
    "rows_before_keys": dict(B=1, H=2, Hkv=2, Nq=80, Nk=60, d=64, causal=True, q_starts=[-37], slopes=True),
    "tokens_16_grouped": dict(B=8, H=32, Hkv=8, Nq=16, Nk=700, d=128, slopes=True, causal=True,
                              q_starts=[684, 500, 31, 0, 3, 600, 64, 255], kv_lens=[700, 516, 47, 16, 19, 616, 80, 271],
                              q_lens=[16, 16, 1, 16, 0, 7, 16, 15]),
    "tokens_32_grouped": dict(B=3, H=12, Hkv=3, Nq=32, Nk=300, d=64, cap=2.0, causal=True, q_starts=[268, 0, 111],
                              kv_lens=[300, 32, 140], q_lens=[32, 32, 29]),
    # grids that fill the device: the whole block shapes
    "whole_d64": dict(B=4, H=24, Hkv=12, Nq=420, Nk=420, d=64, kv_lens=[420, 300, 65, 1], q_lens=[420, 300, 65, 1], cap=2.0,
                      causal=True),
    "whole_d32_slopes": dict(B=4, H=32, Hkv=32, Nq=290, Nk=290, d=32, slopes=True, causal=True, cap=4.0),
    "whole_d64_documents": dict(B=3, H=32, Hkv=32, Nq=300, Nk=300, d=64,
                                documents=docs([100, 28, 1, 71, 100], [300], [-40, 5, 200, -55]), slopes=True),
    "whole_d128_documents": dict(B=3, H=32, Hkv=32, Nq=260, Nk=260, d=128,
                                 documents=docs([100, 28, 1, 31, 100], [260], [-40, 5, 200, -15])),
    "whole_d128_cap": dict(B=3, H=32, Hkv=16, Nq=260, Nk=260, d=128, cap=2.0, causal=True),
    "whole_d256_cap": dict(B=2, H=48, Hkv=48, Nq=200, Nk=200, d=256, cap=2.0, slopes=True),
    "whole_f32": dict(B=2, H=70, Hkv=70, Nq=140, Nk=140, d=64, dtype="f32", cap=3.0, slopes=True, causal=True),
    # few rows against many keys, and few keys against many queries: blocks split over workgroups
    "split_token": dict(B=1, H=2, Hkv=2, Nq=1, Nk=6000, d=64, kv_lens=[5900], cap=2.0),
    "split_rows": dict(B=1, H=2, Hkv=1, Nq=40, Nk=5000, d=64, cap=2.0, slopes=True),
    "split_rows_documents": dict(B=1, H=1, Hkv=1, Nq=60, Nk=4000, d=128, q_starts=[3940],
                                 documents=docs([1500, 2400, 64, 31, 5])),
    "split_cols": dict(B=1, H=2, Hkv=2, Nq=6000, Nk=40, d=64, q_lens=[5800], cap=2.0),
    "split_cols_grouped": dict(B=1, H=8, Hkv=2, Nq=1100, Nk=100, d=128, slopes=True),
    "entries_64": dict(B=64, H=2, Hkv=2, Nq=40, Nk=70, d=64, kv_lens=[(37 * b) % 71 for b in range(64)],
                       q_lens=[(29 * b) % 41 for b in range(64)], cap=2.0),
}
LISTS = ("q_lens", "kv_lens", "q_starts", "documents", "prefix_lens")


def make(c, seed):
    rng = np.random.default_rng(seed)
    dt = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    q = lambda by=1.0: torch.tensor(rng.standard_normal((c["B"], c["H"], c["Nq"], c["d"])) * by, dtype=torch.float32).to(dt)  # noqa: E731
    k = lambda: torch.tensor(rng.standard_normal((c["B"], c["Hkv"], c["Nk"], c["d"])), dtype=torch.float32).to(dt)  # noqa: E731
    x = dict(Q=q(c.get("loud", 1.0)), K=k(), V=k(), dO=q(), UQ=q(), UK=k(), UV=k())
    for n in LISTS:
        if n in c:
            x[n] = torch.tensor(c[n], dtype=torch.int32)
    if c.get("slopes"):
        x["slopes"] = torch.tensor([2.0 ** -(1 + 6 * h / c["H"]) for h in range(c["H"])], dtype=torch.float32)
    return x


def reference(x, c, tau, second=True):
    f = {n: t.double().numpy() if t.is_floating_point() else t.numpy() for n, t in x.items()}
    u = {n: f[n] for n in ("UQ", "UK", "UV")} if second else {}
    return score_oracle.run(f["Q"], f["K"], f["V"], tau, causal=c.get("causal", False), cap=c.get("cap"),
                            slopes=f.get("slopes"), dO=f["dO"], **{n: f.get(n) for n in LISTS}, **u)


def options(xd, c):
    import paper_2609_24089_amd as fb
    spans = None
    if "documents" in c or "prefix_lens" in c:
        spans = fb.attention_spans(c["B"], c["Nk"], xd.get("documents"), xd.get("prefix_lens"))
    return dict(causal=c.get("causal", False), cap=c.get("cap"), slopes=xd.get("slopes"), spans=spans,
                kv_lens=xd.get("kv_lens"), q_lens=xd.get("q_lens"), q_starts=xd.get("q_starts"))


def chain(xd, c, tau):
    """The four calls one by one."""
    import paper_2609_24089_amd as fb
    o = options(xd, c)
    Q, K, V, dO, U = xd["Q"], xd["K"], xd["V"], xd["dO"], [xd[n] for n in ("UQ", "UK", "UV")]
    O, Orest, L = fb.attn_score_fwd_lse(Q, K, V, tau, want_rest=Q.dtype == torch.bfloat16, **o)
    dQ, dK, dV, D = fb.attn_score_bwd(Q, K, V, O, Orest, dO, L, tau, **o)
    Qt, dOt, alpha, E = fb.attn_score_pass1_rows(Q, K, V, O, Orest, dO, *U, L, D, dQ, tau, **o)
    Kt, Vt = fb.attn_score_pass2_cols(Q, K, V, dO, *U, L, D, alpha, E, tau, **o)
    return dict(O=O, L=L, dQ=dQ, dK=dK, dV=dV, D=D, Qt=Qt, dOt=dOt, alpha=alpha, E=E, Kt=Kt, Vt=Vt)


def compare(got, want, c, names):
    errs = {}
    for n in names:
        a, b = got[n].double().cpu().numpy(), want[n]
        assert a.shape == b.shape, n
        if n == "L":
            assert np.array_equal(np.isneginf(a), np.isneginf(b)), n
            a, b = np.where(np.isneginf(a), 0, a), np.where(np.isneginf(b), 0, b)
        assert np.all(np.isfinite(a)), n
        # what is 0 by cancellation (dQ and Qt of a row of one key) keeps the rounding of its terms: tau times an
        # inner product of d terms (6 sqrt(d) with normal values) times a key's element (5), 30 here, of which two
        # bf16 values leave 2^-18 and fp32 some 2^-22 (a score's sum of d)
        assert np.abs(a[b == 0]).max(initial=0.0) <= 30 * (2.0 ** -22 if c.get("dtype") == "f32" else 2.0 ** -18), n
        if n in ("alpha", "E", "D"):
            errs[n] = np.abs(a - b).max(initial=0.0) / max(np.abs(b).max(initial=0.0), 1.0)
        else:
            errs[n] = nrel(a, b) if np.linalg.norm(b) > 1e-12 else float(np.linalg.norm(a))
    say("   errs", {n: f"{e:.1e}" for n, e in errs.items()})
    for n, e in errs.items():
        assert e <= bar(n, c.get("dtype")), (n, e)


@pytest.mark.parametrize("name", CASES)
def test_every_output(name):
    c = CASES[name]
    say(f"[score] {name}")
    x = make(c, 11)
    tau = c["d"] ** -0.5
    xd = {n: t.cuda() for n, t in x.items()}
    got = chain(xd, c, tau)
    torch.cuda.synchronize()
    want = reference(x, c, tau)
    compare(got, want, c, [n for n in want])
