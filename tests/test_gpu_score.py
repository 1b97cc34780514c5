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


# ---------------------------------------------------------------------------
# The differentiable layer
# ---------------------------------------------------------------------------
def layer(xd, c, tau, q, k, v):
    import paper_2609_24089_amd as fb
    return fb.scored_attention(q, k, v, tau, **options(xd, c))


def in_python(xd, c, tau, q, k, v):
    """The layer's functions without the native ones."""
    from paper_2609_24089_amd import score
    o = options(xd, c)
    return score._ScoreFn.apply(q, k, v, *[o[n] for n in ("slopes", "spans", "kv_lens", "q_lens", "q_starts")], tau,
                                o["causal"], o["cap"])


def differentiate(xd, c, tau, fn=layer):
    """The layer's output, its gradients and the gradients of their product with the directions."""
    q, k, v, dO = (xd[n].clone().requires_grad_(True) for n in ("Q", "K", "V", "dO"))
    O = fn(xd, c, tau, q, k, v)
    g = torch.autograd.grad(O, (q, k, v), dO, create_graph=True)
    h = torch.autograd.grad(g, (q, k, v, dO), [xd[n] for n in ("UQ", "UK", "UV")])
    return dict(zip(("O", "dQ", "dK", "dV", "Qt", "Kt", "Vt", "dOt"), [t.detach() for t in (O, *g, *h)]))


LAYERS = ["cap_d64", "slopes_causal", "f32_d128", "empty_entries", "documents_cap", "documents_prefix", "cache_chunk",
          "cache_documents", "split_rows", "split_cols_grouped", "plain", "whole_d64_documents"]


@pytest.mark.parametrize("name", LAYERS)
def test_layers_equal_the_calls(name):
    """Bit for bit, through the native functions and through the Python ones."""
    import paper_2609_24089_amd as fb
    c = CASES[name]
    xd = {n: t.cuda() for n, t in make(c, 12).items()}
    want = chain(xd, c, 0.15)
    got, slow = differentiate(xd, c, 0.15), differentiate(xd, c, 0.15, in_python)
    for n, t in got.items():
        assert torch.equal(t, want[n]), n
        assert torch.equal(slow[n], want[n]), n
    # without a graph of the gradients, and without gradients
    q, k, v = (xd[n].clone().requires_grad_(True) for n in ("Q", "K", "V"))
    for n, t in zip(("dQ", "dK", "dV"), torch.autograd.grad(layer(xd, c, 0.15, q, k, v), (q, k, v), xd["dO"])):
        assert torch.equal(t, want[n]), n
    with torch.no_grad():
        assert torch.equal(layer(xd, c, 0.15, xd["Q"], xd["K"], xd["V"]), want["O"])
    again = chain(xd, c, 0.15)  # no atomics: the same bits twice
    for n, t in want.items():
        assert torch.equal(again[n], t), n
    # into outputs of the caller's, on a stream of the caller's
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, w = options(xd, c), {n: torch.empty_like(t) for n, t in want.items()}
    w["Orest"] = torch.empty_like(xd["Q"]) if xd["Q"].dtype == torch.bfloat16 else None
    Q, K, V, dO, U = xd["Q"], xd["K"], xd["V"], xd["dO"], [xd[n] for n in ("UQ", "UK", "UV")]
    put = lambda *names: tuple(w[n] for n in names)  # noqa: E731
    torch.cuda.synchronize()
    fb.attn_score_fwd_lse(Q, K, V, 0.15, out=put("O", "Orest", "L"), stream=s, **o)
    fb.attn_score_bwd(Q, K, V, w["O"], w["Orest"], dO, w["L"], 0.15, out=put("dQ", "dK", "dV", "D"), stream=s, **o)
    fb.attn_score_pass1_rows(Q, K, V, w["O"], w["Orest"], dO, *U, w["L"], w["D"], w["dQ"], 0.15,
                             out=put("Qt", "dOt", "alpha", "E"), stream=s, **o)
    fb.attn_score_pass2_cols(Q, K, V, dO, *U, w["L"], w["D"], w["alpha"], w["E"], 0.15, out=put("Kt", "Vt"), stream=s,
                             **o)
    s.synchronize()
    for n, t in want.items():
        assert torch.equal(t, w[n]), n


def test_partial_gradients():
    c = CASES["documents_cap"]
    xd = {n: t.cuda() for n, t in make(c, 13).items()}
    want = chain(xd, c, 0.125)
    k = xd["K"].clone().requires_grad_(True)
    (g,) = torch.autograd.grad(layer(xd, c, 0.125, xd["Q"], k, xd["V"]), k, xd["dO"], create_graph=True)
    assert torch.equal(g, want["dK"])
    (h,) = torch.autograd.grad(g, k, xd["UK"])
    zero = {**xd, "UQ": torch.zeros_like(xd["UQ"]), "UV": torch.zeros_like(xd["UV"])}
    assert torch.equal(h, chain(zero, c, 0.125)["Kt"])


@pytest.mark.parametrize("fn", [layer, in_python])
def test_third_derivatives_are_refused(fn):
    """The second gradients may be asked for with a graph; their own are refused."""
    c = CASES["cap_d64"]
    xd = {n: t.cuda() for n, t in make(c, 14).items()}
    want = chain(xd, c, 0.125)
    leaves = [xd[n].clone().requires_grad_(True) for n in ("Q", "K", "V")]
    g = torch.autograd.grad(fn(xd, c, 0.125, *leaves), leaves, xd["dO"], create_graph=True)
    h = torch.autograd.grad(g, leaves, [xd[n] for n in ("UQ", "UK", "UV")], create_graph=True)
    for n, t in zip(("Qt", "Kt", "Vt"), h):
        assert torch.equal(t, want[n]), n
        with pytest.raises(NotImplementedError, match="third derivatives"):
            torch.autograd.grad(t.float().square().sum(), leaves, retain_graph=True, allow_unused=True)


@pytest.mark.parametrize("name", ["cap", "slopes", "prefix"])
def test_gradient_against_differences(name):
    """The fp32 layer's gradients against central differences of its output in float64 sums: with steps of 2^-7
    the third-order term is about 1e-4 of the slope."""
    c = dict(B=1, H=2, Hkv=2, Nq=50, Nk=50, d=32, dtype="f32",
             **{"cap": dict(cap=1.5), "slopes": dict(slopes=True, causal=True, cap=3.0), "prefix": dict(prefix_lens=[20])}[name])
    xd = {n: t.cuda() for n, t in make(c, 14).items()}
    w = xd["dO"].double()
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = chain(xd, c, 0.2)
    for name, out in (("Q", "dQ"), ("K", "dK"), ("V", "dV")):
        u = torch.randn(xd[name].shape, generator=gen, device="cuda")
        ends = []
        for step in (2.0 ** -7, -2.0 ** -7):
            y = {**xd, name: xd[name] + step * u}
            ends.append(float((layer(y, c, 0.2, y["Q"], y["K"], y["V"]).double() * w).sum()))
        slope, exact = (ends[0] - ends[1]) * 2.0 ** 6, float((g[out].double() * u.double()).sum())
        assert abs(slope - exact) <= 2e-3 * max(1.0, abs(exact)), name


# ---------------------------------------------------------------------------
# Padding, masks, memory
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("name", ["tile_edges", "empty_entries", "cap_d128", "f32_d64", "documents_lens", "prefix",
                                  "cache_chunk", "cache_documents", "cache_tokens_grouped", "whole_d64", "split_cols"])
def test_padding_is_never_read(name):
    """NaN and infinities in rows and keys beyond the valid lengths change no output, and padded rows, padded keys
    and empty entries get exact zeros."""
    c = CASES[name]
    xd = {n: t.cuda() for n, t in make(c, 15).items()}
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


def test_documents_do_not_meet():
    """Other values in one document change nothing in another, and padding between them gets exact zeros."""
    c = CASES["documents"]
    xd = {n: t.cuda() for n, t in make(c, 16).items()}
    other = {n: t.cuda() for n, t in make(c, 17).items()}
    at = xd["documents"] == 2  # of entry 0: positions 100 .. 149; of entry 1: 8 .. 39
    mixed = {n: torch.where(at[:, None, :, None], other[n], t) if t.dim() == 4 else t for n, t in xd.items()}
    want, got = chain(xd, c, 0.125), chain(mixed, c, 0.125)
    for n, t in want.items():
        keep = ~at[:, None, :, None] if t.dim() == 4 else ~at[:, None]
        keep = keep.expand(t.shape)
        assert torch.equal(got[n][keep], t[keep]), n
        assert not torch.equal(got[n], t), n
        pad = (xd["documents"] < 0)[:, None] if t.dim() == 3 else (xd["documents"] < 0)[:, None, :, None]
        empty = t[pad.expand(t.shape)]
        assert torch.isneginf(empty).all() if n == "L" else not empty.any(), n


def test_spans_and_the_causal_mask_agree():
    """Spans that say the causal mask give what the mask gives, to rounding: another order of the same tiles."""
    import paper_2609_24089_amd as fb
    c = CASES["cap_d64"]
    x = make(c, 18)
    xd = {n: t.cuda() for n, t in x.items()}
    want = chain(xd, c, 0.125)
    as_spans = {**c, "causal": False, "documents": docs([c["Nk"]]) * c["B"]}
    got = chain({**xd, "documents": torch.tensor(as_spans["documents"], device="cuda")}, as_spans, 0.125)
    for n, t in want.items():
        assert nrel(got[n].double().cpu().numpy(), t.double().cpu().numpy()) <= bar(n, None), n
    spans = fb.attention_spans(c["B"], c["Nk"], device="cuda")
    with pytest.raises(ValueError, match="causal"):
        fb.scored_attention(xd["Q"], xd["K"], xd["V"], causal=True, spans=spans)


def test_bounds_of_spans_beyond_their_range():
    """Bounds beyond 0..Nk count as the nearer end, whatever they hold."""
    import paper_2609_24089_amd as fb
    c = CASES["documents_cap"]
    xd = {n: t.cuda() for n, t in make(c, 19).items()}
    spans = options(xd, c)["spans"]
    wild = spans.clone()
    wild[:, :, 0::2] = torch.where(spans[:, :, 0::2] == 0, -2 ** 31, spans[:, :, 0::2])
    wild[:, :, 1::2] = torch.where(spans[:, :, 1::2] == c["Nk"], 2 ** 31 - 1, spans[:, :, 1::2])
    assert not torch.equal(wild, spans)
    o = {**options(xd, c), "spans": wild}
    O, Orest, L = fb.attn_score_fwd_lse(xd["Q"], xd["K"], xd["V"], 0.125, want_rest=True, **o)
    dQ, dK, dV, D = fb.attn_score_bwd(xd["Q"], xd["K"], xd["V"], O, Orest, xd["dO"], L, 0.125, **o)
    want = chain(xd, c, 0.125)
    for n, t in dict(O=O, L=L, dQ=dQ, dK=dK, dV=dV, D=D).items():
        assert torch.equal(t, want[n]), n


def test_no_queries_and_no_keys():
    import paper_2609_24089_amd as fb
    for B, Nq, Nk in ((2, 0, 40), (2, 30, 0), (2, 0, 0), (0, 5, 6)):
        c = dict(B=B, H=4, Hkv=2, Nq=Nq, Nk=Nk, d=64, cap=2.0, slopes=True, documents=[[0] * Nk] * B)
        x = make(c, 18)
        x["documents"] = x["documents"].reshape(B, Nk)
        got = chain({n: t.cuda() for n, t in x.items()}, c, 0.125)
        for n, t in got.items():
            assert torch.isneginf(t).all() if n == "L" else not t.any(), n
    q, k = torch.zeros(2, 0, 5, 64, device="cuda"), torch.zeros(2, 0, 6, 64, device="cuda")
    assert fb.scored_attention(q, k, k, cap=2.0).shape == q.shape


def test_peaked_rows_and_means():
    """Scores of standard deviation 6, and keys and values with means of three times their spread: the bars stand."""
    for name, by, mean in (("peaks", 6.0, 0.0), ("means", 1.0, 3.0)):
        for more in (dict(causal=True), dict(cap=20.0, causal=True), dict(documents=docs([100, 300, 112]))):
            c = dict(B=1, H=2, Hkv=2, Nq=512, Nk=512, d=64, loud=by, **more)
            x = make(c, 23)
            for n in ("K", "V", "UK", "UV"):
                x[n] = (x[n].float() + mean).to(x[n].dtype)
            say(f"[score] {name} {list(more)}")
            compare(chain({n: t.cuda() for n, t in x.items()}, c, 0.125), reference(x, c, 0.125), c,
                    ("O", "L", "dQ", "dK", "dV", "Qt", "Kt", "Vt", "dOt"))


def test_extreme_scores():
    """Scores that grow late by hundreds (the forward's reference moves), saturated caps, huge slopes and a zero
    scale, against the oracle."""
    import paper_2609_24089_amd as fb
    for tau, grow, more in ((0.125, 40.0, dict(cap=1000.0)), (0.0, 1.0, dict(cap=2.0)), (30.0, 1.0, dict(cap=5.0)),
                            (30.0, 1.0, dict(slopes=True)), (0.125, 1.0, dict(slopes=True, causal=True, by=300.0))):
        c = dict(B=1, H=2, Hkv=2, Nq=90, Nk=400, d=64, **more)
        x = make(c, 19)
        if "slopes" in x:
            x["slopes"] *= more.get("by", 1.0)
        if grow != 1.0:
            x["K"] = (x["K"].float() * 0.1 + 0.05 * torch.linspace(-grow, grow, 400)[:, None]).to(x["K"].dtype)
        want = reference(x, c, tau, second=False)
        xd = {n: t.cuda() for n, t in x.items()}
        O, _, L = fb.attn_score_fwd_lse(xd["Q"], xd["K"], xd["V"], tau, **options(xd, c))
        assert nrel(O.double().cpu().numpy(), want["O"]) <= 2 * BF, (tau, more)
        # L is relative to scores of size up to ~|tau| 8 * 64 * 5
        assert nrel(L.double().cpu().numpy(), want["L"]) <= 1e-5, (tau, more)


@pytest.mark.parametrize("cap", [1e-6, 1e-4, 1e6])
@pytest.mark.parametrize("scale", [1.0, 0.0, 1e-7])
def test_caps_far_from_the_scores(cap, scale):
    """Scores that are 0 or far beyond their cap, and caps far beyond the scores."""
    c = dict(B=1, H=2, Hkv=1, Nq=40, Nk=70, d=64, cap=cap, kv_lens=[67])
    x = make(c, 77)
    x["Q"][:, :, ::3] = 0
    got = chain({n: t.cuda() for n, t in x.items()}, c, scale)
    want = reference(x, c, scale)
    for n in ("O", "L", "D", "dV", "dOt", "Vt"):
        a, b = got[n].double().cpu().numpy(), want[n]
        assert nrel(a, b) <= bar(n, "bf16"), n
    for n in ("dQ", "dK", "Qt", "Kt", "alpha", "E"):
        assert np.all(np.isfinite(got[n].double().cpu().numpy())), n


def test_offsets_past_32_bits():
    """A key/value cache of more than 2^31 elements: the last entry's last keys, under spans and slopes."""
    import paper_2609_24089_amd as fb
    B, H, Nk, d, n = 33, 8, 65536, 128, 700
    assert B * H * Nk * d > 2 ** 31
    k = torch.zeros(B, H, Nk, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    gen = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn(B, H, 1, d, generator=gen, device="cuda").bfloat16()
    k[-1, :, -n:] = torch.randn(H, n, d, generator=gen, device="cuda").bfloat16()
    v[-1, :, -n:] = torch.randn(H, n, d, generator=gen, device="cuda").bfloat16()
    ids = torch.zeros(B, Nk, dtype=torch.int32, device="cuda")
    ids[:, -n:] = 1
    starts = torch.full((B,), Nk - 1, dtype=torch.int32, device="cuda")
    slopes = torch.linspace(0.01, 0.2, H, device="cuda")
    O = fb.scored_attention(q, k, v, 0.1, cap=2.0, slopes=slopes, spans=fb.attention_spans(B, Nk, ids), q_starts=starts)
    S = 0.1 * (k[-1, :, -n:].double() @ q[-1, :, 0].double()[:, :, None])[:, :, 0]
    S = 2 * torch.tanh(S / 2) - slopes.double()[:, None] * torch.arange(n - 1, -1, -1, device="cuda")
    want = (torch.softmax(S, 1)[:, None] @ v[-1, :, -n:].double())[:, 0]
    assert nrel(O[-1, :, 0].double().cpu().numpy(), want.cpu().numpy()) <= 2 * BF
    assert not O[:-1].any()


def test_two_streams_at_once():
    """The whole path on two streams at a time, each with its own inputs and workspaces."""
    jobs = []
    for name in ("split_cols_grouped", "documents_cap"):
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


def test_two_captured_graphs_and_eager_calls_between():
    """A decoding step and a training step captured, replayed in turn on changing inputs with eager work between;
    each replay equals the eager result bit for bit."""
    ct, cg = CASES["cache_token_grouped"], CASES["documents_cap"]
    xt = {n: t.cuda() for n, t in make(ct, 20).items()}
    xg = {n: t.cuda() for n, t in make(cg, 21).items()}
    spans = options(xg, cg)["spans"]

    def token():
        with torch.no_grad():
            return (layer(xt, ct, 0.125, xt["Q"], xt["K"], xt["V"]),)

    def train():
        import paper_2609_24089_amd as fb
        O = fb.scored_attention(*leaves, 0.125, cap=cg["cap"], slopes=xg["slopes"], spans=spans)
        return (O, *torch.autograd.grad(O, leaves, xg["dO"]))

    leaves = [xg[n].requires_grad_(True) for n in ("Q", "K", "V")]
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
        outs.append(o)
    gen = torch.Generator(device="cuda").manual_seed(5)
    for r in range(4):
        with torch.no_grad():
            for t in (xt["Q"], xt["K"], xg["Q"], xg["V"], xg["dO"]):
                t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
            xt["q_starts"].copy_(torch.tensor([299 - r, 100 + r], dtype=torch.int32))
        for i in (r % 2, 1 - r % 2):
            graphs[i].replay()
            want = (token, train)[i]()
            torch.cuda.synchronize()
            for a, b in zip(outs[i], want):
                assert torch.equal(a, b), r


def test_refusals_of_the_layer():
    import paper_2609_24089_amd as fb
    q = torch.zeros(2, 4, 5, 64, device="cuda", dtype=torch.bfloat16)
    k = torch.zeros(2, 2, 7, 64, device="cuda", dtype=torch.bfloat16)
    slopes, spans = torch.zeros(4, device="cuda"), torch.zeros(2, 7, 4, device="cuda", dtype=torch.int32)
    fb.scored_attention(q, k, k, cap=2.0, slopes=slopes, spans=spans)
    for bad, what in ((dict(cap=0.0), "cap"), (dict(cap=-1.0), "cap"), (dict(cap=float("nan")), "cap"),
                      (dict(cap=1e9), "cap"), (dict(slopes=slopes[:3]), "slopes"), (dict(slopes=slopes.double()), "slopes"),
                      (dict(slopes=slopes.cpu()), "slopes"), (dict(slopes=slopes.clone().requires_grad_()), "gradient"),
                      (dict(spans=spans[:, :6]), "spans"), (dict(spans=spans.long()), "spans"),
                      (dict(spans=spans, causal=True), "causal"), (dict(kv_lens=torch.zeros(2, device="cuda")), "kv_lens")):
        with pytest.raises(ValueError, match=what):
            fb.scored_attention(q, k, k, **bad)
    with pytest.raises(ValueError):
        fb.scored_attention(q.transpose(1, 2), k, k, cap=2.0)
