"""Capped attention at caps far from the usual, and at scores that are infinite or NaN.

A cap c far beyond the scores leaves them as they are, so that what tanh is off by, times c, has to stay below what a
score of fp32 is off by anyway, in every kernel: P of a backward pass is formed from the forward's L."""
import numpy as np
import pytest
import torch

import paper_2609_24089_amd as fb
from tests.parity_util import nrel, say
from tests.test_gpu_score import BF, chain, compare, make, reference

pytestmark = pytest.mark.gpu

OUTS = ("O", "L", "dQ", "dK", "dV", "D", "Qt", "Kt", "Vt", "dOt", "alpha", "E")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap,scale,loud", [(1e6, 0.5, 1.0), (2000.0, 0.1, 1.0), (1e4, 0.125, 1.0), (101.0, 0.125, 1.0),
                                            (100.0, 0.125, 1.0), (100.0, 0.5, 1.0), (1e-5, 1.0, 1e-6)])
def test_every_output(cap, scale, loud, dtype):
    """Caps beyond the scores (scale / cap below 1e-4 among them), next to 100, and of the size of tiny scores (scale /
    cap 1e5)."""
    c = dict(B=1, H=2, Hkv=1, Nq=40, Nk=70, d=64, cap=cap, kv_lens=[67], loud=loud, dtype=dtype)
    x = make(c, 78)
    say(f"[cap] {cap} {scale} {dtype}")
    compare(chain({n: t.cuda() for n, t in x.items()}, c, scale), reference(x, c, scale), c, OUTS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["late", "saturated"])
def test_derivatives_at_hard_scores(name, dtype):
    """Scores that grow along the keys, so that the forward's reference moves late, far below their cap; and scores of
    standard deviation 240 under a cap of 5, of which one in thirty has a derivative."""
    cap, tau = (1000.0, 0.125) if name == "late" else (5.0, 30.0)
    c = dict(B=1, H=2, Hkv=2, Nq=90, Nk=400, d=64, cap=cap, dtype=dtype)
    x = make(c, 82)
    if name == "late":
        x["K"] = (x["K"].float() * 0.1 + 0.05 * torch.linspace(-40.0, 40.0, 400)[:, None]).to(x["K"].dtype)
    say(f"[cap] {name} {dtype}")
    compare(chain({n: t.cuda() for n, t in x.items()}, c, tau), reference(x, c, tau), c, OUTS)


def two_tiles(c, seed):
    """All scores of the ordinary rows lie near 0.111 of the cap (c x0, spread 1); row 5 has scores of 0.82 of the cap
    with the first 32 keys and near 0 with the others, so its tile of the first keys is one with scores close to the
    cap and that of the others is not."""
    x = make(c, seed)
    cap = c["cap"]
    Q, K = (torch.zeros_like(x[n]) for n in "QK")
    Q[..., 2:], K[..., 2:] = x["Q"][..., 2:] * 0.125, x["K"][..., 2:]
    K[..., 0] = 128.0
    Q[..., 0] = 0.111 * cap / 128
    K[:, :, :32, 1] = 160.0
    Q[:, :, 5] = 0.0
    Q[:, :, 5, 1] = 0.82 * cap / 160
    x.update(Q=Q, K=K, V=torch.where(torch.arange(64) < 32, 1.0, -1.0)[None, None, :, None] + 0.1 * x["V"].float())
    x["V"] = x["V"].to(x["K"].dtype)
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [3e4, 1e5])
def test_tiles_near_and_far_from_the_cap_agree(cap, dtype):
    """Of a score of c x0 fp32 keeps 2^-24, which eight steps meet: the products' sum (up to four), its scale, the tanh,
    the cap and log2(e), L: P is off by 8 2^-24 c x0, at most 5.3e-3 here, beside its roundings to bf16."""
    c = dict(B=1, H=1, Hkv=1, Nq=16, Nk=64, d=64, cap=cap, dtype=dtype)
    x = two_tiles(c, 79)
    tau = 1.0
    got, want = chain({n: t.cuda() for n, t in x.items()}, c, tau), reference(x, c, tau, second=False)
    score = 8 * 2.0 ** -24 * 0.111 * cap
    for n in ("O", "dV"):
        a, b = got[n].double().cpu().numpy(), want[n]
        say(f"[cap] {cap} {dtype} {n} {nrel(a, b):.1e}")
        assert nrel(a, b) <= score + (2 * BF if dtype == "bf16" else 1e-4), n


# ---------------------------------------------------------------------------
# Infinities and NaN that count
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [5.0, 1e5])
def test_infinite_scores_take_the_cap(cap, dtype):
    """A key with an infinite element has a score of plus or minus the cap, as tanh has it."""
    c = dict(B=1, H=2, Hkv=2, Nq=40, Nk=70, d=64, cap=cap, dtype=dtype)
    x = make(c, 80)
    x["K"][:, :, 7, 3] = float("inf")
    if cap == 1e5:  # minus the cap in every row: with plus that key would have all the weight
        x["K"][:, :, 7, 3] = float("-inf")
        x["Q"][..., 3] = x["Q"][..., 3].abs() + 0.125
    assert (x["Q"][..., 3] != 0).all()
    with np.errstate(invalid="ignore"):
        want = reference(x, c, 0.125, second=False)
    O, _, L = fb.attn_score_fwd_lse(*(x[n].cuda() for n in "QKV"), 0.125, cap=cap)
    for n, t, bar in (("O", O, 2 * BF if dtype == "bf16" else 1e-4), ("L", L, 1e-4)):
        assert np.isfinite(want[n]).all()
        assert nrel(t.double().cpu().numpy(), want[n]) <= bar, n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [None, 5.0, 1e5])
def test_nan_shows_where_it_counts(cap, dtype):
    """NaN in a key reaches every row that sees it; NaN in a query its own row and all gradients of keys and values, and
    no other row."""
    c = dict(B=1, H=2, Hkv=2, Nq=70, Nk=70, d=64, cap=cap, dtype=dtype)
    x = {n: t.cuda() for n, t in make(c, 81).items()}
    clean = chain(x, c, 0.125)
    bad = {**x, "K": x["K"].clone()}
    bad["K"][:, 0, 40, 3] = float("nan")
    got = chain(bad, c, 0.125)
    for n in ("O", "L", "dQ"):
        assert got[n][:, 0].isnan().all() and torch.equal(got[n][:, 1], clean[n][:, 1]), n
    bad = {**x, "Q": x["Q"].clone()}
    bad["Q"][:, 0, 9, 3] = float("nan")
    got = chain(bad, c, 0.125)
    rows = torch.arange(70, device="cuda") != 9
    for n in ("O", "L", "dQ"):
        assert got[n][:, 0, 9].isnan().all(), n
        err = nrel(got[n][:, 0, rows].double().cpu().numpy(), clean[n][:, 0, rows].double().cpu().numpy())
        assert err <= (2 * BF if dtype == "bf16" else 1e-5), n  # its wave may take another of two equal forms
    for n in ("dK", "dV"):
        assert got[n][:, 0].isnan().all() and torch.equal(got[n][:, 1], clean[n][:, 1]), n
