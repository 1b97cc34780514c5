"""Pins of the oracle of attention over capped scores, distance biases and masks by document and prefix
(oracle/score_oracle.py): torch's own double backward in float64 through a forward written with torch operations,
central differences, and the case without any of them against the other oracle.  And of the spans that the library
takes its masks from, against that oracle's masks."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import score_oracle
from paper_2609_24089_amd import attention_spans

DOCS = [[0, 0, 0, 1, 1, 2, 2, 2, 2], [3, 3, 3, 3, 3, 3, 1, -1, -1]]
# B, H, Hkv, Nq, Nk, d and what else the case has
CASES = [
    dict(B=1, H=1, Hkv=1, Nq=1, Nk=1, d=2, cap=2.0),
    dict(B=2, H=2, Hkv=1, Nq=3, Nk=7, d=4, cap=1.5, q_lens=[3, 1], kv_lens=[7, 4]),
    dict(B=1, H=2, Hkv=2, Nq=6, Nk=6, d=3, causal=True, slopes=True),
    dict(B=2, H=4, Hkv=2, Nq=9, Nk=9, d=3, documents=DOCS),
    dict(B=2, H=2, Hkv=1, Nq=9, Nk=9, d=3, documents=DOCS, prefix_lens=[2, 4], cap=2.5, slopes=True),
    dict(B=2, H=2, Hkv=1, Nq=8, Nk=8, d=4, prefix_lens=[3, 0], cap=1.0, q_lens=[8, 5], kv_lens=[8, 5]),
    dict(B=2, H=2, Hkv=1, Nq=2, Nk=9, d=4, causal=True, cap=3.0, slopes=True, kv_lens=[8, 9], q_starts=[6, 7]),
    dict(B=2, H=2, Hkv=1, Nq=3, Nk=9, d=4, documents=DOCS, kv_lens=[8, 9], q_starts=[4, 5]),
]


def inputs(c, seed):
    rng = np.random.default_rng(seed)
    q = lambda: rng.standard_normal((c["B"], c["H"], c["Nq"], c["d"]))  # noqa: E731
    k = lambda: rng.standard_normal((c["B"], c["Hkv"], c["Nk"], c["d"]))  # noqa: E731
    x = dict(Q=q(), K=k(), V=k(), dO=q(), UQ=q(), UK=k(), UV=k())
    opt = {n: c.get(n) for n in ("documents", "prefix_lens", "q_lens", "kv_lens", "q_starts", "cap")}
    opt["causal"] = c.get("causal", False)
    opt["slopes"] = rng.uniform(0.1, 0.8, c["H"]) if c.get("slopes") else None
    return x, opt


def torch_forward(q, k, v, opt, tau):
    """The output with torch operations, the mask from comparisons of whole matrices."""
    B, H, Nq, _ = q.shape
    Hkv, Nk = k.shape[1:3]
    G = H // Hkv
    start = torch.zeros(B, dtype=torch.long) if opt["q_starts"] is None else torch.tensor(opt["q_starts"])
    pos, key = torch.arange(Nq)[None] + start[:, None], torch.arange(Nk)
    ok = torch.ones(B, Nq, Nk, dtype=torch.bool)
    below = key <= pos[:, :, None]
    if opt["documents"] is not None or opt["prefix_lens"] is not None:
        ids = torch.zeros(B, Nk, dtype=torch.long) if opt["documents"] is None else torch.tensor(opt["documents"])
        mine = ids.gather(1, pos.clamp(0, Nk - 1))
        ok &= (mine[:, :, None] == ids[:, None]) & (mine >= 0)[:, :, None] & ((pos >= 0) & (pos < Nk))[:, :, None]
        if opt["prefix_lens"] is not None:
            place = torch.tensor([[sum(int(ids[b, x] == ids[b, j]) for x in range(j)) for j in range(Nk)]
                                  for b in range(B)])
            below = below | (place < torch.tensor(opt["prefix_lens"])[:, None])[:, None]
        ok &= below
    elif opt["causal"]:
        ok &= below
    if opt["kv_lens"] is not None:
        ok &= key < torch.tensor(opt["kv_lens"])[:, None, None]
    if opt["q_lens"] is not None:
        ok &= torch.arange(Nq)[:, None] < torch.tensor(opt["q_lens"])[:, None, None]
    s = tau * q @ k.repeat_interleave(G, 1).transpose(-1, -2)
    if opt["cap"]:
        s = opt["cap"] * torch.tanh(s / opt["cap"])
    if opt["slopes"] is not None:
        s = s - torch.tensor(opt["slopes"])[None, :, None, None] * (key - pos[:, :, None]).abs()[:, None]
    some = ok.any(-1)[:, None, :, None]
    s = torch.where(some, s.masked_fill(~ok[:, None], -math.inf), 0.0)
    return torch.where(some, torch.softmax(s, -1), 0.0) @ v.repeat_interleave(G, 1)


@pytest.mark.parametrize("c", CASES, ids=range(len(CASES)))
def test_matches_torch_double_backward(c):
    x, opt = inputs(c, 3)
    tau = 0.9
    got = score_oracle.run(x["Q"], x["K"], x["V"], tau, dO=x["dO"], UQ=x["UQ"], UK=x["UK"], UV=x["UV"], **opt)
    q, k, v, dO = (torch.tensor(x[n], requires_grad=True) for n in ("Q", "K", "V", "dO"))
    O = torch_forward(q, k, v, opt, tau)
    g = torch.autograd.grad(O, (q, k, v), dO, create_graph=True)
    h = torch.autograd.grad(g, (q, k, v, dO), [torch.tensor(x[n]) for n in ("UQ", "UK", "UV")], allow_unused=True)
    want = dict(zip(("O", "dQ", "dK", "dV"), (O, *g)))
    want.update({n: torch.zeros_like(w) if t is None else t
                 for n, t, w in zip(("Qt", "Kt", "Vt", "dOt"), h, (q, k, v, dO))})
    for n, t in want.items():
        np.testing.assert_allclose(got[n], t.detach().numpy(), rtol=0, atol=1e-11, err_msg=n)


@pytest.mark.parametrize("c", [CASES[1], CASES[4], CASES[6]], ids=("cap", "documents", "cache"))
def test_matches_central_differences(c):
    """Of <O, dO> along a direction, and of <dQ,UQ> + <dK,UK> + <dV,UV> along others, step 1e-5: off by the
    step's square times a third derivative and by rounding over the step, both below 1e-8."""
    x, opt = inputs(c, 5)
    rng = np.random.default_rng(7)
    tau, h = 0.8, 1e-5

    def phi(y):
        r = score_oracle.run(y["Q"], y["K"], y["V"], tau, dO=y["dO"], **opt)
        return (r["O"] * y["dO"]).sum(), sum((r[a] * x[u]).sum() for a, u in (("dQ", "UQ"), ("dK", "UK"), ("dV", "UV")))

    got = score_oracle.run(x["Q"], x["K"], x["V"], tau, dO=x["dO"], UQ=x["UQ"], UK=x["UK"], UV=x["UV"], **opt)
    for name, first, second in (("Q", "dQ", "Qt"), ("K", "dK", "Kt"), ("V", "dV", "Vt"), ("dO", "O", "dOt")):
        w = rng.standard_normal(x[name].shape)
        hi, lo = phi({**x, name: x[name] + h * w}), phi({**x, name: x[name] - h * w})
        assert abs((hi[0] - lo[0]) / (2 * h) - (got[first] * w).sum()) < 1e-7, name
        assert abs((hi[1] - lo[1]) / (2 * h) - (got[second] * w).sum()) < 1e-7, name


def test_plain_case_matches_the_other_oracle():
    c = dict(B=1, H=2, Hkv=2, Nq=6, Nk=6, d=4, causal=True)
    x, opt = inputs(c, 9)
    got = score_oracle.run(x["Q"], x["K"], x["V"], 0.5, dO=x["dO"], UQ=x["UQ"], UK=x["UK"], UV=x["UV"], **opt)
    want = oracle.bob(*[x[n] for n in ("Q", "K", "V", "dO", "UQ", "UK", "UV")], 0.5, causal=True)
    for n in ("Qt", "Kt", "Vt", "dOt", "alpha", "E"):
        np.testing.assert_allclose(got[n], want[n], rtol=0, atol=1e-12, err_msg=n)


def masks(spans, N):
    """The mask that the rows' intervals tell, and the one that the columns' tell."""
    at = torch.arange(N)
    s = spans.long()
    rows = (at >= s[:, :, 0, None]) & (at < s[:, :, 1, None])
    cols = (at >= s[:, :, 2, None]) & (at < s[:, :, 3, None])
    return rows, cols.transpose(1, 2)


@pytest.mark.parametrize("N", [1, 2, 17, 40])
def test_spans_tell_the_mask_on_both_sides(N):
    rng = np.random.default_rng(N)
    for case in range(12):
        B = 3
        docs = np.repeat(rng.integers(-1, 4, (B, N)), rng.integers(1, 6), 1)[:, :N] if case % 3 else None
        prefix = rng.integers(-2, N + 3, B) if case % 2 else None
        spans = attention_spans(B, N, None if docs is None else torch.tensor(docs),
                                None if prefix is None else torch.tensor(prefix, dtype=torch.int32))
        assert spans.dtype == torch.int32 and spans.shape == (B, N, 4) and spans.is_contiguous()
        assert int(spans.min()) >= 0 and int(spans.max()) <= N
        rows, cols = masks(spans, N)
        assert torch.equal(rows, cols)
        for b in range(B):
            want = score_oracle.valid_pairs(b, N, N, 0, True, docs, prefix)
            assert np.array_equal(rows[b].numpy(), want), (case, b)


def test_prefix_of_each_document():
    docs = torch.tensor([[5, 5, 5, 5, 2, 2, 2]])
    spans = attention_spans(1, 7, docs, torch.tensor([[2, 9, 9, 9, 3, 0, 0]]))
    rows, cols = masks(spans, 7)
    assert torch.equal(rows, cols)
    assert rows[0].int().tolist() == [[1, 1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0, 0], [1, 1, 1, 0, 0, 0, 0],
                                      [1, 1, 1, 1, 0, 0, 0], [0, 0, 0, 0, 1, 1, 1], [0, 0, 0, 0, 1, 1, 1],
                                      [0, 0, 0, 0, 1, 1, 1]]


def test_spans_refuse():
    with pytest.raises(ValueError, match="documents"):
        attention_spans(2, 5, torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="documents"):
        attention_spans(2, 5, torch.zeros(2, 5))
    with pytest.raises(ValueError, match="prefix_lens"):
        attention_spans(2, 5, prefix_lens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="negative"):
        attention_spans(-1, 5)
    assert attention_spans(0, 5).shape == (0, 5, 4) and attention_spans(2, 0, torch.zeros(2, 0, dtype=torch.int32)).shape == (2, 0, 4)
