"""Pins of the oracle of attention between sequences of two lengths with a position bias
(oracle/ext_oracle.py), and of the bucket map: torch's own double backward in float64
through a forward written with torch operations, central differences, the case without
bias and lengths against the other oracle, and the bucket rule by logarithms."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import ext_oracle
from paper_2609_24089_amd import relative_buckets

# B, H, Hkv, Nq, Nk, d, causal, biased, q_lens, kv_lens, q_starts
CASES = [
    (1, 1, 1, 1, 1, 2, False, False, None, None, None),
    (2, 2, 1, 3, 7, 4, False, False, [3, 1], [7, 4], None),
    (2, 4, 2, 5, 9, 3, False, True, [5, 4], [9, 6], [0, 2]),
    (1, 2, 2, 6, 6, 4, True, True, None, None, None),
    (2, 2, 1, 2, 11, 4, True, True, None, [8, 11], [6, 9]),
]


def inputs(case, seed):
    B, H, Hkv, Nq, Nk, d, causal, biased, ql, kl, qs = case
    rng = np.random.default_rng(seed)
    q = lambda: rng.standard_normal((B, H, Nq, d))  # noqa: E731
    k = lambda: rng.standard_normal((B, Hkv, Nk, d))  # noqa: E731
    x = dict(Q=q(), K=k(), V=k(), dO=q(), UQ=q(), UK=k(), UV=k())
    opt = dict(causal=causal, q_lens=ql, kv_lens=kl, q_starts=qs)
    if biased:
        buckets = relative_buckets(6, 4, bidirectional=not causal).numpy()
        opt.update(table=rng.standard_normal((6, H)), buckets=buckets)
        x["UT"] = rng.standard_normal((6, H))
    return x, opt


def torch_forward(q, k, v, t, opt, tau):
    """The output on the valid rows (others 0), with torch operations."""
    B, H, Nq, _ = q.shape
    Hkv, Nk = k.shape[1:3]
    rows = []
    for b in range(B):
        n = Nq if opt["q_lens"] is None else opt["q_lens"][b]
        m = Nk if opt["kv_lens"] is None else opt["kv_lens"][b]
        s = 0 if opt["q_starts"] is None else opt["q_starts"][b]
        gap = torch.arange(m)[None, :] - torch.arange(s, s + n)[:, None]
        for h in range(H):
            S = tau * q[b, h, :n] @ k[b, h // (H // Hkv), :m].T
            if t is not None:
                R = (len(opt["buckets"]) - 1) // 2
                S = S + t[:, h][torch.as_tensor(opt["buckets"]).long()[gap.clamp(-R, R) + R]]
            if opt["causal"]:
                S = S.masked_fill(gap > 0, -math.inf)
            o = torch.softmax(S, -1) @ v[b, h // (H // Hkv), :m]
            rows.append(torch.cat([o, torch.zeros(Nq - n, q.shape[-1], dtype=torch.float64)]))
    return torch.stack(rows).reshape(q.shape)


@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
def test_matches_torch_double_backward(case):
    x, opt = inputs(case, 3)
    tau = 0.7
    got = ext_oracle.run(x["Q"], x["K"], x["V"], tau, dO=x["dO"], UQ=x["UQ"], UK=x["UK"], UV=x["UV"], UT=x.get("UT"),
                         **opt)
    leaf = lambda a: torch.tensor(a, requires_grad=True)  # noqa: E731
    q, k, v, dO = (leaf(x[n]) for n in ("Q", "K", "V", "dO"))
    leaves = [q, k, v] + ([leaf(opt["table"])] if "table" in opt else [])
    O = torch_forward(q, k, v, leaves[3] if len(leaves) > 3 else None, opt, tau)
    g = torch.autograd.grad(O, leaves, dO, create_graph=True)
    u = [torch.tensor(x[n]) for n in ("UQ", "UK", "UV", "UT") if n in x]
    h = torch.autograd.grad(g, [*leaves, dO], u, allow_unused=True)
    want = dict(zip(("O", "dQ", "dK", "dV", "dT"), (O, *g)))
    second = ["Qt", "Kt", "Vt"] + (["Tt"] if "table" in opt else []) + ["dOt"]
    want.update({n: torch.zeros_like(w) if t is None else t for n, t, w in zip(second, h, [*leaves, dO])})
    for n, t in want.items():
        np.testing.assert_allclose(got[n], t.detach().numpy(), rtol=0, atol=1e-11, err_msg=n)


def test_differences_of_phi():
    """Phi's gradients in every input by central differences of the first backward."""
    x, opt = inputs(CASES[2], 5)
    tau, eps = 0.9, 1e-5
    got = ext_oracle.run(x["Q"], x["K"], x["V"], tau, dO=x["dO"], UQ=x["UQ"], UK=x["UK"], UV=x["UV"], UT=x["UT"], **opt)

    def phi(y, o):
        r = ext_oracle.run(y["Q"], y["K"], y["V"], tau, dO=y["dO"], **o)
        return sum((r[a] * x[b]).sum() for a, b in (("dQ", "UQ"), ("dK", "UK"), ("dV", "UV"), ("dT", "UT")))

    rng = np.random.default_rng(6)
    for name, out in (("Q", "Qt"), ("K", "Kt"), ("V", "Vt"), ("dO", "dOt"), ("table", "Tt")):
        src = opt if name == "table" else x
        w = rng.standard_normal(src[name].shape)
        ends = []
        for s in (eps, -eps):
            y, o = dict(x), dict(opt)
            (o if name == "table" else y)[name] = src[name] + s * w
            ends.append(phi(y, o))
        assert abs((ends[0] - ends[1]) / (2 * eps) - (got[out] * w).sum()) < 1e-6 * (1 + abs((got[out] * w).sum())), name


@pytest.mark.parametrize("causal", [False, True])
def test_reduces_to_self_attention(causal):
    rng = np.random.default_rng(8)
    args = [rng.standard_normal((1, 2, 9, 4)) for _ in range(7)]
    a = oracle.bob(*args, 0.6, causal=causal)
    Q, K, V, dO, UQ, UK, UV = args
    b = ext_oracle.run(Q, K, V, 0.6, causal=causal, dO=dO, UQ=UQ, UK=UK, UV=UV)
    for n in ("O", "L", "D", "dQ", "dK", "dV", "alpha", "E", "Qt", "Kt", "Vt", "dOt"):
        np.testing.assert_allclose(b[n], a[n], rtol=0, atol=1e-12, err_msg=n)


def test_empty_rows_and_masked_buckets():
    """No key, a masked bucket that is all a row sees, and rows past their length."""
    rng = np.random.default_rng(9)
    Q, K, V, dO = (rng.standard_normal((2, 1, 3, 4)) for _ in range(4))
    r = ext_oracle.run(Q, K, V, 1.0, dO=dO, UQ=Q, UK=K, UV=V, kv_lens=[0, 3], q_lens=[3, 2])
    assert np.all(r["O"][0] == 0) and np.all(np.isneginf(r["L"][0])) and np.isneginf(r["L"][1, 0, 2])
    assert all(np.all(np.isfinite(r[n])) for n in r if n != "L")
    assert all(np.all(r[n][0] == 0) for n in ("dQ", "dK", "dV", "Qt", "Kt", "Vt", "dOt"))
    table = np.array([[np.finfo(np.float32).min], [0.5], [-np.inf], [0.0]])
    buckets = np.array([1, 0, 2])  # step 0 masked: the first causal row sees nothing
    r = ext_oracle.run(Q, K, V, 1.0, causal=True, table=table, buckets=buckets, dO=dO)
    assert np.all(r["O"][:, :, 0] == 0) and np.all(r["dT"][[0, 2]] == 0) and np.all(np.isfinite(r["O"]))


@pytest.mark.parametrize("num,far,both", [(32, 128, True), (32, 128, False), (16, 40, True), (64, 500, False),
                                          (4, 2, True), (2, 2, False), (8, 1024, True)])
def test_bucket_rule(num, far, both):
    """Against the rule by logarithms, which can only be off where a power is exact."""
    got = relative_buckets(num, far, bidirectional=both).tolist()
    assert len(got) == 2 * far + 1
    n = num // 2 if both else num
    e = n // 2
    for step, c in zip(range(-far, far + 1), got):
        x = abs(step) if both or step < 0 else 0
        base = n if both and step > 0 else 0
        if x < e:
            assert c == base + x
            continue
        y = math.log(x / e) / math.log(far / e) * (n - e)
        ok = {base + min(n - 1, e + int(v)) for v in (y - 1e-9, y + 1e-9)}
        assert c in ok, (step, c, ok)
    assert max(got) == num - 1 or (both and far < e) or not both
    assert got[0] == n - 1 and got[far] == 0


@pytest.mark.parametrize("num,far,both", [(3, 10, True), (2, 10, True), (1, 10, False), (32, 8, True), (32, 1025, True),
                                          (1 << 17, 1024, False)])
def test_bucket_refusals(num, far, both):
    with pytest.raises(ValueError):
        relative_buckets(num, far, bidirectional=both)
