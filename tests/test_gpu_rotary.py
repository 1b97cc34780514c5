"""GPU parity of normalised, rotated heads against their float64 oracle: forward, backward and the backward of that, at
the layouts, sizes and positions where they can go wrong.

Bars are on ||x - y||_F / ||y||_F per output.  A result is formed in fp32 and rounded once: bf16 at most half a step of
2^-7, 2^-8 of each value.  fp32: sums over up to 256 elements, a few products and a cosine from a float angle of at most
half a turn (off by 2^-24 of pi): 64 2^-24 = 4e-6.  The weights' gradients are sums of up to 10^5 fp32 terms, each workgroup's
in order and then theirs: the rounding of the longest run (2^9 terms) and of the values around it, 2^-13 of their size at
most and 1e-5 of the sum where the terms' signs are mixed; bars 1e-5, and 2^-8 for bf16 weights."""
import numpy as np
import pytest
import torch

from oracle import rotary_oracle
from tests.parity_util import nrel, say

pytestmark = pytest.mark.gpu

# id: B, H, Hkv, N, d and what else the case has
CASES = {
    "token": dict(B=1, H=1, Hkv=1, N=1, d=64),
    "tokens": dict(B=5, H=8, Hkv=2, N=1, d=128, far=120000),
    "d32": dict(B=2, H=3, Hkv=1, N=77, d=32),
    "d64_half": dict(B=2, H=6, Hkv=2, N=131, d=64, pairs=16),
    "d128": dict(B=2, H=4, Hkv=4, N=300, d=128, weights="bf16"),
    "d256": dict(B=1, H=2, Hkv=1, N=65, d=256, pairs=64),
    "f32_d32": dict(B=1, H=2, Hkv=2, N=40, d=32, dtype="f32", pairs=8),
    "f32_d64": dict(B=2, H=3, Hkv=1, N=90, d=64, dtype="f32", interleaved=True),
    "f32_d256": dict(B=1, H=2, Hkv=2, N=33, d=256, dtype="f32"),
    "interleaved": dict(B=2, H=4, Hkv=2, N=100, d=128, interleaved=True, pairs=40),
    "interleaved_d32": dict(B=2, H=4, Hkv=2, N=100, d=32, interleaved=True, weights="bf16"),
    "no_norm": dict(B=2, H=4, Hkv=2, N=150, d=64, norm=""),
    "no_norm_f32": dict(B=2, H=4, Hkv=2, N=150, d=128, norm="", dtype="f32", interleaved=True),
    "queries_normed": dict(B=2, H=4, Hkv=2, N=50, d=64, norm="q"),
    "keys_normed": dict(B=2, H=4, Hkv=2, N=50, d=64, norm="k"),
    "no_rotation": dict(B=2, H=4, Hkv=2, N=50, d=64, pairs=0),
    "axes_2": dict(B=2, H=4, Hkv=2, N=120, d=64, sections=(12, 20), dtype="f32"),
    "axes_3": dict(B=2, H=4, Hkv=2, N=120, d=128, sections=(16, 24, 24), norm=""),
    "far": dict(B=2, H=2, Hkv=1, N=64, d=64, far=2000000000, dtype="f32"),
    "far_negative": dict(B=2, H=2, Hkv=1, N=64, d=64, far=-2000000000, dtype="f32"),
    "many_heads": dict(B=1, H=70, Hkv=35, N=20, d=32),
    "keys_alone": dict(B=2, H=0, Hkv=3, N=20, d=64),
    "queries_alone": dict(B=2, H=3, Hkv=0, N=20, d=64),
    "large": dict(B=3, H=16, Hkv=8, N=1500, d=128),
    "head_major": dict(B=2, H=4, Hkv=2, N=90, d=64, order="heads"),
    "packed": dict(B=2, H=4, Hkv=2, N=90, d=64, order="packed"),
    "unaligned": dict(B=2, H=4, Hkv=2, N=90, d=64, order="unaligned"),
    "loud": dict(B=1, H=4, Hkv=4, N=50, d=64, by=1e4, dtype="f32"),
    "quiet": dict(B=1, H=4, Hkv=4, N=50, d=64, by=1e-3, dtype="f32"),
}


def make(c, seed):
    rng = np.random.default_rng(seed)
    dt = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    B, H, Hkv, N, d = (c[n] for n in ("B", "H", "Hkv", "N", "d"))
    norm = c.get("norm", "qk")
    pairs = c.get("pairs", d // 2)
    t = lambda *s, dtype=dt, by=1.0: torch.tensor(rng.standard_normal(s) * by, dtype=torch.float32).to(dtype)  # noqa: E731
    x = {}
    for n, heads in (("q", H), ("k", Hkv)):
        x[n] = t(B, N, heads, d, by=c.get("by", 1.0)).transpose(1, 2)
        x["g" + n] = t(B, heads, N, d)
        x["u" + n] = t(B, N, heads, d).transpose(1, 2)
        wt = torch.bfloat16 if c.get("weights") == "bf16" else torch.float32
        if n in norm:
            x["w" + n], x["uw" + n] = 1 + t(d, dtype=wt, by=0.3), t(d, dtype=wt)
    sections = c.get("sections", (pairs,))
    x["freqs"] = torch.tensor([10000.0 ** (-i / max(pairs, 1)) for i in range(pairs)], dtype=torch.float64)
    x["axes"] = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], dtype=torch.int32)
    steps = np.sort(rng.integers(0, 5000, (len(sections), B, N)))
    x["positions"] = torch.tensor(steps + c.get("far", 0), dtype=torch.int32)
    return x


def placed(x, c):
    """On the device, the heads in the case's order."""
    xd = {n: v.cuda() for n, v in x.items()}
    order = c.get("order")
    if order == "heads":
        xd.update({n: xd[n].contiguous() for n in ("q", "k")})
    if order in ("packed", "unaligned"):
        H, Hkv = c["H"], c["Hkv"]
        lead = 3 if order == "unaligned" else 0
        both = torch.cat([xd["q"], xd["k"]], 1).transpose(1, 2).flatten(2)
        room = torch.zeros(*both.shape[:2], both.shape[2] + 2 * lead, dtype=both.dtype, device="cuda")
        room[..., lead:lead + both.shape[2]] = both
        heads = room[..., lead:lead + both.shape[2]].unflatten(2, (H + Hkv, c["d"])).transpose(1, 2)
        xd["q"], xd["k"] = heads[:, :H], heads[:, H:]
    return xd


def reference(x, c):
    f = {n: v.double().numpy() if v.is_floating_point() else v.numpy() for n, v in x.items()}
    angle = rotary_oracle.angles(f["positions"], f["freqs"], f["axes"])
    want = {}
    for n in ("q", "k"):
        r = rotary_oracle.run(f[n], angle, f.get("w" + n), 1e-6, c.get("interleaved", False), f["g" + n], f["u" + n],
                              f.get("uw" + n))
        want.update({n: r["y"], "d" + n: r["dx"], "h" + n: r["xt"], "hg" + n: r["dyt"]})
        if "dw" in r:
            want.update({"dw" + n: r["dw"], "hw" + n: r["wt"]})
    return want


def options(xd, c):
    return dict(positions=xd["positions"], freqs=xd["freqs"], axes=xd["axes"], q_weight=xd.get("wq"),
                k_weight=xd.get("wk"), interleaved=c.get("interleaved", False))


def chain(xd, c):
    """The three calls one by one."""
    import paper_2609_24089_amd as fb
    o = options(xd, c)
    q, k, gq, gk = (xd[n] for n in ("q", "k", "gq", "gk"))
    yq, yk = fb.attn_rotary_fwd(q, k, **o)
    dq, dk, dwq, dwk = fb.attn_rotary_bwd(q, k, gq, gk, **o)
    hq, hk, hgq, hgk, hwq, hwk = fb.attn_rotary_bwd2(q, k, gq, gk, xd["uq"], xd["uk"], gdWq=xd.get("uwq"),
                                                     gdWk=xd.get("uwk"), **o)
    out = dict(q=yq, k=yk, dq=dq, dk=dk, dwq=dwq, dwk=dwk, hq=hq, hk=hk, hgq=hgq, hgk=hgk, hwq=hwq, hwk=hwk)
    return {n: t for n, t in out.items() if t is not None}


def bar(name, x, c):
    if "w" in name:
        return 2.0 ** -8 if c.get("weights") == "bf16" else 1e-5
    return 4e-6 if c.get("dtype") == "f32" else 2.0 ** -8


def compare(got, want, x, c):
    errs = {}
    for n, a in got.items():
        a, b = a.double().cpu().numpy(), want[n]
        assert a.shape == b.shape and np.all(np.isfinite(a)), n
        errs[n] = nrel(a, b) if a.size and np.linalg.norm(b) > 0 else float(np.linalg.norm(a))
    say("   errs", {n: f"{e:.1e}" for n, e in errs.items()})
    for n, e in errs.items():
        assert e <= bar(n, x, c), (n, e)


@pytest.mark.parametrize("name", CASES)
def test_every_output(name):
    c = CASES[name]
    say(f"[rotary] {name}")
    x = make(c, 21)
    xd = placed(x, c)
    got = chain(xd, c)
    torch.cuda.synchronize()
    want = reference(x, c)
    for n in want:  # what the calls leave out is 0
        assert n in got or not want[n].any(), n
    compare(got, want, x, c)


def differentiate(xd, c):
    import paper_2609_24089_amd as fb
    names = [n for n in ("q", "k", "wq", "wk") if n in xd]
    leaves = [xd[n].detach().requires_grad_(True) for n in names]
    t = dict(zip(names, leaves))
    up = [xd[n].clone().requires_grad_(True) for n in ("gq", "gk")]
    y = fb.rotate_heads(t["q"], t["k"], xd["positions"], (xd["freqs"], xd["axes"]), t.get("wq"), t.get("wk"),
                        interleaved=c.get("interleaved", False))
    g = torch.autograd.grad(y, leaves, up, create_graph=True)
    h = torch.autograd.grad(g, up + leaves, [xd["u" + n] for n in names], allow_unused=True)
    out = dict(zip(["q", "k"] + ["d" + n for n in names] + ["hgq", "hgk"] + ["h" + n for n in names], (*y, *g, *h)))
    return {n: v.detach() for n, v in out.items() if v is not None}


@pytest.mark.parametrize("name", ["token", "d64_half", "d128", "f32_d64", "no_norm", "queries_normed", "axes_3", "packed",
                                  "unaligned", "head_major", "keys_alone"])
def test_layers_equal_the_calls(name):
    c = CASES[name]
    xd = placed(make(c, 22), c)
    want = chain(xd, c)
    got = differentiate(xd, c)
    assert set(want) <= set(got)
    for n, t in got.items():
        assert n in want and torch.equal(t, want[n]) or n not in want and not t.any(), n
    again = chain(xd, c)  # no atomics: the same bits twice
    for n, t in want.items():
        assert torch.equal(again[n], t), n
