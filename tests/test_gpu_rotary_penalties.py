"""Second derivatives of rotate_heads that reach a weight whose own first gradient nobody took (gradient penalties,
forces), through the native functions and the Python ones."""
import numpy as np
import pytest
import torch

import paper_2609_24089_amd as fb
from oracle import rotary_oracle
from tests.parity_util import nrel
from tests.test_gpu_rotary import CASES, bar, in_python, make, options, placed

pytestmark = pytest.mark.gpu


def native(t, xd, c):
    return fb.rotate_heads(t["q"], t["k"], xd["positions"], (xd["freqs"], xd["axes"]), t.get("wq"), t.get("wk"),
                           interleaved=c.get("interleaved", False))


LAYERS = pytest.mark.parametrize("fn", [native, in_python])


def start(name, seed, frozen=()):
    c = CASES[name]
    x = make(c, seed)
    xd = placed(x, c)
    t = {n: xd[n].detach().requires_grad_(n not in frozen) for n in ("q", "k", "wq", "wk") if n in xd}
    return c, x, xd, t


@LAYERS
@pytest.mark.parametrize("first", ["qk", "q", "k"])
@pytest.mark.parametrize("name", ["d64_half", "d128", "f32_d64", "queries_normed", "keys_normed", "packed", "unaligned"])
def test_weights_of_a_gradient_by_the_heads(name, first, fn):
    """First gradients by the queries and keys, or one of them, alone; then by the weights."""
    c, x, xd, t = start(name, 41)
    weights = [n for n in ("wq", "wk") if n in t]
    y = fn(t, xd, c)
    g = torch.autograd.grad(y, [t[n] for n in first], [xd["gq"], xd["gk"]], create_graph=True)
    h = torch.autograd.grad(g, [t[n] for n in weights], [xd["u" + n] for n in first], allow_unused=True)
    u = {n: xd["u" + n] if n in first else None for n in "qk"}
    want = fb.attn_rotary_bwd2(xd["q"], xd["k"], xd["gq"], xd["gk"], u["q"], u["k"], **options(xd, c))
    f = {n: v.double().numpy() if v.is_floating_point() else v.numpy() for n, v in x.items()}
    angle = rotary_oracle.angles(f["positions"], f["freqs"], f["axes"])
    for n, got in zip(weights, h):
        exact = want[4 if n == "wq" else 5]
        if n[1] not in first:  # dq does not depend on the keys' weight
            assert got is None or not got.any(), n
            continue
        assert got is not None and torch.equal(got, exact), n
        side = n[1]
        r = rotary_oracle.run(f[side], angle, f[n], 1e-6, c.get("interleaved", False), f["g" + side], f["u" + side],
                              np.zeros(c["d"]))
        assert nrel(got.double().cpu().numpy(), r["wt"]) <= bar("hw" + side, x, c), n


@LAYERS
@pytest.mark.parametrize("frozen", [(), ("wq",), ("wk",), ("q", "k")])
def test_a_penalty_in_a_loss(fn, frozen):
    """A loss of the rotated heads and of the square of its gradients by the queries and keys, against torch operations
    in float64.  Each of the two terms' gradients is within 1e-5 of its size, as a sum of fp32 terms."""
    c, x, xd, t = start("f32_d64", 42)
    if frozen == ("q", "k"):  # the penalty's gradients are those of the heads before a scale, which is no leaf
        frozen, scale = (), {n: torch.ones(1, device="cuda", requires_grad=True) for n in "qk"}
        t.update({n: t[n].detach() * scale[n] for n in "qk"})
    for n in frozen:
        t[n].requires_grad_(False)

    def total(t, layer, gq, gk):
        y = layer(t)
        loss = (y[0] * gq).sum() + (y[1] * gk).sum()
        return loss + sum((a * a).sum() for a in torch.autograd.grad(loss, [t["q"], t["k"]], create_graph=True)) / 2

    total(t, lambda t: fn(t, xd, c), xd["gq"], xd["gk"]).backward()

    def plain(t):
        angle = (xd["positions"].double()[0, :, None, :, None] * xd["freqs"])
        out = []
        for n in "qk":
            v = t[n] / torch.sqrt(t[n].square().mean(-1, keepdim=True) + 1e-6) * t["w" + n]
            a, b = v[..., 0::2], v[..., 1::2]
            out.append(torch.stack([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1).flatten(3))
        return out

    wide = {n: v.detach().double().requires_grad_(True) for n, v in t.items()}
    total(wide, plain, xd["gq"].double(), xd["gk"].double()).backward()
    for n in ("wq", "wk"):
        if n in frozen:
            assert t[n].grad is None
        else:
            assert nrel(t[n].grad.double().cpu().numpy(), wide[n].grad.cpu().numpy()) <= 2e-5, n


@LAYERS
def test_heads_of_a_gradient_by_the_weights(fn):
    """First gradients by the weights alone, then by everything."""
    c, x, xd, t = start("d64_half", 43)
    y = fn(t, xd, c)
    up = [xd[n].clone().requires_grad_(True) for n in ("gq", "gk")]
    g = torch.autograd.grad(y, [t["wq"], t["wk"]], up, create_graph=True)
    h = torch.autograd.grad(g, [*t.values(), *up], [xd["uwq"], xd["uwk"]])
    hq, hk, hgq, hgk, hwq, hwk = fb.attn_rotary_bwd2(xd["q"], xd["k"], xd["gq"], xd["gk"], None, None, gdWq=xd["uwq"],
                                                     gdWk=xd["uwk"], **options(xd, c))
    for a, b in zip(h, (hq, hk, hwq, hwk, hgq, hgk)):
        assert torch.equal(a, b)


def test_captured_and_replayed():
    """The weights' part of a penalty's gradient captured and replayed on changing inputs, with eager work between."""
    c, x, xd, t = start("d128", 44)

    def step():
        y = native(t, xd, c)
        g = torch.autograd.grad(y, [t["q"], t["k"]], [xd["gq"], xd["gk"]], create_graph=True)
        h = torch.autograd.grad(g, list(t.values()), [xd["uq"], xd["uk"]])
        return [a.detach() for a in (*y, *g, *h)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    gen = torch.Generator(device="cuda").manual_seed(5)
    for _ in range(4):
        with torch.no_grad():
            for a in (*t.values(), xd["gq"], xd["uk"]):
                a.copy_(torch.randn(a.shape, generator=gen, device="cuda"))
            xd["positions"].add_(7)
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
