"""Forward-mode tangents of upstream gradients: the layers have no forward mode, and refuse them rather than returning
gradients without theirs, from the first backward and from the second."""
import pytest
import torch
import torch.autograd.forward_ad as fw

import paper_2609_24089_amd as fb
from paper_2609_24089_amd import ext, rotary, score

pytestmark = pytest.mark.gpu

N, H, d = 16, 2, 64


def constants():
    pos = torch.arange(N, device="cuda", dtype=torch.int32)[None].contiguous()
    return pos, fb.rotary_frequencies(d, device="cuda"), torch.ones(d, device="cuda")


def rotate(norm, native):
    pos, (freqs, axes), w = constants()
    w = w if norm else None
    if native:
        return lambda q, k, v: fb.rotate_heads(q, k, pos, (freqs, axes), w, w)[0]
    if norm:
        return lambda q, k, v: rotary._RotaryFn.apply(q, k, w, w, pos, freqs, axes, 1e-6, False)[0]
    return lambda q, k, v: rotary._RotateFn.apply(q, k, pos, freqs, axes, False, False, (False, False))[0]


def biased():
    bias = torch.zeros(32, H, device="cuda"), fb.relative_buckets(32, 128, device="cuda")
    return lambda q, k, v: fb.biased_attention(q, k, v, *bias)


LAYERS = {
    "attention": lambda: lambda q, k, v: fb.attention(q, k, v, 0.125, True),
    "cross": lambda: fb.cross_attention,
    "biased": biased,
    "cross_python": lambda: lambda q, k, v: ext._ExtFn.apply(q, k, v, *(None,) * 5, 0.125, False),
    "scored": lambda: lambda q, k, v: fb.scored_attention(q, k, v, cap=5.0),
    "scored_python": lambda: lambda q, k, v: score._ScoreFn.apply(q, k, v, *(None,) * 5, 0.125, False, 5.0),
    "rotated": lambda: rotate(True, True),
    "rotated_python": lambda: rotate(True, False),
    "turned": lambda: rotate(False, True),
    "turned_python": lambda: rotate(False, False),
}


def leaves():
    gen = torch.Generator(device="cuda").manual_seed(7)
    return [torch.randn(1, H, N, d, generator=gen, device="cuda", requires_grad=True) for _ in range(3)]


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("name", LAYERS)
def test_first_backward(name, graph):
    layer, (q, k, v) = LAYERS[name](), leaves()
    y = layer(q, k, v)
    plain, = torch.autograd.grad(y, q, torch.ones_like(y), retain_graph=True)
    with fw.dual_level():
        up = fw.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises(Exception, match="jvp|forward"):
            torch.autograd.grad(y, q, up, create_graph=graph, retain_graph=True)
        again, = torch.autograd.grad(y, q, torch.ones_like(y))  # without a tangent, inside the level
    assert torch.equal(again, plain)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("name", [n for n in LAYERS if not n.startswith(("attention", "turned"))])
def test_second_backward(name, graph):
    layer, (q, k, v) = LAYERS[name](), leaves()
    y = layer(q, k, v)
    g, = torch.autograd.grad(y, q, torch.ones_like(y), create_graph=True)
    plain, = torch.autograd.grad(g, q, torch.ones_like(g), retain_graph=True)
    with fw.dual_level():
        u = fw.make_dual(torch.ones_like(g), torch.ones_like(g))
        with pytest.raises(Exception, match="jvp|forward"):
            torch.autograd.grad(g, q, u, create_graph=graph, retain_graph=True)
        again, = torch.autograd.grad(g, q, torch.ones_like(g))
    assert torch.equal(again, plain)
