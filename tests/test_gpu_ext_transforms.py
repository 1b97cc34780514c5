"""The two-length layers under saved-tensor hooks, transforms, tensor subclasses and changes of
their inputs between the passes, as test_gpu_native_binding.py has them for attention()."""
import pytest
import torch

import paper_2609_24089_amd as fb
from tests.test_gpu_ext import CASES, chain, layer, make

pytestmark = pytest.mark.gpu

NAMES = ["tile_edges", "bias_grouped"]


def inputs(name, seed=71):
    c = CASES[name]
    xd = {n: t.cuda() for n, t in make(c, seed).items()}
    leaves = [xd[n].clone().requires_grad_(True) for n in ("Q", "K", "V") + (("table",) if "bias" in c else ())]
    return c, xd, leaves


def run(xd, c, leaves):
    return layer(xd, c, 0.125, *leaves[:3], leaves[3] if len(leaves) > 3 else None)


@pytest.mark.parametrize("name", NAMES)
def test_saved_tensor_hooks(name):
    """Hooks see what both passes keep, and what they return is what is used."""
    c, xd, leaves = inputs(name)
    want = chain(xd, c, 0.125)
    packed = []
    with torch.autograd.graph.saved_tensors_hooks(lambda x: packed.append(x.shape) or x.clone(), lambda x: x):
        O = run(xd, c, leaves)
        assert len(packed) >= 5
        g = torch.autograd.grad(O, leaves, xd["dO"], create_graph=True)
        u = [xd[n] for n in ("UQ", "UK", "UV", "UT") if n in xd]
        h = torch.autograd.grad(g, leaves, u)
    for n, t in zip(["dQ", "dK", "dV"] + ["dT"] * ("bias" in c) + ["Qt", "Kt", "Vt"] + ["Tt"] * ("bias" in c), (*g, *h)):
        assert torch.equal(t, want[n]), n


@pytest.mark.parametrize("name", NAMES)
def test_transforms_are_refused(name):
    c, xd, leaves = inputs(name)
    plain = [t.detach() for t in leaves]
    with pytest.raises(Exception):
        torch.func.vmap(lambda x: run(xd, c, [x, *plain[1:]]))(plain[0][None])
    with torch.autograd.forward_ad.dual_level():
        for i in range(len(plain)):
            dual = list(plain)
            dual[i] = torch.autograd.forward_ad.make_dual(plain[i], torch.ones_like(plain[i]))
            with pytest.raises(Exception):
                run(xd, c, dual)
    with torch.no_grad():
        assert run(xd, c, leaves).grad_fn is None


@pytest.mark.parametrize("name", NAMES)
def test_inputs_changed_in_place_are_noticed(name):
    """Every saved input, the lengths and the buckets among them, between the forward and the
    backward, and between the backward and the second one."""
    c = CASES[name]
    extras = [n for n in ("kv_lens", "q_lens", "buckets") if n in make(c, 71)]
    for which in list(range(4 if "bias" in c else 3)) + extras:
        for second in (False, True):
            c, xd, leaves = inputs(name)
            made = [t * 1 for t in leaves]
            O = run(xd, c, made)
            if second:
                g = torch.autograd.grad(O, leaves, xd["dO"], create_graph=True)
            with torch.no_grad():
                (xd[which] if isinstance(which, str) else made[which]).mul_(2)
            with pytest.raises(RuntimeError, match="inplace|in-place"):
                if second:
                    torch.autograd.grad(g, leaves, [torch.ones_like(t) for t in g])
                else:
                    torch.autograd.grad(O, leaves, xd["dO"])


class Tagged(torch.Tensor):
    """A subclass that takes part in torch's functions."""


@pytest.mark.parametrize("name", NAMES)
def test_tensor_subclasses_keep_their_type(name):
    c, xd, leaves = inputs(name)
    want = chain(xd, c, 0.125)
    sub = [t.detach().as_subclass(Tagged) for t in leaves]
    O = run(xd, c, sub)
    assert type(O) is Tagged and torch.equal(O.as_subclass(torch.Tensor), want["O"])
    q = torch.nn.Parameter(leaves[0].detach())
    O = run(xd, c, [q, *leaves[1:]])
    assert type(O) is torch.Tensor
    assert torch.equal(torch.autograd.grad(O, q, xd["dO"])[0], want["dQ"])


def test_gradients_of_one_use_twice():
    """A graph kept and used again, an upstream gradient without strides, and the same tensor as
    queries, keys and values."""
    c, xd, leaves = inputs("bias_grouped")
    O = run(xd, c, leaves)
    a = torch.autograd.grad(O, leaves, xd["dO"], retain_graph=True)
    b = torch.autograd.grad(O, leaves, xd["dO"], retain_graph=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    one = torch.autograd.grad(O.float().sum(), leaves, retain_graph=True)
    ones = torch.autograd.grad(O, leaves, torch.ones_like(O))
    assert all(torch.equal(x, y) for x, y in zip(one, ones))
    x = torch.randn(2, 3, 50, 64, device="cuda", requires_grad=True)
    d = torch.randn_like(x)
    same, = torch.autograd.grad(fb.cross_attention(x, x, x), x, d)
    parts = [x.detach().clone().requires_grad_(True) for _ in range(3)]
    apart = torch.autograd.grad(fb.cross_attention(*parts), parts, d)
    # added in one order or another: two roundings of fp32 sums of three
    assert (same - (apart[0] + apart[1] + apart[2])).abs().max() <= 4 * 2.0 ** -24 * sum(t.abs().max() for t in apart)
