"""Upstream gradients of rotate_heads that do not lie where the kernels can read them: the values, and what depends on
them beyond the second derivative."""
import pytest
import torch

from tests.test_gpu_rotary_penalties import LAYERS, start

pytestmark = pytest.mark.gpu


def turned_round(t):
    """(a leaf, t as a view of it whose last stride is not 1)."""
    base = t.transpose(2, 3).contiguous().requires_grad_(True)
    return base, base.transpose(2, 3)


def shifted(t):
    """(a leaf, t as a view of it that is not aligned)."""
    base = torch.zeros(t.numel() + 3, dtype=t.dtype, device=t.device)
    base[3:] = t.flatten()
    base.requires_grad_(True)
    return base, base[3:].view(t.shape)


@LAYERS
@pytest.mark.parametrize("view", [turned_round, shifted])
@pytest.mark.parametrize("name", ["d64_half", "f32_d64", "no_norm"])
def test_values_through_any_strides(name, view, fn):
    c, x, xd, t = start(name, 51)
    leaves = list(t.values())
    dirs = [xd["u" + n] for n in t]
    runs = []
    for made in (lambda v: (v.clone().requires_grad_(True),) * 2, view):
        bases, up = zip(*(made(xd[n]) for n in ("gq", "gk")))
        g = torch.autograd.grad(fn(t, xd, c), leaves, up, create_graph=True)
        runs.append((*g, *torch.autograd.grad(g, [*leaves, *up], dirs, allow_unused=True)))
    for a, b in zip(*runs):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


@LAYERS
@pytest.mark.parametrize("view", [turned_round, shifted])
def test_third_derivatives_by_the_upstream_gradient_are_refused(view, fn):
    """With a norm every second derivative depends on the upstream gradients, however they lie."""
    c, x, xd, t = start("d64_half", 52)
    leaves = list(t.values())
    bases, up = zip(*(view(xd[n]) for n in ("gq", "gk")))
    g = torch.autograd.grad(fn(t, xd, c), leaves, up, create_graph=True)
    h = torch.autograd.grad(g, leaves, [xd["u" + n] for n in t], create_graph=True)
    for a in h:
        with pytest.raises(NotImplementedError, match="third derivatives"):
            torch.autograd.grad(a.float().square().sum(), bases, retain_graph=True, allow_unused=True)
