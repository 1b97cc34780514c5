"""What scored_attention and rotate_heads have no gradient for is refused where one is asked for, never left out."""
import pytest
import torch

import paper_2609_24089_amd as fb

pytestmark = pytest.mark.gpu


def inputs(dtype=torch.bfloat16):
    q = torch.randn(2, 4, 5, 64, device="cuda", dtype=dtype, requires_grad=True)
    k = torch.randn(2, 2, 5, 64, device="cuda", dtype=dtype, requires_grad=True)
    return q, k


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("aligned", [True, False])
def test_frequencies_that_require_a_gradient(norm, aligned):
    """Through the native functions, and (an unaligned head) the Python ones."""
    q, k = inputs()
    if not aligned:
        q = torch.randn(2 * 4 * 5 * 64 + 3, device="cuda", dtype=q.dtype)[3:].view(2, 4, 5, 64).requires_grad_(True)
    pos = torch.arange(10, device="cuda", dtype=torch.int32).view(2, 5)
    freqs, axes = fb.rotary_frequencies(64, device="cuda")
    w = torch.ones(64, device="cuda") if norm else None
    want = fb.rotate_heads(q, k, pos, (freqs, axes), w, w)
    learned = freqs.clone().requires_grad_(True)
    for f in (learned, learned * 1):
        with pytest.raises(ValueError, match="gradient"):
            fb.rotate_heads(q, k, pos, (f, axes), w, w)
        with pytest.raises(ValueError, match="gradient"):
            fb.rotary_attention(q, k, k, pos, (f, axes), w, w)
        with pytest.raises(ValueError, match="gradient"):  # nothing else requires one
            fb.rotate_heads(q.detach(), k.detach(), pos, (f, axes), w, w)
        for y in (fb.rotate_heads(q, k, pos, (f.detach(), axes), w, w), torch.no_grad()(fb.rotate_heads)(
                q, k, pos, (f, axes), w, w)):
            assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1])
    # a training step that follows keeps its gradients
    y = fb.rotate_heads(q, k, pos, (learned.detach(), axes), w, w)
    torch.autograd.grad(y, (q, k), [torch.ones_like(t) for t in y])


def test_tangents_of_constants():
    """Forward-mode tangents of the frequencies and slopes alone."""
    q, k = (t.detach() for t in inputs())
    pos = torch.arange(10, device="cuda", dtype=torch.int32).view(2, 5)
    freqs, axes = fb.rotary_frequencies(64, device="cuda")
    slopes = torch.full((4,), 0.5, device="cuda")
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual
        with pytest.raises(ValueError, match="gradient"):
            fb.rotate_heads(q, k, pos, (dual(freqs, torch.ones_like(freqs)), axes))
        with pytest.raises(ValueError, match="gradient"):
            fb.scored_attention(q, k, k, slopes=dual(slopes, torch.ones_like(slopes)))
        fb.rotate_heads(q, k, pos, (freqs, axes))
        fb.scored_attention(q, k, k, slopes=slopes)
