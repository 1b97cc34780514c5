"""Layers and single calls inside functions that torch.compile takes: they run outside its graphs, with the same results
and gradients."""
import pytest
import torch

import paper_2609_24089_amd as fb

pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore:Dynamo does not know:UserWarning")]

N, H, Hkv, d = 40, 4, 2, 64


def inputs():
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = {n: torch.randn(2, h, N, d, generator=gen, device="cuda").bfloat16() for n, h in (("q", H), ("k", Hkv), ("v", Hkv))}
    x["w"] = torch.rand(d, generator=gen, device="cuda") + 0.5
    x["pos"] = torch.arange(N, dtype=torch.int32, device="cuda").expand(2, N).contiguous()
    x["freqs"], x["axes"] = fb.rotary_frequencies(d, device="cuda")
    x["slopes"] = torch.linspace(0.1, 0.4, H, device="cuda")
    x["spans"] = fb.attention_spans(2, N, prefix_lens=torch.tensor([5, 0], device="cuda"))
    return x


def rotary(x):
    return x["pos"], (x["freqs"], x["axes"])


LAYERS = {
    "cross": lambda x, q, k, v, w: fb.cross_attention(q * 2, k, v) + 1,
    "scored": lambda x, q, k, v, w: fb.scored_attention(q * 2, k, v, cap=5.0, causal=True) + 1,
    "scored_all": lambda x, q, k, v, w: fb.scored_attention(q * 2, k, v, cap=5.0, slopes=x["slopes"],
                                                            spans=x["spans"]) + 1,
    "turned": lambda x, q, k, v, w: fb.rotate_heads(q * 2, k, *rotary(x))[0] + 1,
    "rotated": lambda x, q, k, v, w: sum(t.float().sum() for t in fb.rotate_heads(q * 2, k, *rotary(x), w, w)),
    "whole": lambda x, q, k, v, w: fb.rotary_attention(q * 2, k, v, *rotary(x), w, w, slopes=x["slopes"],
                                                       causal=True) + 1,
}


@pytest.mark.parametrize("backend", ["eager", "aot_eager"])
@pytest.mark.parametrize("name", LAYERS)
def test_a_training_step(name, backend):
    x, runs = inputs(), []
    for fn in (LAYERS[name], torch.compile(LAYERS[name], backend=backend)):
        leaves = [x[n].clone().requires_grad_(True) for n in ("q", "k", "v", "w")]
        for _ in range(2):
            y = fn(x, *leaves)
            g = torch.autograd.grad(y.float().square().sum(), leaves, allow_unused=True)
        runs.append((y, *g))
        with torch.no_grad():
            runs[-1] += (fn(x, *leaves),)
    for a, b in zip(*runs):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    torch._dynamo.reset()


def test_second_derivatives():
    x, runs = inputs(), []
    for fn in (LAYERS["whole"], torch.compile(LAYERS["whole"], backend="eager")):
        leaves = [x[n].clone().requires_grad_(True) for n in ("q", "k", "v", "w")]
        g = torch.autograd.grad(fn(x, *leaves).float().square().sum(), leaves, create_graph=True)
        runs.append(torch.autograd.grad(sum(t.float().square().sum() for t in g), leaves))
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    torch._dynamo.reset()


def test_single_calls():
    x = inputs()
    q, k, v = (x[n] for n in "qkv")
    dO = torch.ones_like(q)

    def scored():
        O, rest, L = fb.attn_score_fwd_lse(q * 1, k, v, 0.125, cap=5.0, want_rest=True)
        return (O + 0, L, *fb.attn_score_bwd(q, k, v, O, rest, dO, L, 0.125, cap=5.0))

    def decoded():
        cache = torch.zeros(2, Hkv, 2 * N, d, device="cuda", dtype=k.dtype)
        out = torch.empty_like(q)
        fb.attn_rotary_fwd(q * 1, k, x["pos"], x["freqs"], x["axes"], x["w"], x["w"], out=(out, cache[:, :, 3:3 + N]))
        return out + 0, cache * 1

    def two_lengths():
        O, L = fb.attn_ext_fwd_lse(q * 1, k, v, 0.125, out=(torch.empty_like(q), torch.empty(2, H, N, device="cuda")))
        return O + 0, L

    for fn in (scored, decoded, two_lengths):
        for a, b in zip(fn(), torch.compile(fn, backend="eager")()):
            assert torch.equal(a, b), fn.__name__
    torch._dynamo.reset()
