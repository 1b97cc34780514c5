"""Outputs that the caller gives to attn_rotary_bwd for the weights' gradients."""
import pytest
import torch

import paper_2609_24089_amd as fb
from tests.test_gpu_rotary import CASES, chain, make, options, placed

pytestmark = pytest.mark.gpu


def test_outputs_of_the_callers():
    c = CASES["d64_half"]
    xd = placed(make(c, 61), c)
    want = chain(xd, c)
    args = [xd[n] for n in ("q", "k", "gq", "gk")]
    out = [torch.full_like(want[n], 7.0) for n in ("dq", "dk", "dwq", "dwk")]
    fb.attn_rotary_bwd(*args, out=out, **options(xd, c))
    for t, n in zip(out, ("dq", "dk", "dwq", "dwk")):
        assert torch.equal(t, want[n]), n
    # every check comes before the launch
    w = out[2]
    for bad in (w.cpu(), w.double(), w[:32], torch.zeros(128, device="cuda")[::2]):
        for at in (2, 3):
            with pytest.raises(ValueError, match="must be like its weight"):
                fb.attn_rotary_bwd(*args, out=[bad if i == at else t for i, t in enumerate(out)], **options(xd, c))
    more = {**options(xd, c), "k_weight": None}
    with pytest.raises(ValueError, match="must be like its weight"):
        fb.attn_rotary_bwd(*args, out=out, **more)
