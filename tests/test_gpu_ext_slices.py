"""GPU parity of the two-length column kernels where the parts' sums of all blocks would pass
the bound on their workspace: slices of the blocks, which begin and end inside a head, inside
a batch entry and behind its valid keys, against the float64 oracle."""
import pytest
import torch

import paper_2609_24089_amd as fb
from tests.parity_util import say
from tests.test_ext_slices_cpu import SLICE
from tests.test_gpu_ext import chain, compare, make, reference

pytestmark = pytest.mark.gpu

CASES = {
    "ragged": dict(B=2, H=24, Hkv=3, Nq=40, Nk=12007, d=128, bias=(32, 128), kv_lens=[12007, 5003], q_lens=[33, 40],
                   q_starts=[11000, 4000]),
    "f32_causal": dict(B=3, H=32, Hkv=4, Nq=5, Nk=22001, d=32, dtype="f32", bias=(8, 20), causal=True,
                       q_starts=[21996, 100, 9000]),
    "three_slices": dict(B=1, H=32, Hkv=1, Nq=33, Nk=20011, d=256, bias=(32, 128), table_dtype="bf16"),
}


@pytest.mark.parametrize("name", CASES)
def test_slices(name):
    c = CASES[name]
    say(f"[slices] {name} {c}")
    dt = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    for kernel in (fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS2):
        got = fb.attn_ext_layout(kernel, dt, c["B"], c["H"], c["Hkv"], c["Nq"], c["Nk"], c["d"], c.get("causal", False),
                                 c["bias"])
        assert 2 * got.parts * c["B"] * c["Hkv"] * c["Nk"] * c["d"] * 4 > SLICE, got
    x = make(c, 31)
    tau = c["d"] ** -0.5
    xd = {n: t.cuda() for n, t in x.items()}
    got = chain(xd, c, tau)
    torch.cuda.synchronize()
    want = reference(x, c, tau)
    compare(got, want, c, [n for n in want])
    again = chain(xd, c, tau)
    for n, t in got.items():
        assert torch.equal(again[n], t), n
