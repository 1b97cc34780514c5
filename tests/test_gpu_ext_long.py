"""Query sequences long enough that a column block's sum would pass what one accumulator may
add: the column kernels divide it, however many parts that takes, in a bounded workspace, and
the sums keep their accuracy."""
import numpy as np
import pytest
import torch

import paper_2609_24089_amd as fb
from tests.parity_util import say
from tests.test_ext_slices_cpu import SLICE, sizes
from tests.test_gpu_ext import F32, chain, compare, make, reference

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CHAIN = 16384   # tiles of 32 rows into one accumulator


@pytest.mark.parametrize("dt,d", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64),
                                  ("f32", 128)])
@pytest.mark.parametrize("bias", [None, (32, 128)])
def test_no_chain_passes_the_limit(dt, d, bias):
    for kernel in (fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS2):
        for H, Hkv in ((1, 1), (8, 1), (16, 16)):
            for Nq in (1 << 19, (1 << 19) + 1, 1 << 20, (1 << 22) + 100, 1 << 25, 1 << 28):
                for Nk in (16, 5000):
                    if H * Nq >= 1 << 30:
                        continue
                    got = fb.attn_ext_layout(kernel, DT[dt], 1, H, Hkv, Nq, Nk, d, False, bias)
                    tiles, grp = -(-Nq // 32), H // Hkv
                    # a part takes one head's tiles or a share of them, an unsplit block the group's
                    each = tiles * grp if got.parts == 1 else -(-tiles // (got.parts // grp))
                    assert -(-each // got.wave_sets) <= CHAIN, (kernel, H, Nq, Nk, got)


@pytest.mark.parametrize("bias", [None, (32, 128)])
def test_no_grid_passes_a_launch(bias):
    """A grid's second dimension, the parts, ends at 65535; groups of tens of thousands of heads
    whose tiles already pass a chain."""
    for kernel in (fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS2):
        for H in (65535, 40000, 32768, 20000, 4096):
            for Nq in (1, 100, 5000, (1 << 30) // H - 1):
                for Nk in (1, 300):
                    if H * max(Nk, 64) // 64 >= 1 << 24 or H * ((max(Nq, Nk) + 63) // 64) >= 1 << 24:
                        continue
                    got = fb.attn_ext_layout(kernel, torch.bfloat16, 1, H, 1, Nq, Nk, 64, False, bias)
                    assert 1 <= got.parts <= 65535, (H, Nq, Nk, got)


def test_workspaces_of_the_longest_sequences():
    """B1 H16 d64 at 2^22 rows: parts of the whole problem would take 275 GB.  Step sums: a row
    of 5 floats a wave."""
    lib = fb.load_library()
    for N in (1 << 20, 1 << 22):
        for bias in (None, (32, 1)):
            steps = 16 * (N // 16) * 5 * 4 * 16 if bias else 0
            for n, got in sizes(lib, 1, 16, 16, N, N, 64, bias=bias).items():
                assert got <= SLICE + steps, (N, n, got)


def terms(x, c, tau):
    """dS and St of one head in float64: the terms of the tables' sums."""
    n = c["q_lens"][0]
    Q, dO, UQ = (x[m][0, 0, :n].cuda().double() for m in ("Q", "dO", "UQ"))
    K, V, UK, UV = (x[m][0, 0].cuda().double() for m in ("K", "V", "UK", "UV"))
    table, ut, buckets = x["table"][:, 0].cuda().double(), x["UT"][:, 0].cuda().double(), x["buckets"].cuda().long()
    R = (len(buckets) - 1) // 2
    step = torch.arange(c["Nk"], device="cuda")[None] - (c["q_starts"][0] + torch.arange(n, device="cuda")[:, None])
    bucket = buckets[step.clamp(-R, R) + R]
    mean = lambda P, y: (P * y).sum(1, keepdim=True)  # noqa: E731
    P = torch.softmax(tau * Q @ K.T.contiguous() + table[bucket], 1)
    dP = dO @ V.T.contiguous()
    D = mean(P, dP)
    F = tau * (UQ @ K.T.contiguous() + Q @ UK.T.contiguous()) + ut[bucket]
    alpha = mean(P, F)
    Pt = dO @ UV.T.contiguous() + F * (dP - D) - alpha * dP
    return P * (dP - D), P * (Pt - mean(P, Pt))


@pytest.mark.parametrize("name", ["cross", "bias"])
def test_long_queries(name):
    """2^20 and a few queries against 24 keys: 32770 tiles a column block."""
    c = dict(B=1, H=1, Hkv=1, Nq=(1 << 20) + 37, Nk=24, d=32, q_lens=[(1 << 20) + 5])
    if name == "bias":
        c.update(bias=(16, 40), q_starts=[-(1 << 19)])
    x = make(c, 41)
    say(f"[long] {name} {c}")
    for kernel in (fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS2):
        got = fb.attn_ext_layout(kernel, torch.bfloat16, 1, 1, 1, c["Nq"], c["Nk"], c["d"], False, c.get("bias"))
        assert got.parts * got.wave_sets >= 3, got
    got = chain({n: t.cuda() for n, t in x.items()}, c, 0.15)
    torch.cuda.synchronize()
    want = reference(x, c, 0.15)
    compare(got, want, c, [n for n in want if n not in ("dT", "Tt")])
    if name == "bias":
        # Most rows see one bucket alone, in which their terms cancel to 0: half a million rows leave
        # the far buckets what the rounding of 24 terms each leaves.  A term that is rounded once, to
        # fp32, is off by up to 2^-24 of itself, so 2^-24 of the sum of all terms' sizes is what one
        # rounding a term can leave; beside it the bar of all other tables, of the whole result.
        sizes_of = dict(zip(("dT", "Tt"), (float(t.abs().sum()) for t in terms(x, c, 0.15))))
        for n, size in sizes_of.items():
            off = np.linalg.norm(got[n].double().cpu().numpy() - want[n])
            say(f"   {n}: off {off:.1e} of {np.linalg.norm(want[n]):.1e}, terms {size:.1e}")
            assert off <= 2.0 ** -24 * size + F32 * np.linalg.norm(want[n]), n
    # the key rows' sums cancel to zero over the keys (dK, Kt, Vt): what is left is their rounding
    for n in ("dK", "Kt", "Vt"):
        a = got[n][0, 0].double().cpu().numpy()
        assert np.linalg.norm(a.sum(0)) <= 2.0 ** -8 * np.linalg.norm(a) * len(a) ** 0.5, n
