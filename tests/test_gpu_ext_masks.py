"""Table entries that stand for a mask without being the type's lowest, and large entries that
do not: rows that see such keys alone, in the forward and both derivatives, against the
float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import ext_oracle
from tests.parity_util import say
from tests.test_gpu_ext import bar, chain, compare, make, reference

pytestmark = pytest.mark.gpu

# far keys share the last bucket of their side; queries 12 and more positions behind the keys see no other
CASE = dict(B=2, H=2, Hkv=1, Nq=90, Nk=50, d=64, bias=(8, 12), kv_lens=[50, 33])


def inputs(entry, dtype="bf16"):
    c = dict(CASE, dtype=dtype)
    x = make(c, 51)
    x["table"][3, 1] = entry    # two-sided: bucket 3 is every key 12 and more positions before the query
    return c, x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("entry", [-2.0 ** 24, -1e8, -1e9, -3e9, -1e10, -1e20, -9e29, -1e30])
def test_masks_of_every_size(entry, dtype):
    c, x = inputs(entry, dtype)
    say(f"[masks] {entry} {dtype}")
    got = chain({n: t.cuda() for n, t in x.items()}, c, 0.125)
    for n, t in got.items():
        assert not torch.isnan(t).any(), n
    empty = slice(CASE["Nk"] + 12, None)    # rows whose every key is masked
    assert torch.isneginf(got["L"][:, 1, empty]).all() and not got["O"][:, 1, empty].any()
    for n in ("dQ", "Qt", "dOt", "D", "alpha", "E"):
        assert not got[n][:, 1, empty].any(), n
    assert not got["dT"][3, 1] and not got["Tt"][3, 1]
    compare(got, reference(x, c, 0.125), c, list(got))


@pytest.mark.parametrize("entry", [-1e4, -65504.0, 3e4])
def test_large_entries_are_no_masks(entry):
    """The exponent of P in the backward kernels is off by the roundings of the score, of L, of L
    times log2(e) and of the two constants' product, each at most half a step of a number of the
    entry's size: 2^-22 of it in all, and P by that much.  Every output is a sum of products with P
    once to three times (itself, through alpha or D, and those through E)."""
    c, x = inputs(entry)
    got = chain({n: t.cuda() for n, t in x.items()}, c, 0.125)
    want = reference(x, c, 0.125)
    off = 3 * 2.0 ** -22 * abs(entry)
    for n, w in want.items():
        a = got[n].double().cpu().numpy()
        e = np.linalg.norm(a - w) / np.linalg.norm(w)
        say(f"   {n} {e:.1e}")
        assert np.isfinite(a).all() and e <= bar(n, None, "f32") + (0 if n in ("O", "L") else off), (n, e)


def test_the_oracle_masks_from_the_same_size():
    assert ext_oracle.MASKED == -2.0 ** 24
    c, x = inputs(float(np.nextafter(np.float32(-2.0 ** 24), np.float32(0))))
    assert np.isfinite(reference(x, c, 0.125, second=False)["L"]).all()
    L = chain({n: t.cuda() for n, t in x.items()}, c, 0.125)["L"]
    assert torch.isfinite(L).all()
