"""Row vectors (L, D, alpha, E) of another device than the matrices are refused before the library is called: a kernel
would read and write where its device has nothing.  On host tensors, with the check that the matrices lie on a GPU off."""
import pytest
import torch

import paper_2609_24089_amd as fb
from paper_2609_24089_amd import ext, score

ROWS = {"L": 0, "D": 1, "alpha": 2, "E": 3}


@pytest.fixture
def host(monkeypatch):
    def passed(*args):
        raise AssertionError("the checks are behind")

    for mod in (fb, ext, score):
        monkeypatch.setattr(mod, "_check_mats", lambda *ts: ts[0].shape)
        monkeypatch.setattr(mod, "_stream", passed)
        monkeypatch.setattr(mod, "load_library", passed)

    class Slow:  # the native functions take none of these calls
        def __getattr__(self, name):
            return lambda *args: None

    for mod in (fb, ext, score):
        monkeypatch.setattr(mod, "_fast", Slow)


def calls():
    """Every call that takes row vectors: {name: (function of its row vectors by name, their names)}."""
    q, k = torch.zeros(2, 4, 8, 64), torch.zeros(2, 2, 8, 64)
    out = (torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(k))
    pair = (torch.zeros_like(q), torch.zeros_like(q))
    first, second = (q, k, k), (q, q, k, k)  # ... and o, dO, gdQ, gdK, gdV
    found = {}
    for name, fwd, bwd, p1, p2 in (
            ("attn", fb.attn_fwd_lse, fb.attn_bwd, fb.attn_bob_pass1_rows, fb.attn_bob_pass2_cols),
            ("ext", fb.attn_ext_fwd_lse, fb.attn_ext_bwd, fb.attn_ext_pass1_rows, fb.attn_ext_pass2_cols),
            ("score", fb.attn_score_fwd_lse, fb.attn_score_bwd, fb.attn_score_pass1_rows, fb.attn_score_pass2_cols)):
        rest = (None,) if name == "score" else ()
        dq = () if name == "attn" else (q,)
        found.update({
            name + "_fwd": (lambda r, f=fwd, rest=rest: f(*first, 0.1, out=(q, *rest, r["L"])), ("L",)),
            name + "_bwd": (lambda r, f=bwd, rest=rest: f(*first, q, *rest, q, r["L"], 0.1, out=(
                *out, r["D"], *((None,) if f is fb.attn_ext_bwd else ()))), ("L", "D")),
            name + "_pass1": (lambda r, f=p1, rest=rest, dq=dq: f(*first, q, *rest, *second, r["L"], r["D"], *dq, 0.1,
                                                out=(*pair, r["alpha"], r["E"])), tuple(ROWS)),
            name + "_pass2": (lambda r, f=p2: f(*first, *second, *r.values(), 0.1), tuple(ROWS)),
        })
    found["pass2_noalloc"] = (lambda r: fb.attn_bob_pass2_cols_noalloc(*first, *second, *r.values(), 0.1), tuple(ROWS))
    same, four = (q, q, q), (q, q, q, q)
    found["alpha"] = (lambda r: fb.attn_bob3_alpha_rows(*four, r["L"], 0.1, out=r["alpha"]), ("L", "alpha"))
    found["rows3"] = (lambda r: fb.attn_bob3_rows(*same, *four, r["L"], r["D"], r["alpha"], 0.1, out=(*pair, r["E"])),
                      tuple(ROWS))
    return found


@pytest.mark.parametrize("name", calls())
def test_rows_of_another_device(host, name):
    fn, rows = calls()[name]
    good = {n: torch.zeros(2, 4, 8) for n in ROWS}
    with pytest.raises(AssertionError, match="behind"):
        fn(good)
    for n in rows:
        for bad in (good[n].to("meta"), good[n].double(), good[n][..., :4], torch.zeros(2, 4, 16)[..., ::2]):
            with pytest.raises(ValueError, match="row vectors"):
                fn({**good, n: bad})
