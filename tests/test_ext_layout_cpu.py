"""The two-length kernels' layout query where no device decides: its refusals, problems that
launch nothing, and what holds of every answer."""
import ctypes
import os

import pytest

import paper_2609_24089_amd as fb

KERNELS = [fb.ATTN_EXT_FWD, fb.ATTN_EXT_ROWS, fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS1, fb.ATTN_EXT_PASS2]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2609_24089_amd.build import build_library
        build_library()
    return fb.load_library()


def query(lib, kernel, dtype=fb.BOB_BF16, B=1, H=4, Hkv=2, Nq=100, Nk=300, d=64, causal=0, bias=None, out=True):
    e = fb.AttnExt()
    if bias is not None:
        e = fb.AttnExt(None, None, None, 16, 16, fb.BOB_F32, *bias)
    got = fb.AttnExtLaunch(-7, -7, -7, -7, -7)
    rc = lib.attn_ext_layout(kernel, dtype, B, H, Hkv, Nq, Nk, d, causal, ctypes.byref(e),
                             ctypes.byref(got) if out else None)
    return rc, (got.rows, got.wave_sets, got.parts, got.folded, got.resident)


@pytest.mark.parametrize("kernel", KERNELS)
def test_refusals(lib, kernel):
    for kw in (dict(B=-1), dict(Nq=-1), dict(H=4, Hkv=3), dict(causal=2), dict(dtype=9), dict(bias=(0, 128)),
               dict(bias=(32, 0)), dict(bias=(32, 1025)), dict(Nk=(1 << 30) + 1), dict(out=False)):
        rc, got = query(lib, kernel, **kw)
        assert rc == fb.BOB_EINVAL and got == (-7,) * 5, kw
    assert query(lib, kernel, d=96)[0] == fb.BOB_EUNSUPPORTED
    for bad in (-1, 5):
        assert query(lib, bad)[0] == fb.BOB_EINVAL


@pytest.mark.parametrize("kernel", KERNELS)
def test_nothing_to_launch(lib, kernel):
    columns = kernel in (fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS2)
    for kw in (dict(B=0), dict(H=0, Hkv=0), dict(Nk=0) if columns else dict(Nq=0), dict(Nq=0, Nk=0)):
        assert query(lib, kernel, **kw) == (fb.BOB_OK, (0,) * 5), kw
    # keys without queries get zeros from their kernel, queries without keys an output
    assert query(lib, kernel, **(dict(Nq=0) if columns else dict(Nk=0)))[1][0] > 0


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("bias", [None, (32, 128)])
def test_answers(lib, kernel, bias):
    """Blocks of whole 16-row sets; the column kernels give each query head of a group a part of
    its own where a head has its own table column."""
    for dtype, dims in ((fb.BOB_BF16, (32, 64, 128, 256)), (fb.BOB_F32, (32, 64, 128))):
        for d in dims:
            for Nq, Nk in ((1, 700), (100, 300), (5000, 40)):
                rc, (rows, sets, parts, folded, resident) = query(lib, kernel, dtype, H=8, Hkv=2, Nq=Nq, Nk=Nk, d=d,
                                                                  bias=bias)
                assert rc == fb.BOB_OK and rows in (16, 32, 64, 128) and sets in (1, 2, 4, 8, 16), (d, Nq, Nk)
                assert folded == (1 if kernel == fb.ATTN_EXT_FWD and Nq == 1 else 0)
                columns = kernel in (fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS2)
                assert parts >= (4 if columns and bias else 1) and parts % (4 if columns and parts > 1 else 1) == 0
                assert resident >= 0
