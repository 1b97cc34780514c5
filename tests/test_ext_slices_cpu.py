"""Workspaces of the two-length column kernels stay bounded: a group's heads with a bias have
a part each, whose fp32 sums are kept for a slice of the blocks at a time.  No GPU decides
these sizes."""
import ctypes
import os

import pytest

import paper_2609_24089_amd as fb

SLICE = 512 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2609_24089_amd.build import build_library
        build_library()
    return fb.load_library()


def sizes(lib, B, H, Hkv, Nq, Nk, d, dtype=fb.BOB_BF16, bias=(32, 1)):
    e = fb.AttnExt(None, None, None, 16, 16, fb.BOB_F32, *bias) if bias else fb.AttnExt()
    args = (dtype, B, H, Hkv, Nq, Nk, d, 0, ctypes.byref(e))
    return {n: getattr(lib, f"attn_ext_{n}_workspace_bytes")(*args) for n in ("bwd", "pass2")}


@pytest.mark.parametrize("B,H,Hkv,N,d", [(4, 64, 8, 32768, 128), (1, 64, 8, 131072, 128), (1, 32, 1, 1 << 20, 64),
                                         (3, 48, 6, 100003, 256)])
def test_long_grouped_batches_with_a_bias(lib, B, H, Hkv, N, d):
    """The parts' sums of all blocks would take several GB; the step sums (a row of 2 R + 3 = 5
    floats a wave and 16 key rows at most) stay beside the bound."""
    assert 2 * B * H * N * d * 4 > 3 * SLICE
    steps = B * H * (N // 16 + 1) * 5 * 4
    for n, got in sizes(lib, B, H, Hkv, N, N, d).items():
        assert 0 < got <= SLICE + 2 * steps, (n, got)


def test_small_problems_keep_all_parts(lib):
    """Below the bound every part of every block has its place: 2 fp32 matrices a part."""
    for B, H, Hkv, N, d in ((1, 4, 2, 300, 64), (2, 16, 2, 4096, 128)):
        for n, got in sizes(lib, B, H, Hkv, 100, N, d).items():
            assert got >= 2 * B * H * N * d * 4, (n, got)
