"""The workgroups a compute unit holds, which the forms, parts and block orders are chosen by,
count the LDS that the bias takes beside a kernel's own."""
import pytest
import torch

import paper_2609_24089_amd as fb

pytestmark = pytest.mark.gpu

LDS = 160 * 1024


def steps(far):
    """Bytes of a table by steps of position: one float a step of +-(R + 64)."""
    return 4 * ((2 * (far + 64) + 1 + 3) // 4 * 4)


def test_the_tables_of_a_large_distance_leave_room_for_fewer():
    """Pass 2 in blocks of 32 keys and four wave sets at bf16 d32: 48 KB of rings, 8 KB of row scalars
    and the eight waves' buffers of step sums.  Two workgroups fit with the two tables of a distance
    of 128, one with those of 1024."""
    own = 4 * (3 * 2 * 32 * 32 * 2 + 2 * 2 * 4 * 32 * 4) + 8 * 4 * 76 * 4
    assert 2 * (own + 2 * steps(128)) <= LDS < 2 * (own + 2 * steps(1024))
    for far, fit in ((128, 2), (1024, 1)):
        got = fb.attn_ext_layout(fb.ATTN_EXT_PASS2, torch.bfloat16, 1, 4, 4, 523, 1500, 32, False, (32, far))
        assert (got.rows, got.wave_sets, got.resident) == (32, 4, fit), (far, got)


@pytest.mark.parametrize("kernel", [fb.ATTN_EXT_FWD, fb.ATTN_EXT_ROWS, fb.ATTN_EXT_COLS, fb.ATTN_EXT_PASS1,
                                    fb.ATTN_EXT_PASS2])
@pytest.mark.parametrize("dt,d", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64),
                                  ("f32", 128)])
def test_what_is_resident_fits(kernel, dt, d):
    """Two stages of the streamed tensors and the tables, of every workgroup at once."""
    tensors = {fb.ATTN_EXT_PASS1: 4, fb.ATTN_EXT_PASS2: 3}.get(kernel, 2)
    tables = 2 if kernel in (fb.ATTN_EXT_PASS1, fb.ATTN_EXT_PASS2) else 1
    dtype, size = (torch.bfloat16, 2) if dt == "bf16" else (torch.float32, 4)
    for B, H, N in ((1, 2, 60), (1, 12, 700), (2, 24, 1500), (8, 32, 4096), (1, 16, 1), (2, 32, 3), (16, 64, 20)):
        for group in (1, 8):
            for far in (16, 128, 500, 1024):
                if H < group:
                    continue
                got = fb.attn_ext_layout(kernel, dtype, B, H, H // group, N, N, d, False, (32, far))
                ring = got.wave_sets * tensors * 2 * 32 * d * size
                heads = min(group, (got.rows - 2) // N + 2) if got.folded else 1
                room = got.resident * (ring + heads * tables * steps(far))
                assert got.resident >= 1 and room <= LDS, (B, H, group, N, far, got)
