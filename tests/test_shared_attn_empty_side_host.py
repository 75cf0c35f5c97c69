"""A side of pc_shared_attn without segments holds nothing: whatever its pointers are, no body that reads through them is
chosen, and the call is planned as if the side were not given."""
import ctypes

import pytest

import paper_2502_14317_amd as pc

AT = ctypes.c_void_p(256)                                                   # never dereferenced


def rows(n_seg, k_scale=None, v_scale=None, cap=64):
    return pc.pc_row_cache(AT, AT, k_scale, v_scale, AT, 0, n_seg, cap)


SCALES = [(AT, None), (None, AT), (AT, AT)]


@pytest.mark.parametrize("eight_bit", [False, True], ids=["16bit", "8bit"])
@pytest.mark.parametrize("cap", [40, 5000])
@pytest.mark.parametrize("scales", SCALES, ids=["keys", "values", "both"])
def test_a_tail_without_segments(scales, cap, eight_bit):
    prefix = rows(1, *([AT, AT] if eight_bit else [None, None]), cap=cap)
    sizes = (2, 1, 1, 8, 2, 128)
    got, want = pc.pc_shared_attn_plan(prefix, rows(0, *scales), *sizes), pc.pc_shared_attn_plan(prefix, None, *sizes)
    assert got["alone"] == (cap == 40) and got["tail_format"] != 2 and got == want
    need = pc.pc_shared_attn_workspace_bytes
    assert need(prefix, rows(0, *scales), *sizes) == need(prefix, None, *sizes) > 0


@pytest.mark.parametrize("scales", SCALES, ids=["keys", "values", "both"])
def test_a_prefix_without_segments(scales):
    tail, sizes = rows(1), (2, 1, 1, 8, 2, 128)
    assert pc.pc_shared_attn_plan(rows(0, *scales), tail, *sizes) == pc.pc_shared_attn_plan(None, tail, *sizes)
