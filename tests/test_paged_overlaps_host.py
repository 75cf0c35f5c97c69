"""Outputs that share memory with what every workgroup of a sequence reads are refused, before any launch: also where they only overlap."""
import ctypes

import pytest

from test_paged_errors_host import APPEND, OK, SHAPE, _call

at = ctypes.c_void_p                                                        # never dereferenced
BATCH, NODES = APPEND["batch"], APPEND["n_new"]


@pytest.mark.parametrize("name,entries", [("len_in", BATCH), ("n_rows", BATCH), ("pos", BATCH), ("parent", BATCH * NODES)])
def test_lengths_that_an_append_writes_over_what_it_reads(name, entries):
    for shift in (0, 4 * (entries - 1), -4 * (BATCH - 1)):
        assert _call("pc_kv_append_paged", APPEND, **{name: at(4096), "len_out": at(4096 + shift)}) == SHAPE, shift
    assert _call("pc_kv_append_paged", APPEND, batch=0, **{name: at(4096), "len_out": at(4096)}) == OK
