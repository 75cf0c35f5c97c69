"""Outputs that share memory with what every workgroup of a sequence reads are refused, before any launch: also where they only overlap."""
import ctypes

import pytest

from test_paged_errors_host import ACCEPT, APPEND, NULL, OK, SHAPE, _call

at = ctypes.c_void_p                                                        # never dereferenced
BATCH, NODES = APPEND["batch"], APPEND["n_new"]


@pytest.mark.parametrize("name,entries", [("len_in", BATCH), ("n_rows", BATCH), ("pos", BATCH), ("parent", BATCH * NODES)])
def test_lengths_that_an_append_writes_over_what_it_reads(name, entries):
    for shift in (0, 4 * (entries - 1), -4 * (BATCH - 1)):
        assert _call("pc_kv_append_paged", APPEND, **{name: at(4096), "len_out": at(4096 + shift)}) == SHAPE, shift
    assert _call("pc_kv_append_paged", APPEND, batch=0, **{name: at(4096), "len_out": at(4096)}) == OK


# every argument in a place of its own; 3 sequences of 5 nodes, a node's choice every 4 entries
N, STRIDE = ACCEPT["n"], 4
INPUTS = {"tokens": 3 * N, "parent": 3 * N, "choice": (3 * N - 1) * STRIDE + 1, "n_rows": 3, "len_in": 3}
OUTPUTS = {"path": 3 * N, "n_kept": 3, "next_token": 3, "len_out": 3, "pos": 3}
APART = {name: at(4096 * (i + 1)) for i, name in enumerate([*INPUTS, *OUTPUTS])}


@pytest.mark.parametrize("given", INPUTS)
@pytest.mark.parametrize("out", OUTPUTS)
def test_an_acceptance_that_writes_over_what_it_reads(out, given):
    call = lambda **change: _call("pc_tree_accept", {**ACCEPT, **APART, "batch": 3, "choice_stride": STRIDE}, **change)
    ends = (0, 4 * (INPUTS[given] - 1), -4 * (OUTPUTS[out] - 1))
    for shift in ends:
        assert call(**{out: at(APART[given].value + shift)}) == SHAPE, shift
    assert call(**{out: at(APART[given].value), "tokens": None}) == NULL
