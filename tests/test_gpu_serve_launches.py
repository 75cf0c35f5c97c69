"""The launches of pc_shared_attn and pc_verify_drafts as the library's own records name them, against the plan of the call."""
import pytest

import paper_2502_14317_amd as pc
import test_gpu_verify_drafts as verify
from shared_bodies import CASES, build, plan
from test_gpu_shared_attn_bodies import call

pytestmark = pytest.mark.gpu


def launches(run):
    pc.pc_profile_begin()
    run()
    pc.pc_profile_end()
    return [name for name, _ in pc.pc_profile_records()]


@pytest.mark.parametrize("case", CASES[::4], ids=lambda c: "-".join(map(str, c)))
def test_shared_attention(case):
    c, p = build(case, False), plan(case)
    want = ["shared_alone_kernel"] if p["alone"] else \
        ["shared_rows_kernel (prefix)"] * (p["prefix_rows"] > 0) + ["shared_rows_kernel (tails)"] * (p["tail_rows"] > 0 and not p["tails_behind"]) + \
        ["shared_merge_kernel"]
    assert launches(lambda: call(c)) == want


@pytest.mark.parametrize("V,want", [(1000, ["verify_alone_kernel"]), (20000, ["verify_race_kernel", "verify_pick_kernel"])])
def test_verification(V, want):
    args = verify.build(3, 2, V, 1)
    assert launches(lambda: verify.call(*args)) == want
