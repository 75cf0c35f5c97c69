"""pc_shared_attn body by body (row tiles, few rows of 16, 32 and 64, tails behind the prefix's workgroups and in a launch of
their own, one launch for everything; 16-bit and 8-bit rows, 64 and 128 values) against 64 bits."""
import pytest
import torch

import paper_2502_14317_amd as pc
from shared_bodies import CASES, build, check

pytestmark = pytest.mark.gpu
each = pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))


def call(c):
    args = tuple(c[k] for k in ("B", "P", "nq", "Hq", "Hkv", "D"))
    prefix = c["prefix"] and pc.make_row_cache(*c["prefix"], seg_len=c["seg_len"], seg_len_per_head=1)
    tail = c["tail"] and pc.make_row_cache(*c["tail"], seg_len=c["tail_len"])
    out = torch.full_like(c["q"], float("nan"))
    lse = torch.full((c["B"], c["Hq"], c["nq"]), float("nan"), device="cuda")
    ws = pc.alloc_workspace(pc.pc_shared_attn_workspace_bytes(prefix, tail, *args))
    ws.fill_(255)                                                           # NaN where nothing has been written
    pc.pc_shared_attn(c["q"], prefix, tail, *args, out, lse, ws, q_pos=c["pos"], pos0=c["pos0"], rope_base=c["base"],
                      tail_own=tail is not None)
    return out, lse


def checked(c, what):
    out, lse = call(c)
    check(out.float().cpu().numpy(), lse.cpu().numpy(), c, what)
    return out, lse


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@each
@pytest.mark.parametrize("rotated", [False, True], ids=["as is", "rotated"])
def test_against_64_bits(case, rotated):
    print("bodies", case, rotated, flush=True)
    c = build(case, rotated)
    out, lse = checked(c, "deviation 2")
    again, again_lse = call(c)
    assert same(out, again) and same(lse, again_lse), "another order of sums"


@each
def test_large_logits(case):
    """Logits of deviation 60: a row's weight sits on few keys, and the reference moves often."""
    print("bodies, large logits", case, flush=True)
    checked(build(case, False, gain=60.0), "deviation 60")
    checked(build(case, True, gain=60.0), "deviation 60, rotated")


@each
def test_empty_segments_and_tails(case):
    print("bodies, empty", case, flush=True)
    c = build(case, True)
    if c["prefix"]:
        c["seg_len"][:, ::2] = 0
    if c["tail"]:
        c["tail_len"][::2] = 0
        c["tail_len"][1::4] = 1
    checked(c, "every second segment and tail empty")
    for name in ("seg_len", "tail_len"):
        if c[name] is not None:
            c[name].fill_(-2)
    out, lse = call(c)
    assert not out.any() and torch.isneginf(lse).all()


@each
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")], ids=str)
def test_what_nobody_sees_stays_out(case, bad):
    print("bodies, not finite", case, bad, flush=True)
    c = build(case, True)
    clean, clean_lse = call(c)

    def spoil(rows, at):                                                    # at: [.., cap]
        for x, scale in zip(rows[:2], rows[2:]):
            if scale is None:
                x[at] = bad
            else:
                scale[at] = bad
                if bad != bad:
                    x[at] = 0x7f
    for name, lens in (("prefix", "seg_len"), ("tail", "tail_len")):
        if c[name]:
            n, cap = c[lens].view(*c[name][0].shape[:2], -1, 1), c[name][0].shape[3]
            spoil(c[name], (torch.arange(cap, device="cuda") >= n).expand(c[name][0].shape[:4]))
    out, lse = call(c)
    assert same(out, clean) and same(lse, clean_lse), "behind the lengths"
    if not c["tail"]:
        return
    # the last query row's own key and value: no other row sees them
    spoil(c["tail"], (torch.arange(c["tail"][0].shape[3], device="cuda") == c["tail_len"].view(-1, 1, 1, 1) - 1).expand(c["tail"][0].shape[:4]))
    out, lse = call(c)
    assert same(out[:, :-1], clean[:, :-1]) and same(lse[:, :, :-1], clean_lse[:, :, :-1]), "rows that do not see them"
    some = c["tail_len"] > 0
    assert not some.any() or not torch.equal(out[some, -1], clean[some, -1])
