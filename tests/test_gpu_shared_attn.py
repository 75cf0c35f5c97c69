"""pc_shared_attn against 64 bits on the CPU: head layouts, formats, one row to several hundred a KV head, odd sizes,
lengths of zero and one, rows that see nothing, infinities and NaN where nobody looks, offsets beyond 32 bits, other
streams, graphs."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from serving import check_attention, make_rows

pytestmark = pytest.mark.gpu

# B, P, n_q, H_q, H_kv, D, segments, k_t, tail cap (0: no tail), prefix format, tail format, per-head lengths, rotate, own
CASES = [
    (1, 1, 1, 4, 4, 128, 1, 1, 1, "bf16", "bf16", 0, False, True),
    (2, 1, 1, 32, 8, 128, 2, 33, 17, "bf16", "bf16", 0, True, True),
    (4, 2, 1, 8, 2, 128, 3, 65, 40, "row8", "row8", 1, True, True),
    (3, 1, 2, 6, 2, 64, 2, 100, 31, "bf16", "row8", 1, False, True),
    (6, 3, 3, 12, 4, 64, 4, 37, 32, "row8", "bf16", 0, True, True),
    (5, 1, 5, 7, 7, 128, 2, 47, 70, "bf16", "row8", 1, False, True),
    (12, 1, 4, 8, 2, 128, 2, 129, 20, "bf16", "bf16", 0, False, False),      # 192 rows a KV head
    (9, 1, 8, 14, 2, 64, 3, 50, 90, "row8", "row8", 1, True, True),          # 504 rows a KV head, 56 of a sequence
    (2, 2, 40, 3, 1, 128, 2, 64, 200, "bf16", "bf16", 0, True, True),        # many rows a sequence
    (33, 1, 1, 16, 1, 64, 1, 96, 5, "row8", "bf16", 0, False, True),
    (3, 1, 2, 4, 2, 128, 3, 40, 0, "bf16", "bf16", 1, True, False),          # no tail
    (3, 1, 6, 4, 2, 128, 0, 1, 45, "bf16", "row8", 0, False, True),          # no prefix
    (2, 1, 1, 40, 2, 64, 70, 9, 8, "row8", "row8", 1, False, True),          # more segments than lanes
]


def build(B, P, nq, Hq, Hkv, D, S, kt, cap, pf, tf, per_head, rot, own, seed=0, gain=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000 * B + 10 * nq + kt)
    c = {"B": B, "P": P, "nq": nq, "Hq": Hq, "Hkv": Hkv, "D": D, "per_head": per_head, "own": own, "base": 1.0e4, "pos0": 11}
    c["q"] = (gain * torch.randn((B, nq, Hq, D), generator=gen, device="cuda")).to(torch.bfloat16)
    c["spread"] = gain
    c["prefix"] = make_rows(gen, pf, (P, S, Hkv, kt, D)) if S else None
    c["tail"] = make_rows(gen, tf, (B, 1, Hkv, cap, D)) if cap else None
    c["seg_len"] = torch.randint(0, kt + 1, (P, S, Hkv) if per_head else (P, S), generator=gen, device="cuda", dtype=torch.int32) if S else None
    c["tail_len"] = torch.randint(0, cap + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if cap else None
    c["pos"] = torch.randint(0, 9000, (B,), generator=gen, device="cuda", dtype=torch.int32) if rot else None
    return c


def call(c, lse=True):
    B, nq, Hq, D = c["B"], c["nq"], c["Hq"], c["D"]
    rows = lambda n, ln, ph: None if c[n] is None else pc.make_row_cache(*c[n], seg_len=c[ln], seg_len_per_head=ph)
    prefix, tail = rows("prefix", "seg_len", c["per_head"]), rows("tail", "tail_len", 0)
    out = torch.full((B, nq, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    ls = torch.full((B, Hq, nq), float("nan"), dtype=torch.float32, device="cuda") if lse else None
    args = (B, c["P"], nq, Hq, c["Hkv"], D)
    ws = pc.alloc_workspace(pc.pc_shared_attn_workspace_bytes(prefix, tail, *args))
    ws.fill_(255)                                                           # NaN where nothing has been written
    run = lambda: pc.pc_shared_attn(c["q"], prefix, tail, *args, out, ls, ws, q_pos=c["pos"], pos0=c["pos0"],
                                    rope_base=c["base"], softmax_scale=c.get("scale", 0.0), tail_own=c["own"])
    run()
    return out, ls, run


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_64_bits(case):
    print("shared attention", case, flush=True)
    c = build(*case)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "shared attention")


def test_rows_that_see_nothing_and_single_keys():
    c = build(4, 2, 2, 8, 2, 128, 2, 40, 9, "row8", "bf16", 0, False, True)
    c["seg_len"].zero_()
    c["tail_len"].copy_(torch.tensor([0, 1, 2, 9]))                         # sequence 0: nothing; 1: only its last row
    out, lse, _ = call(c)
    check_attention(out, lse, c, "empty rows")
    assert not out[0].any() and torch.isneginf(lse[0]).all() and torch.isneginf(lse[1, :, 0]).all()
    c["seg_len"].fill_(-5); c["tail_len"].fill_(-1)                         # clamped
    out, lse, _ = call(c)
    assert not out.any() and torch.isneginf(lse).all()


def test_no_lengths_a_scale_and_no_logsumexp():
    c = build(3, 1, 2, 4, 4, 64, 3, 45, 33, "bf16", "row8", 0, True, False)
    c["seg_len"] = c["tail_len"] = None
    c["scale"] = 0.2
    c["spread"] = 2.0 * 0.2 * 8.0
    out, _, _ = call(c, lse=False)
    check_attention(out, None, c, "scale 0.2")


@pytest.mark.parametrize("fmt", ["bf16", "row8"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")], ids=str)
def test_what_nobody_sees_stays_out(fmt, bad):
    """Rows behind the lengths and later rows of the query block, with keys, values and scales that are not finite."""
    c = build(3, 1, 4, 8, 2, 128, 2, 70, 50, fmt, fmt, 0, False, True)
    c["seg_len"].copy_(torch.tensor([[37, 64]])); c["tail_len"].copy_(torch.tensor([9, 33, 50]))
    clean, clean_lse, _ = call(c)
    pre, tail = list(c["prefix"]), list(c["tail"])
    code = 0x7f if bad != bad else None

    def spoil(x, scale, at):
        if scale is None:
            x[at] = bad
        elif code is not None:
            x[at] = code
            scale[at] = bad
        else:
            scale[at] = bad
    for s, n in ((0, 37), (1, 64)):
        for x, sc in zip(pre[:2], pre[2:]):
            spoil(x, sc, (0, s, slice(None), slice(n, None)))
    for b, n in enumerate((9, 33, 50)):
        for x, sc in zip(tail[:2], tail[2:]):
            spoil(x, sc, (b, 0, slice(None), slice(n, None)))
    out, lse, _ = call(c)
    assert torch.equal(out.view(torch.int16), clean.view(torch.int16)) and torch.equal(lse, clean_lse), "behind the lengths"
    # the last row's own key and value: rows 0 .. 2 do not see them, row 3 does
    for b, n in enumerate((9, 33, 50)):
        for x, sc in zip(tail[:2], tail[2:]):
            spoil(x, sc, (b, 0, slice(None), slice(n - 1, n)))
    out, lse, _ = call(c)
    assert torch.equal(out[:, :3].view(torch.int16), clean[:, :3].view(torch.int16)), "rows that do not see them"
    assert torch.equal(lse[:, :, :3], clean_lse[:, :, :3])
    assert not torch.equal(out[:, 3], clean[:, 3])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")], ids=str)
def test_a_value_that_is_not_finite_shows_where_it_is_seen(bad):
    c = build(2, 1, 4, 8, 2, 64, 1, 40, 50, "bf16", "bf16", 0, False, True)
    c["tail_len"].copy_(torch.tensor([20, 50]))
    for b, n in enumerate((20, 50)):
        c["tail"][1][b, 0, :, n - 2, 5] = bad                               # seen by rows 2 and 3, value 5 alone
    out, lse, _ = call(c)
    check_attention(out, lse, c, "a value that is not finite")


def test_large_logits():
    """Logits of deviation 60: a row's weight sits on one key; the running maximum moves often."""
    c = build(4, 1, 2, 8, 2, 128, 3, 90, 40, "bf16", "row8", 0, False, True, gain=60.0)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "large logits")


def test_same_bits_again_on_another_stream_and_in_a_graph():
    c = build(10, 2, 3, 8, 2, 128, 4, 150, 60, "row8", "bf16", 1, True, True)
    out, lse, run = call(c)
    want, want_lse = out.clone(), lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse, want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    q = c["q"].clone()
    for i in range(3):
        c["q"].copy_(q * (1.0 + i))                                         # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        run()
        assert torch.equal(out.view(torch.int16), got.view(torch.int16)) and torch.equal(lse, got_lse), i
    c["q"].copy_(q)


@pytest.mark.parametrize("fmt", ["bf16", "row8"])
def test_offsets_beyond_32_bits(fmt):
    """Tails of 2^19 rows: the last sequence's rows lie 4.3 G values behind the first one's."""
    B, Hkv, D, cap, n = 33, 2, 128, 1 << 19, 41
    gen = torch.Generator(device="cuda").manual_seed(5)
    small = make_rows(gen, fmt, (B, 1, Hkv, n, D))
    c = build(B, 1, 1, 4, Hkv, D, 1, 8, 1, "bf16", fmt, 0, False, True)
    c["tail"] = small
    c["tail_len"] = torch.full((B,), n, dtype=torch.int32, device="cuda")
    want, want_lse, _ = call(c)
    big = [None if x is None else torch.empty((B, 1, Hkv, cap, *x.shape[4:]), dtype=x.dtype, device="cuda") for x in small]
    for x, y in zip(big, small):
        if x is not None:
            x[:, :, :, :n] = y
    c["tail"] = tuple(big)
    out, lse, _ = call(c)
    check_attention(want, want_lse, {**c, "tail": small}, "short tails")
    # the tail's capacity decides into how many parts its keys are cut: equal but for rounding
    assert torch.allclose(out.float(), want.float(), atol=2 ** -7, rtol=2 ** -7) and torch.allclose(lse, want_lse, atol=1e-5)


def test_shared_rows_equal_copied_rows():
    """One prefix for five sequences, and five copies of it: the same keys, so the same results to rounding."""
    c = build(5, 1, 2, 8, 2, 128, 3, 77, 30, "bf16", "row8", 1, True, True)
    out, lse, _ = call(c)
    copied = {**c, "P": 5, "prefix": tuple(None if x is None else x.expand(5, *x.shape[1:]).contiguous() for x in c["prefix"]),
              "seg_len": c["seg_len"].expand(5, *c["seg_len"].shape[1:]).contiguous()}
    out2, lse2, _ = call(copied)
    assert torch.allclose(out.float(), out2.float(), atol=2 ** -7, rtol=2 ** -7) and torch.allclose(lse, lse2, atol=2e-5)
