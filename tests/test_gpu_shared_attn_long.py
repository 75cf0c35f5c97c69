"""pc_shared_attn where prefix and tails take workgroups of their own: 1 to 1200 rows a KV head, runs cut into parts,
tails of one to eight wavefronts and of several parts, rows that are not finite, against 64 bits on the CPU."""
import pytest
import torch

from serving import check_attention
from test_gpu_shared_attn import build, call

pytestmark = pytest.mark.gpu

# B, P, n_q, H_q, H_kv, D, segments, k_t, tail cap (0: no tail), prefix format, tail format, per-head lengths, rotate, own
CASES = [
    (1, 1, 1, 8, 2, 128, 3, 300, 20, "bf16", "bf16", 0, True, True),          # 4 rows a KV head
    (4, 1, 1, 8, 2, 64, 2, 700, 1, "row8", "row8", 1, True, True),            # 16
    (3, 1, 3, 8, 2, 128, 5, 233, 50, "bf16", "row8", 1, True, True),          # 36
    (5, 1, 2, 12, 2, 128, 4, 257, 90, "row8", "bf16", 1, False, True),        # 60
    (2, 2, 4, 32, 4, 64, 9, 129, 33, "bf16", "bf16", 0, True, True),          # 32 of each prefix and of each tail
    (8, 2, 5, 8, 2, 128, 3, 401, 33, "row8", "row8", 0, True, True),          # 80, 20 of a tail
    (6, 1, 4, 8, 2, 64, 3, 511, 65, "bf16", "row8", 1, True, False),          # 96
    (16, 2, 4, 8, 2, 128, 2, 290, 31, "bf16", "bf16", 0, True, True),         # 128
    (43, 1, 3, 1, 1, 64, 2, 290, 31, "row8", "bf16", 0, True, True),          # 129
    (40, 2, 3, 4, 1, 128, 2, 300, 40, "bf16", "bf16", 1, True, True),         # 240 of each prefix
    (45, 1, 6, 2, 1, 64, 3, 222, 31, "row8", "row8", 0, True, True),          # 540
    (50, 1, 2, 16, 2, 128, 1, 640, 12, "row8", "bf16", 0, False, True),       # 800
    (3, 1, 1, 8, 2, 128, 1, 64, 1500, "bf16", "bf16", 0, True, True),         # a tail in parts
    (2, 1, 2, 4, 2, 64, 3, 333, 5001, "row8", "row8", 0, True, True),
    (20, 1, 20, 2, 1, 64, 2, 300, 60, "bf16", "bf16", 0, True, True),         # 40 of a tail
    (3, 1, 130, 2, 2, 128, 2, 300, 300, "row8", "row8", 0, True, True),       # 130 of a tail
    (70, 1, 1, 4, 2, 128, 0, 1, 1300, "bf16", "row8", 0, True, True),         # no prefix
    (2, 1, 300, 2, 1, 128, 2, 301, 0, "bf16", "bf16", 1, True, False),        # no tail, 600
    (1, 1, 1, 4, 1, 128, 3, 20000, 0, "row8", "bf16", 0, False, False),
]
# many tails behind a prefix's workgroups: 8, 4, 2 and 1 wavefronts each
TAILS = [
    (40, 1, 1, 8, 4, 64, 2, 300, 16, "row8", "bf16", 0, True, True),
    (40, 1, 2, 8, 8, 64, 2, 300, 100, "row8", "row8", 0, True, True),
    (100, 1, 1, 8, 8, 128, 2, 300, 40, "bf16", "bf16", 0, True, True),
    (160, 2, 2, 8, 8, 64, 2, 300, 100, "bf16", "row8", 0, True, True),
    (300, 1, 1, 4, 4, 128, 2, 300, 9, "bf16", "row8", 0, True, True),
    (300, 3, 3, 8, 4, 64, 2, 300, 37, "row8", "bf16", 0, False, True),
]


@pytest.mark.parametrize("case", CASES + TAILS, ids=lambda c: "-".join(map(str, c)))
def test_against_64_bits(case):
    print("shared attention", case, flush=True)
    c = build(*case)
    out, lse, run = call(c)
    check_attention(out, lse, c, "shared attention")
    first, first_lse = out.clone(), lse.clone()
    run()
    assert torch.equal(out.view(torch.int16), first.view(torch.int16)) and torch.equal(lse, first_lse), "another order of sums"


@pytest.mark.parametrize("case", [CASES[1], CASES[5], CASES[10], CASES[13], *TAILS], ids=lambda c: "-".join(map(str, c)))
def test_empty_segments_and_tails(case):
    print("empty rows", case, flush=True)
    c = build(*case)
    c["seg_len"].flatten()[::2] = 0
    c["tail_len"][::2] = 0
    c["tail_len"][1::4] = 1
    out, lse, _ = call(c)
    check_attention(out, lse, c, "every second segment and tail empty")
    c["seg_len"].fill_(-3)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "no prefix rows")
    assert not out[::2].any() and torch.isneginf(lse[::2]).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("case", [CASES[2], CASES[5], CASES[9], CASES[10], CASES[14], CASES[15], *TAILS[1:4], TAILS[5]],
                         ids=lambda c: "-".join(map(str, c)))
def test_what_nobody_sees_stays_out(case, bad):
    """Rows behind the lengths and later rows of the query block, with keys, values and scales that are not finite."""
    print("not finite", case, bad, flush=True)
    c = build(*case)
    B, P, nq, D, cap = c["B"], c["P"], c["nq"], c["D"], case[8]
    clean, clean_lse, _ = call(c)

    def spoil(x, scale, at):
        if scale is None:
            x[at] = bad
        else:
            if bad != bad:
                x[at] = 0x7f
            scale[at] = bad
    lens = c["seg_len"].cpu()
    for p in range(P):
        for s in range(case[6]):
            for g in range(c["Hkv"]):
                n = int(lens[p, s, g] if c["per_head"] else lens[p, s])
                for x, sc in zip(c["prefix"][:2], c["prefix"][2:]):
                    spoil(x, sc, (p, s, g, slice(n, None)))
    tails = c["tail_len"].tolist()
    for b, n in enumerate(tails):
        for x, sc in zip(c["tail"][:2], c["tail"][2:]):
            spoil(x, sc, (b, 0, slice(None), slice(n, None)))
    out, lse, _ = call(c)
    assert torch.equal(out.view(torch.int16), clean.view(torch.int16)) and torch.equal(lse, clean_lse), "behind the lengths"
    # the block's last row's own key and value: no other row sees them
    for b, n in enumerate(tails):
        if n:
            for x, sc in zip(c["tail"][:2], c["tail"][2:]):
                spoil(x, sc, (b, 0, slice(None), slice(n - 1, n)))
    out, lse, _ = call(c)
    assert torch.equal(out[:, :nq - 1].view(torch.int16), clean[:, :nq - 1].view(torch.int16)), "rows that do not see them"
    assert torch.equal(lse[:, :, :nq - 1], clean_lse[:, :, :nq - 1])
    seen = [b for b, n in enumerate(tails) if n]
    assert not torch.equal(out[seen, nq - 1], clean[seen, nq - 1])


@pytest.mark.parametrize("case", [CASES[1], CASES[7], CASES[9], CASES[13], TAILS[2], TAILS[4]], ids=lambda c: "-".join(map(str, c)))
def test_large_logits(case):
    """Logits of deviation 60: a row's weight sits on one key; the running maximum moves often."""
    print("large logits", case, flush=True)
    c = build(*case, gain=60.0)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "large logits")
