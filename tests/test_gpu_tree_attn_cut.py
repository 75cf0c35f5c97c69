"""pc_tree_attn where its tables are wide, so that sequences are cut into shares and joined, and its bodies of many query rows: the
same statement in 64 bits as for small tables."""
import pytest
import torch

from test_gpu_tree_attn import NO, call
from trees import build, check_attention

pytestmark = pytest.mark.gpu


def wide(c, places=4096):
    """More columns in the table, without pages: room for `places` rows a sequence."""
    t = c["table"]
    more = max(0, places // c["page"] + 1 - t.shape[1])
    return dict(c, table=torch.cat([t, torch.full((c["B"], more), -1, dtype=torch.int32, device="cuda")], 1))


# B, n, H_q, H_kv, D, page, most rows in front, format, tree, ragged, rotate
CASES = [
    (5, 1, 8, 2, 128, 64, 1500, "bf16", False, True, True),
    (5, 4, 8, 2, 64, 16, 900, "row8", True, True, True),             # 16 query rows a KV head
    (4, 8, 8, 2, 128, 32, 900, "row8", True, False, True),           # 32
    (4, 7, 12, 3, 64, 16, 700, "bf16", True, True, False),           # 28
    (4, 16, 8, 2, 128, 16, 900, "bf16", True, True, True),           # 64
    (4, 15, 8, 2, 64, 64, 700, "bf16", True, False, True),           # 60
    (3, 9, 14, 2, 128, 32, 800, "row8", True, True, True),           # 63
    (3, 33, 1, 1, 64, 16, 900, "row8", True, True, True),            # 33
    (3, 32, 8, 2, 128, 16, 800, "bf16", True, True, True),           # 128
    (3, 31, 8, 2, 64, 32, 600, "bf16", True, False, False),          # 124
    (3, 26, 10, 2, 128, 128, 700, "row8", True, True, True),         # 130: a second tile of two
    (2, 64, 14, 2, 64, 16, 500, "row8", True, True, True),           # 448
    (300, 2, 4, 2, 64, 16, 60, "bf16", True, True, True),            # more sequences than threads
    (270, 16, 4, 1, 128, 16, 40, "row8", True, True, False),
    (600, 1, 1, 1, 64, 16, 30, "row8", False, True, True),
    (1, 16, 8, 2, 128, 64, 9000, "row8", True, False, True),         # one sequence, more shares than pieces of 8 blocks
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_64_bits(case):
    print("tree attention, cut", case, flush=True)
    c = wide(build(*case))
    out, lse, _ = call(c)
    check_attention(out, lse, c, "cut", NO)


MANY = [(16, 8, 2, 128, "bf16"), (16, 4, 1, 64, "row8"), (8, 16, 2, 128, "row8"), (32, 4, 1, 128, "bf16"), (21, 12, 2, 64, "bf16"), (32, 4, 1, 64, "row8")]
TABLES = [0, 4096]


@pytest.mark.parametrize("places", TABLES)
@pytest.mark.parametrize("shape", [(2, 4, 1, 128, "bf16"), (8, 4, 1, 64, "row8")] + MANY, ids=lambda s: "-".join(map(str, s)))
def test_pages_that_are_not_there(shape, places):
    n, Hq, Hkv, D, fmt = shape
    c = build(4, n, Hq, Hkv, D, 16, 0, fmt, True, False, True, lens=[100, 64, 190, 440])
    t = c["table"]
    t[0, 1], t[0, 4] = -1, c["n_pages"]                                     # in the middle of a sequence
    t[1] = -5                                                               # all of one
    t[2, 11] = 2 ** 31 - 1                                                  # rows of the tree's own
    t[3, 3], t[3, 6:8] = -2, c["n_pages"] + 7
    c = wide(c, places)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "pages", NO)
    assert not out[1].any() and torch.isneginf(lse[1]).all()


@pytest.mark.parametrize("places", TABLES)
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "-".join(map(str, s)))
def test_empty_sequences_and_sequences_shorter_than_their_trees(shape, places):
    n, Hq, Hkv, D, fmt = shape
    c = build(8, n, Hq, Hkv, D, 16, 0, fmt, True, False, True, lens=[n, n, n, 300, n, 33, n, n + 1])
    c["len"].copy_(torch.tensor([0, 1, n, 300, -4, 33, n - 1, n + 1]))
    c["n_rows"] = torch.tensor([n, n, 0, n + 5, n, -3, n, 1], dtype=torch.int32, device="cuda")
    c = wide(c, places)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "few rows", NO)
    assert not out[0].any() and torch.isneginf(lse[0]).all()


@pytest.mark.parametrize("places", TABLES)
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")], ids=str)
def test_what_a_node_does_not_see_stays_out(shape, bad, places):
    """A node's row that is not finite belongs to it and to those below it."""
    n, Hq, Hkv, D, fmt = shape
    c = build(3, n, Hq, Hkv, D, 16, 0, fmt, True, False, False, lens=[n, 70 + n, 333 + n])
    c["parent"][:, 0], c["parent"][:, 1:4] = -1, 0
    c["parent"][:, 4:6], c["parent"][:, 6:] = 2, 0                          # 4 and 5 are below node 2
    c = wide(c, places)
    clean, clean_lse, _ = call(c)
    for b in range(3):
        j = int(c["len"][b]) - n + 2
        at = (int(c["table"][b, j // 16]), slice(None), j % 16)
        if fmt == "bf16":
            c["v"][at] = bad
        elif bad != bad:
            c["v"][at] = 0x7f
        else:
            c["v_scale"][at] = bad
    out, lse, _ = call(c)
    seen = [2, 4, 5]
    unseen = [t for t in range(n) if t not in seen]
    assert torch.equal(out[:, unseen], clean[:, unseen]) and torch.equal(lse, clean_lse)
    assert not torch.isfinite(out[:, seen].float()).any()
    if fmt == "bf16":
        assert (out[:, seen].isnan().all() if bad != bad else (out[:, seen].float() == bad).all())


@pytest.mark.parametrize("places", TABLES)
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "-".join(map(str, s)))
def test_single_values_that_are_not_finite(shape, places):
    """One value of a row in front of the tree, and one of a node's: they reach their own place of the result and no other."""
    n, Hq, Hkv, D, fmt = shape
    c = build(2, n, Hq, Hkv, D, 16, 0, fmt, True, False, False, lens=[40 + n, 333 + n])
    c = wide(c, places)
    for b in range(2):
        base = int(c["len"][b]) - n
        for j, g, d in ((base - 3, Hkv - 1, 5), (base + n // 2, 0, D - 1)):
            c["v"][int(c["table"][b, j // 16]), g, j % 16, d] = 0x7f if fmt == "row8" else float("nan")
    out, lse, _ = call(c)
    check_attention(out, lse, c, "single values", NO)


@pytest.mark.parametrize("places", TABLES)
@pytest.mark.parametrize("n,Hq", [(1, 4), (8, 4), (16, 4), (32, 4)])
def test_keys_that_are_not_finite(n, Hq, places):
    c = build(2, n, Hq, 1, 128, 32, 0, "bf16", False, False, False, lens=[90 + n, 40 + n])
    c = wide(c, places)
    c["parent"] = torch.full((2, n), -1, dtype=torch.int32, device="cuda")
    clean, clean_lse, _ = call(c)
    t = n - 1
    for b in range(2):
        j = int(c["len"][b]) - n + t
        c["k"][int(c["table"][b, j // 32]), :, j % 32] = float("nan")
    out, lse, _ = call(c)
    assert torch.equal(out[:, :t], clean[:, :t]) and torch.equal(lse[:, :, :t], clean_lse[:, :, :t])
    assert out[:, t].isnan().all()


@pytest.mark.parametrize("shape", [(1, 4, 1, 128, "bf16"), (8, 4, 1, 64, "row8")] + MANY, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("places", [512, 2112])
def test_lengths_behind_the_table(shape, places):
    """Rows without a place in the table are seen by nobody, however long a sequence is said to be."""
    n, Hq, Hkv, D, fmt = shape
    c = build(2, n, Hq, Hkv, D, 64, 0, fmt, True, False, True, lens=[places, places])
    c["table"] = c["table"][:, :places // 64].contiguous()
    c["len"].fill_(places + n)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "behind the table", NO)
    c["len"].fill_(2 ** 31 - 1)
    far, far_lse, _ = call(c)
    assert torch.equal(far, out) and torch.equal(far_lse, lse)


@pytest.mark.parametrize("shape", MANY, ids=lambda s: "-".join(map(str, s)))
def test_large_logits(shape):
    n, Hq, Hkv, D, fmt = shape
    c = wide(build(3, n, Hq, Hkv, D, 16, 600, fmt, True, False, True, gain=7.0))
    out, lse, _ = call(c)
    check_attention(out, lse, c, "large logits", NO)


@pytest.mark.parametrize("n,Hq,fmt", [(1, 4, "bf16"), (16, 4, "bf16"), (16, 4, "row8"), (32, 4, "row8")])
def test_pools_beyond_32_bits(n, Hq, fmt):
    """Pages whose rows start beyond 2^32 bytes (and, in 8 bits, codes)."""
    c = wide(build(2, n, Hq, 1, 128, 128, 700, fmt, True, False, True))
    total = 2 ** 32 // (128 * 128 * (2 if fmt == "bf16" else 1)) + 40
    shift = total - c["n_pages"]
    big = {}
    for name in ("k", "v", "k_scale", "v_scale"):
        if c[name] is not None:
            big[name] = torch.empty((total, *c[name].shape[1:]), dtype=c[name].dtype, device="cuda")
            big[name][shift:] = c[name]
    want, want_lse, _ = call(c)
    check_attention(want, want_lse, c, "small pool", NO)
    out, lse, _ = call(dict(c, **big, table=torch.where(c["table"] >= 0, c["table"] + shift, -1), n_pages=total))
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("shape", [(1, 4, 1, 128, "bf16"), (8, 4, 1, 64, "row8")] + MANY, ids=lambda s: "-".join(map(str, s)))
def test_graph_whose_lengths_change_and_another_stream(shape):
    n, Hq, Hkv, D, fmt = shape
    c = wide(build(5, n, Hq, Hkv, D, 16, 900, fmt, True, True, True))
    full = c["len"].clone()
    out, lse, run = call(c)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run()
    side = torch.cuda.Stream()
    for cut in (0, 37, 2000, 5):
        c["len"].copy_((full - cut).clamp(min=0))
        out.fill_(NO); lse.fill_(NO)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out.fill_(NO); lse.fill_(NO)
            run()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, out) and torch.equal(got_lse, lse), cut
    c["len"].copy_(full)
    graph.replay()
    check_attention(out, lse, c, "replayed", NO)


def test_sequences_that_share_pages():
    """One prompt's pages in several sequences' tables: each attends its own copy of them."""
    c = wide(build(3, 16, 8, 2, 128, 16, 0, "bf16", True, False, True, lens=[480, 480, 480]))
    c["table"][1:, :29] = c["table"][0, :29]                                # 464 rows, the trees' rows are their own
    out, lse, _ = call(c)
    check_attention(out, lse, c, "shared", NO)


@pytest.mark.parametrize("gaps", [False, True], ids=["whole", "gaps"])
@pytest.mark.parametrize("n,Hq,Hkv,D,fmt", [(1, 512, 512, 64, "bf16"), (1, 512, 512, 128, "row8"), (24, 512, 512, 64, "row8"), (24, 256, 256, 64, "bf16"),
                                            (24, 256, 256, 128, "bf16"), (64, 256, 256, 64, "bf16"), (64, 256, 256, 128, "row8"),
                                            (64, 256, 128, 128, "bf16"), (64, 256, 128, 64, "row8")], ids=str)
def test_pieces_of_many_pages(n, Hq, Hkv, D, fmt, gaps):
    """A workgroup's piece of a sequence that spans several windows of 64 table entries: pages of 16 rows give what the same rows in
    pages of 256 do, bit for bit."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    B, big, lens = 2, 256, [4500 + n, 3111 + n]
    P = 2 * 20
    shape, c = (P, Hkv, big), {"B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "pos0": 3, "base": 1e4, "n_rows": None}
    for name in "kv":
        if fmt == "bf16":
            c[name], c[name + "_scale"] = torch.randn((*shape, D), generator=gen, device="cuda", dtype=torch.bfloat16), None
        else:
            c[name] = torch.randint(0, 127, (*shape, D), generator=gen, device="cuda", dtype=torch.uint8)
            c[name + "_scale"] = torch.rand(shape, generator=gen, device="cuda") / 200
    c["table"] = torch.randperm(P, generator=gen, device="cuda").to(torch.int32).view(B, 20)
    if gaps:
        c["table"][0, 9], c["table"][1, 2], c["table"][1, 10:] = -1, P, -1
    c["len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c["pos"] = c["len"] + 10
    c["parent"] = None
    c["q"] = torch.randn((B, n, Hq, D), generator=gen, device="cuda").to(torch.bfloat16)
    want, want_lse, _ = call(c)
    order = torch.randperm(16 * P, generator=gen, device="cuda")
    place = torch.empty_like(order)
    place[order] = torch.arange(16 * P, device="cuda")                      # small page -> where it lies now
    small = dict(c)
    for name in ("k", "v", "k_scale", "v_scale"):
        t = c[name]
        if t is not None:
            small[name] = t.view(P, Hkv, 16, 16, -1).transpose(1, 2).reshape(16 * P, Hkv, 16, *t.shape[3:])[order].contiguous()
    table = c["table"].long()
    there = (table >= 0) & (table < P)
    at = place[(table.clamp(0, P - 1)[..., None] * 16 + torch.arange(16, device="cuda")).view(B, -1)]
    small["table"] = torch.where(there.repeat_interleave(16, 1), at, -1).to(torch.int32)
    out, lse, _ = call(small)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert torch.isfinite(want.float()).all() and want.abs().sum() > 0
