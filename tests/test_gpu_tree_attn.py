"""pc_tree_attn against 64 bits on the CPU: head layouts, formats, page sizes, trees of one node to 64, lengths of zero and one,
odd sizes, strides, rows that see nothing, pages that are not there, infinities and NaN where nobody looks, offsets beyond 32
bits, other streams, graphs."""
import pytest
import torch

import paper_2502_14317_amd as pc
from trees import build, check_attention

pytestmark = pytest.mark.gpu

# B, n, H_q, H_kv, D, page, most rows in front, format, tree, ragged, rotate
CASES = [
    (1, 1, 4, 4, 128, 16, 1, "bf16", False, False, False),
    (2, 1, 8, 8, 64, 16, 90, "bf16", False, False, True),
    (5, 1, 32, 8, 128, 64, 700, "bf16", False, True, True),
    (4, 1, 28, 4, 128, 32, 333, "row8", False, False, True),
    (3, 2, 6, 2, 64, 16, 100, "row8", True, False, False),
    (6, 7, 7, 7, 128, 32, 210, "bf16", True, True, True),
    (4, 8, 8, 2, 128, 128, 150, "bf16", True, False, False),         # 32 rows a KV head
    (5, 16, 12, 4, 64, 16, 500, "row8", True, True, True),           # 48 rows
    (3, 16, 8, 2, 128, 64, 1100, "bf16", True, True, True),          # 64 rows
    (2, 33, 14, 2, 64, 256, 300, "bf16", True, False, True),         # 231 rows
    (3, 64, 4, 2, 128, 16, 130, "row8", True, True, True),           # 128 rows
    (2, 64, 16, 1, 64, 32, 77, "bf16", True, False, False),          # 1024 rows
    (2, 64, 3, 3, 128, 16, 0, "bf16", True, True, True),             # nothing but the trees
    (40, 3, 4, 1, 128, 16, 60, "row8", True, True, False),
    (300, 1, 2, 1, 64, 16, 40, "bf16", False, True, True),           # more sequences than threads
    (1, 5, 8, 2, 128, 64, 20000, "row8", True, False, True),         # one long sequence
]
NO = -77.0                                                                  # where nothing may be written


def call(c, lse=True):
    B, n, Hq, D = c["B"], c["n"], c["Hq"], c["D"]
    cache = pc.make_page_cache(c["k"], c["v"], c["table"], c["k_scale"], c["v_scale"])
    out = torch.full((B, n, Hq, D), NO, dtype=torch.bfloat16, device="cuda")
    ls = torch.full((B, Hq, n), NO, dtype=torch.float32, device="cuda") if lse else None
    sizes = (B, n, Hq, c["Hkv"], D)
    ws = pc.alloc_workspace(pc.pc_tree_attn_workspace_bytes(cache, *sizes))
    ws.fill_(255)                                                           # NaN where nothing has been written
    run = lambda: pc.pc_tree_attn(c["q"], cache, c["len"], *sizes, out, ls, ws, parent=c["parent"], n_rows=c["n_rows"], pos=c["pos"],
                                  pos0=c["pos0"], rope_base=c["base"], softmax_scale=c.get("scale", 0.0))
    run()
    return out, ls, run


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_64_bits(case):
    print("tree attention", case, flush=True)
    c = build(*case)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "tree attention", NO)


def test_empty_sequences_and_single_rows():
    c = build(5, 2, 8, 2, 128, 16, 0, "bf16", False, False, True, lens=[2, 2, 33, 2, 18])
    c["len"].copy_(torch.tensor([0, 1, 33, -4, 18]))                        # 0, -4: nothing is there; 1: only node 1's row is
    out, lse, _ = call(c)
    check_attention(out, lse, c, "few rows", NO)
    assert not out[0].any() and torch.isneginf(lse[0]).all() and not out[1, 0].any() and out[1, 1].any()


def test_pages_that_are_not_there():
    c = build(4, 3, 4, 2, 64, 16, 0, "row8", True, False, True, lens=[100, 64, 90, 300])
    t = c["table"]
    t[0, 1], t[0, 4] = -1, c["n_pages"]                                     # in the middle of a sequence
    t[1] = -5                                                               # all of one
    t[2, 5] = 2 ** 31 - 1                                                   # the tree's own
    c["table"] = t[:, :18].contiguous()                                     # 300 rows, 288 of them have pages
    out, lse, _ = call(c)
    check_attention(out, lse, c, "pages", NO)
    assert not out[1].any() and torch.isneginf(lse[1]).all()


def test_parents_outside_of_the_tree_are_roots():
    c = build(2, 9, 4, 2, 64, 16, 40, "bf16", True, False, True)
    c["parent"][0] = torch.tensor([-1, 0, 7, 1, 2 ** 31 - 1, 5, -2 ** 31, 6, 8])       # later nodes, itself, anything
    out, lse, _ = call(c)
    check_attention(out, lse, c, "parents", NO)


@pytest.mark.parametrize("fmt", ["bf16", "row8"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")], ids=str)
def test_what_a_node_does_not_see_stays_out(fmt, bad):
    """A node's row that is not finite belongs to it and to those below it."""
    c = build(3, 6, 8, 2, 128, 16, 70, fmt, True, False, False)
    c["parent"].copy_(torch.tensor([-1, 0, 0, 1, 2, 2]))
    clean, clean_lse, _ = call(c)
    for b in range(3):
        j = int(c["len"][b]) - 6 + 2                                        # node 2: below it 4 and 5
        at = (int(c["table"][b, j // 16]), slice(None), j % 16)
        if fmt == "bf16":
            c["v"][at] = bad
        elif bad != bad:
            c["v"][at] = 0x7f
        else:
            c["v_scale"][at] = bad
    out, lse, _ = call(c)
    seen, unseen = [2, 4, 5], [0, 1, 3]
    assert torch.equal(out[:, unseen], clean[:, unseen]) and torch.equal(lse, clean_lse)
    assert not torch.isfinite(out[:, seen].float()).any()
    if fmt == "bf16":
        assert (out[:, seen].isnan().all() if bad != bad else (out[:, seen].float() == bad).all())


def test_keys_that_are_not_finite():
    c = build(2, 4, 4, 2, 64, 32, 50, "bf16", True, False, False)
    c["parent"].copy_(torch.tensor([-1, 0, 0, 1]))
    clean, clean_lse, _ = call(c)
    for b in range(2):
        j = int(c["len"][b]) - 4 + 2
        c["k"][int(c["table"][b, j // 32]), :, j % 32] = float("nan")
    out, lse, _ = call(c)
    assert torch.equal(out[:, [0, 1, 3]], clean[:, [0, 1, 3]]) and torch.equal(lse[:, :, [0, 1, 3]], clean_lse[:, :, [0, 1, 3]])
    assert out[:, 2].isnan().all()


def test_strides_a_scale_and_no_logsumexp():
    c = build(3, 5, 8, 2, 64, 16, 120, "bf16", True, False, True)
    packed = torch.full((3, 5, 12, 64), float("nan"), dtype=torch.bfloat16, device="cuda")        # q, k, v of one projection
    packed[:, :, :8] = c["q"]
    c["q"], c["scale"] = packed[:, :, :8], 0.21
    out, _, _ = call(c, lse=False)
    check_attention(out, None, c, "packed", NO)


def test_large_logits():
    """Logits of a deviation of 40 and more: the softmax is one row's."""
    c = build(3, 6, 4, 2, 128, 16, 300, "bf16", True, False, True, gain=7.0)
    out, lse, _ = call(c)
    check_attention(out, lse, c, "large logits", NO)


@pytest.mark.parametrize("fmt", ["bf16", "row8"])
def test_pools_beyond_32_bits(fmt):
    """Pages whose rows start beyond 2^32 bytes (and, in 8 bits, codes)."""
    c = build(2, 3, 4, 4, 128, 128, 200, fmt, True, False, True)
    n = 2 ** 32 // (4 * 128 * 128 * (2 if fmt == "bf16" else 1)) + 40
    shift = n - c["n_pages"]
    big = {}
    for name in ("k", "v", "k_scale", "v_scale"):
        if c[name] is not None:
            big[name] = torch.empty((n, *c[name].shape[1:]), dtype=c[name].dtype, device="cuda")
            big[name][shift:] = c[name]
    want, want_lse, _ = call(c)
    check_attention(want, want_lse, c, "small pool", NO)
    out, lse, _ = call(dict(c, **big, table=torch.where(c["table"] >= 0, c["table"] + shift, -1), n_pages=n))
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_same_bits_again_and_on_another_stream():
    c = build(7, 9, 16, 4, 128, 16, 900, "bf16", True, True, True)
    out, lse, run = call(c)
    first, first_lse = out.clone(), lse.clone()
    run()
    assert torch.equal(out, first) and torch.equal(lse, first_lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.fill_(NO); lse.fill_(NO)
        run()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, first) and torch.equal(lse, first_lse)


def test_graph_whose_lengths_grow():
    c = build(4, 4, 8, 2, 128, 16, 400, "row8", True, True, True)
    full = c["len"].clone()
    out, lse, run = call(c)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run()
    for cut in (0, 37, 1000, 5):
        c["len"].copy_((full - cut).clamp(min=0))
        out.fill_(NO); lse.fill_(NO)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        out.fill_(NO); lse.fill_(NO)
        run()
        assert torch.equal(got, out) and torch.equal(got_lse, lse), cut
    c["len"].copy_(full)
    graph.replay()
    check_attention(out, lse, c, "replayed", NO)


def test_two_workspaces_on_two_streams():
    cs = [build(6, 5, 8, 2, 128, 32, 600, "bf16", True, True, True, seed=s) for s in (1, 2)]
    want = [call(c)[:2] for c in cs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cs], []
    for _ in range(3):
        for c, st in zip(cs, streams):
            with torch.cuda.stream(st):
                got.append(call(c)[:2])
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(l, want[i % 2][1])
