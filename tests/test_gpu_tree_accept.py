"""pc_tree_accept against its definition on the CPU: every number equal, every row where it belongs, every other bit as it was."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from trees import accept, build

pytestmark = pytest.mark.gpu

# B, n, H_kv, D, page, rows in front (at most), format, tree, ragged, different tokens
CASES = [
    (1, 1, 1, 64, 16, 0, "bf16", False, False, 5),
    (4, 5, 8, 128, 16, 40, "bf16", True, False, 1),
    (7, 64, 3, 128, 16, 90, "row8", True, True, 2),
    (9, 64, 2, 64, 32, 33, "row8", True, True, 3),
    (5, 64, 5, 64, 64, 70, "bf16", False, True, 1),                  # chains that stand: nothing moves
    (300, 9, 1, 128, 16, 30, "bf16", True, True, 2),
    (6, 33, 2, 128, 128, 300, "bf16", True, False, 1),
]


def call(c, tokens, choice, stride=1, cache=True, pos=None):
    i32 = lambda *s: torch.full(s, -9, dtype=torch.int32, device="cuda")
    path, kept, following, len_out = i32(c["B"], c["n"]), i32(c["B"]), i32(c["B"]), i32(c["B"])
    more = {}
    if cache:
        more = dict(cache=pc.make_page_cache(c["k"], c["v"], c["table"], c["k_scale"], c["v_scale"]), n_kv_heads=c["Hkv"], head_dim=c["D"],
                    len_in=c["len"], len_out=len_out)
    pc.pc_tree_accept(tokens, c["parent"], choice, c["B"], c["n"], path, kept, following, choice_stride=stride, pos=pos, n_rows=c["n_rows"], **more)
    return path, kept, following, len_out


def make(B, n, Hkv, D, page, most, fmt, tree, ragged, kinds):
    c = build(B, n, Hkv, Hkv, D, page, most, fmt, tree, ragged, False)
    gen = torch.Generator(device="cuda").manual_seed(n + kinds)
    draw = lambda: torch.randint(0, kinds, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    return c, draw(), draw()


def check(c, tokens, choice, start, got, pos=None, what="accept"):
    path, kept, following, moves = accept(c, tokens.tolist(), choice.tolist())
    for x, y, name in zip(got, (path, kept, following), ("path", "n_kept", "next_token")):
        assert np.array_equal(x.cpu().numpy(), y), f"{what}: {name}"
    rows = [c["n"] if c["n_rows"] is None else int(c["n_rows"][b]) for b in range(c["B"])]
    assert got[3].tolist() == [int(n) - r + int(k) for n, r, k in zip(c["len"], rows, kept)], f"{what}: lengths"
    if pos is not None:
        assert pos.tolist() == [100 + 3 * b + int(k) for b, k in enumerate(kept)], f"{what}: positions"
    for name, before in start.items():
        want = before.clone()
        for line in moves:
            for frm, to in line:
                if frm is not None and to is not None:
                    want[to[0], :, to[1]] = before[frm[0], :, frm[1]]
        assert torch.equal(want.view(torch.uint8), c[name].view(torch.uint8)), f"{what}: {name}"
    return kept


def pools(c):
    return {x: c[x].clone() for x in ("k", "v", "k_scale", "v_scale") if c[x] is not None}


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_the_definition(case):
    print("accept", case, flush=True)
    c, tokens, choice = make(*case)
    start, pos = pools(c), 100 + 3 * torch.arange(c["B"], dtype=torch.int32, device="cuda")
    check(c, tokens, choice, start, call(c, tokens, choice, pos=pos), pos)


def test_paths_of_every_length():
    """A bush whose path takes every other node: every row of it moves over one that a later row comes from."""
    c, tokens, choice = make(8, 64, 2, 128, 16, 50, "bf16", True, False, 1)
    up = [-1] + [max(0, (t - 1) // 2 * 2) for t in range(1, 64)]             # 1, 2 below 0; 3, 4 below 2; ..
    c["parent"].copy_(torch.tensor(up, dtype=torch.int32).expand(8, 64))
    tokens.copy_(torch.arange(64, device="cuda") % 2)                       # even nodes have token 0
    choice.zero_()
    for b in range(8):
        choice[b, 8 * b:] = 1 if b < 4 else 5
    kept = check(c, tokens, choice, pools(c), call(c, tokens, choice))
    assert len(set(kept.tolist())) == 8 and max(kept) > 28


def test_choices_with_a_stride_parents_anywhere_and_no_cache():
    c, tokens, choice = make(5, 12, 2, 64, 16, 20, "bf16", True, True, 2)
    c["parent"][0] = torch.tensor([3, 0, 1, 2 ** 31 - 1, -2, 0, 11, 6, 8, 2, 5, -1])
    wide = torch.full((5, 12, 7), -1, dtype=torch.int32, device="cuda")
    wide[:, :, 0] = choice
    start = pools(c)
    alone = call(c, tokens, wide, stride=7, cache=False)
    assert all(torch.equal(start[x].view(torch.uint8), c[x].view(torch.uint8)) for x in start) and (alone[3] == -9).all()
    got = call(c, tokens, wide, stride=7)
    check(c, tokens, choice, start, got)
    assert all(torch.equal(x, y) for x, y in zip(alone[:3], got[:3]))


def test_pages_that_are_not_there():
    c, tokens, choice = make(3, 40, 2, 64, 16, 30, "row8", True, False, 1)
    c["table"][0, int(c["len"][0] - 10) // 16] = -1
    c["table"][1, int(c["len"][1] - 38) // 16] = c["n_pages"]
    c["table"] = c["table"][:, :3].contiguous()
    check(c, tokens, choice, pools(c), call(c, tokens, choice))


def test_graph_goes_on_from_replay_to_replay():
    c, tokens, choice = make(4, 6, 2, 128, 16, 0, "bf16", True, False, 1)
    c["len"].fill_(6)
    cache = pc.make_page_cache(c["k"], c["v"], c["table"], c["k_scale"], c["v_scale"])
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    path, kept, following, out, pos = i32(4, 6), i32(4), i32(4), i32(4), i32(4)
    run = lambda: pc.pc_tree_accept(tokens, c["parent"], choice, 4, 6, path, kept, following, cache=cache, n_kv_heads=2, head_dim=128,
                                    len_in=c["len"], len_out=out, pos=pos)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run()
    start, total = pools(c), np.zeros(4, int)
    for _ in range(3):
        for name, t in start.items():
            c[name].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        total += check(c, tokens, choice, start, (path, kept, following, out))
        assert pos.tolist() == total.tolist()
