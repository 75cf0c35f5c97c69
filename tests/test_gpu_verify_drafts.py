"""pc_verify_drafts against the definition, one 32-bit operation at a time on the CPU: every number equal."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from serving import verify

pytestmark = pytest.mark.gpu


def build(B, k, V, seed, near=0.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    logits = 2 * torch.randn((B, k + 1, V), generator=gen, device="cuda")
    target = torch.softmax(logits, -1)
    draft_prob = torch.softmax(logits[:, :k] + near * torch.randn((B, k, V), generator=gen, device="cuda"), -1)
    noise = torch.empty((B, V), device="cuda").exponential_(generator=gen)
    if k:
        draft = (draft_prob / torch.empty((B, k, V), device="cuda").exponential_(generator=gen)).argmax(-1).int()
    else:
        draft = torch.zeros((B, 0), dtype=torch.int32, device="cuda")
    u = torch.rand((B, k), generator=gen, device="cuda")
    return draft, draft_prob, target, u, noise


def call(draft, draft_prob, target, u, noise, draft_len=None, lens=None):
    B, k, V = draft.shape[0], draft.shape[1], target.shape[2]
    tokens = torch.full((B, k + 1), -9, dtype=torch.int32, device="cuda")
    count = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    ws = pc.alloc_workspace(pc.pc_verify_drafts_workspace_bytes(B, k, V))
    ws.fill_(255)
    pc.pc_verify_drafts(draft, draft_prob, target, u, noise, B, k, V, tokens, count, ws, draft_len=draft_len,
                        len_in=lens, len_out=lens)
    return tokens, count


def check(args, draft_len=None, what=""):
    lens = torch.arange(args[0].shape[0], dtype=torch.int32, device="cuda") * 7
    tokens, count = call(*args, draft_len=draft_len, lens=lens)
    cpu = [None if x is None else x.cpu().numpy() for x in args]
    want, want_count = verify(*cpu, draft_len=None if draft_len is None else draft_len.cpu().numpy())
    assert np.array_equal(count.cpu().numpy(), want_count), what
    assert np.array_equal(tokens.cpu().numpy(), want), what
    assert np.array_equal(lens.cpu().numpy(), np.arange(len(want_count)) * 7 + 1 + want_count), what
    return want, want_count


@pytest.mark.parametrize("B,k,V", [(1, 1, 1), (1, 4, 32000), (3, 0, 50), (7, 8, 1023), (64, 3, 4097), (2, 5, 128256), (600, 2, 65)])
@pytest.mark.parametrize("point", [False, True], ids=["drawn", "point"])
def test_against_the_definition(B, k, V, point):
    print("verify", B, k, V, point, flush=True)
    args = list(build(B, k, V, B + k + V))
    if point:
        args[1] = None
    want, count = check(args)
    gen = torch.Generator(device="cuda").manual_seed(1)
    check(args, torch.randint(-2, k + 3, (B,), generator=gen, device="cuda", dtype=torch.int32), "lengths")


def test_all_stand_and_none_stands():
    draft, dp, tp, u, noise = build(5, 6, 777, 3)
    _, count = check((draft, dp, tp, torch.zeros_like(u), noise), what="u = 0")
    assert (count == 6).all()
    _, count = check((draft, dp, dp.new_zeros(tp.shape).index_fill_(2, torch.tensor([5], device="cuda"), 1.0), u, noise), what="no mass on the drafts")


def test_more_drafts_than_lanes():
    draft, dp, tp, u, noise = build(3, 150, 97, 9, near=0.02)
    u *= 0.9
    _, count = check((draft, dp, tp, u, noise))
    u.zero_()
    _, count = check((draft, dp, tp, u, noise))
    assert (count == 150).all()


def test_ties_go_to_the_lowest_token():
    B, V = 2, 5000
    tp = torch.zeros((B, 1, V), device="cuda")
    tp[0, 0, [4999, 17, 3000]] = 0.25
    tp[1, 0, 1024:] = 2.0 ** -12
    noise = torch.ones((B, V), device="cuda")
    args = (torch.zeros((B, 0), dtype=torch.int32, device="cuda"), None, tp, torch.zeros((B, 0), device="cuda"), noise)
    want, _ = check(args)
    assert want[:, 0].tolist() == [17, 1024]


def test_edges():
    draft, dp, tp, u, noise = build(6, 2, 300, 11)
    draft[0, 0], draft[1, 1] = -1, 300                                      # outside the vocabulary
    u[2] = 1.0
    dp[2] = tp[2, :2]                                                       # p = q: nothing is left where u q < p fails
    tp[3, 0] = float("nan")
    noise[4, :150] = 0.0                                                    # infinite quotients: the lowest of them
    tp[5] = 0.0                                                             # no mass at all
    want, count = check((draft, dp, tp, u, noise))
    assert count[0] == 0 and count[2] == 0 and want[5, 0] == -1
    check((draft, None, tp, u, noise), what="point mass")


def test_a_graph_replays():
    args = build(8, 4, 3001, 21)
    B, k, V = 8, 4, 3001
    tokens, count = torch.empty((B, k + 1), dtype=torch.int32, device="cuda"), torch.empty((B,), dtype=torch.int32, device="cuda")
    ws = pc.alloc_workspace(pc.pc_verify_drafts_workspace_bytes(B, k, V))
    run = lambda: pc.pc_verify_drafts(*args, B, k, V, tokens, count, ws)
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        args[3].copy_(torch.rand((B, k), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want, want_count = verify(*[x.cpu().numpy() for x in args])
        assert np.array_equal(tokens.cpu().numpy(), want) and np.array_equal(count.cpu().numpy(), want_count), i
