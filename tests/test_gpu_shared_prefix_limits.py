"""SharedPrefixDecoder up to the last row of its tails: the step that fills them against 64 bits, the one behind it refused
with every cache as it was."""
import pytest
import torch

from paper_2502_14317_amd.layer import SharedPrefixDecoder
from serving import check_attention

pytestmark = pytest.mark.gpu

B, P, S, KT, CAP, HQ, HKV, D, BASE, POS0 = 4, 2, 2, 75, 34, 8, 2, 128, 1.0e4, 500


def mk(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)


def new_rows(gen, n):
    return mk(gen, B, n, HQ, D), mk(gen, B, n, HKV, D), mk(gen, B, n, HKV, D)


def check_step(dec, out, q, before, what):
    n = q.shape[1]
    c = {"B": B, "P": P, "nq": n, "Hq": HQ, "Hkv": HKV, "D": D, "q": q, "pos": before, "pos0": POS0, "base": BASE, "own": True,
         "per_head": 0, "seg_len": None, "tail_len": before + n, "tail": tuple(dec.tail), "prefix": (*dec.prefix, None, None)}
    check_attention(out, dec.lse.view(-1)[:B * HQ * n].view(B, HQ, n), c, what)


def test_the_last_rows_of_a_tail():
    gen = torch.Generator(device="cuda").manual_seed(3)
    dec = SharedPrefixDecoder(B, P, S, KT, CAP, HQ, HKV, D, BASE, POS0, max_rows=4)
    dec.load(mk(gen, P, S, HKV, KT, D), mk(gen, P, S, HKV, KT, D), k_tail=mk(gen, B, CAP - 5, HKV, D), v_tail=mk(gen, B, CAP - 5, HKV, D))
    for n in (3, 2):
        q, k, v = new_rows(gen, n)
        before = dec.len.clone()
        check_step(dec, dec.step(q, k, v), q, before, f"{n} rows")
        dec.accept()
    assert dec.len.tolist() == [CAP] * B
    held = [x.clone() for x in (*dec.tail, dec.len)]
    for n in (1, 4):
        with pytest.raises(ValueError, match="hold 34 rows"):
            dec.step(*new_rows(gen, n))
    assert all(torch.equal(x, y) for x, y in zip(held, (*dec.tail, dec.len)))


@pytest.mark.parametrize("drafts", [False, True], ids=["accepted", "verified"])
def test_a_graph_of_steps_goes_on(drafts):
    """One captured step, its rows accepted or verified: every replay writes behind the rows that stand, and equals steps that
    are called one by one."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, V = (3, 301) if drafts else (1, 0)
    doc, head = [mk(gen, P, S, HKV, KT, D) for _ in "kv"], [mk(gen, B, 5, HKV, D) for _ in "kv"]
    one, other = (SharedPrefixDecoder(B, P, S, KT, CAP, HQ, HKV, D, BASE, POS0, max_rows=n) for _ in range(2))
    for dec in (one, other):
        dec.load(*doc, k_tail=head[0], v_tail=head[1])
    rows = new_rows(gen, n)
    if drafts:
        import paper_2502_14317_amd as pc
        ws = pc.alloc_workspace(pc.pc_verify_drafts_workspace_bytes(B, n - 1, V))
        probs = lambda k: torch.softmax(torch.randn((B, k, V), generator=gen, device="cuda"), -1)
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
        args = dict(draft=i32(B, n - 1), draft_prob=probs(n - 1), target_prob=probs(n), u=torch.rand((B, n - 1), generator=gen, device="cuda"),
                    noise=torch.ones((B, V), device="cuda"), tokens=i32(B, n), n_accepted=i32(B), ws=ws)

    def go(dec):
        out = dec.step(*rows)
        dec.verify(**args) if drafts else dec.accept()
        return out
    go(one); go(other)                                                      # an eager step first
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = go(one)
    for i in range(4):
        for x in rows:
            x.copy_(mk(gen, *x.shape))                                      # eager work between the replays
        if drafts:
            args["draft"].copy_(torch.randint(0, V, (B, n - 1), generator=gen, device="cuda", dtype=torch.int32))
        before = one.len.clone()
        graph.replay()
        torch.cuda.synchronize()
        got, got_len = out.clone(), one.len.clone()
        want = go(other)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16)), i
        assert torch.equal(got_len, other.len) and (got_len > before).all(), i
        assert all(torch.equal(x, y) for x, y in zip(one.tail, other.tail)), i
    go(one); go(other)                                                      # and an eager one behind them
    assert torch.equal(one.len, other.len) and all(torch.equal(x, y) for x, y in zip(one.tail, other.tail))
    while int(one.len.max()) + n <= CAP:
        go(one)
    with pytest.raises(ValueError, match="hold 34 rows"):                   # (the replays moved the lengths unseen by the host)
        one.step(*rows)
