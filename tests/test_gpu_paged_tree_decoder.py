"""PagedTreeDecoder: append, attention, log probabilities and acceptance together, step after step, against 64 bits over the
rows that stand; pages taken as sequences grow and given back; a captured run of steps."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from paper_2502_14317_amd.layer import PagedTreeDecoder
from serving import f64, rotate
from trees import random_tree

pytestmark = pytest.mark.gpu

Hq, Hkv, D, BASE = 8, 2, 64, 1e4


class Rows:
    """A sequence's rows that stand, in 64 bits: rotated keys and values."""

    def __init__(self):
        self.k, self.v, self.pos = np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D)), 0


def attend(rows, q, k, v, lines, t, n_rows):
    """Node t's result [Hq, D]; lines: every node's way up."""
    depth = [len(x) - 1 for x in lines]
    seen = lines[t]
    keys = np.concatenate([rows.k, rotate(k, rows.pos + np.array(depth), BASE)[seen]])
    vals = np.concatenate([rows.v, v[seen]])
    qt = rotate(q[t:t + 1], [rows.pos + depth[t]], BASE)[0]
    out = np.zeros((Hq, D))
    for h in range(Hq):
        x = keys[:, h // (Hq // Hkv)] @ qt[h] / D ** 0.5
        p = np.exp(x - x.max())
        out[h] = p / p.sum() @ vals[:, h // (Hq // Hkv)]
    return out


def ways(up, n):
    lines = []
    for t in range(n):
        line = [t]
        while 0 <= up[line[-1]] < line[-1]:
            line.append(up[line[-1]])
        lines.append(line)
    return lines


@pytest.mark.parametrize("eight_bit", [False, True], ids=["bf16", "row8"])
def test_steps_of_trees_against_64_bits(eight_bit):
    B, n, V, gen = 3, 9, 50, torch.Generator(device="cuda").manual_seed(3)
    rng = np.random.default_rng(5)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    d = PagedTreeDecoder(B, 40, 16, 14, Hq, Hkv, D, BASE, max_rows=n, eight_bit=eight_bit)
    all_rows = [Rows() for _ in range(B)]
    for b, segs in enumerate((2, 1, 3)):
        kc, vc = mk(segs, Hkv, 30, D), mk(segs, Hkv, 30, D)
        kt, vt = mk(4, Hkv, D), mk(4, Hkv, D)
        lens = [30 - 7 * s for s in range(segs)]
        d.load(b, kc, vc, 500 + b, seg_len=lens, k_tail=kt, v_tail=vt)
        r = all_rows[b]
        r.k = np.concatenate([f64(kc)[s, :, :m].transpose(1, 0, 2) for s, m in enumerate(lens)] + [f64(kt)])
        r.v = np.concatenate([f64(vc)[s, :, :m].transpose(1, 0, 2) for s, m in enumerate(lens)] + [f64(vt)])
        r.pos = 500 + b
    ws = pc.alloc_workspace(pc.pc_token_logprobs_workspace_bytes(B * n, V, 3))
    kept_in_all = 0
    for step in range(12):
        m = int(rng.integers(1, n + 1))
        up = [[-1] + [max(0, x) for x in random_tree(rng, m)[1:]] for _ in range(B)]
        n_rows = [int(rng.integers(1, m + 1)) for _ in range(B)]
        if step == 4:
            n_rows[1] = 0                                                   # a sequence that does not take part
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        parent, rows_t = i32(up), i32(n_rows)
        qkv = mk(B, m, Hq + 2 * Hkv, D)                                     # one projection's rows
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        out = d.step(q, k, v, parent=parent, n_rows=rows_t)
        got, q64, k64, v64 = f64(out), f64(q), f64(k), f64(v)
        # a row: 2^-8 of the output's and the probabilities' roundings, 2^-8 of a key's (16 bits), a logit's error times 2 on the
        # probabilities; 8 bits: 2^-4 a value instead.  As a share of the norm those average out below a tenth and a hundredth
        for b in range(B):
            lines = ways(up[b], m)
            for t in range(n_rows[b]):
                want = attend(all_rows[b], q64[b], k64[b], v64[b], lines, t, n_rows[b])
                rel = np.linalg.norm(got[b, t] - want) / np.linalg.norm(want)
                assert rel < (0.1 if eight_bit else 0.015), (step, b, t, rel)
        # the caller's logits behind every node: three tokens each, so that drafts stand now and then
        tokens = i32(rng.integers(0, 3, (B, m)).tolist())
        logits = mk(B * m, V)
        logits[:, :3] += 8
        top, lp = torch.empty((B, m, 3), dtype=torch.int32, device="cuda"), torch.empty((B * m, 1), device="cuda")
        pc.pc_token_logprobs(logits, B * m, V, tokens, 1, 3, lp, None, top, None, ws)
        want_lp = torch.log_softmax(logits.double(), 1).gather(1, tokens.view(-1, 1).long())
        assert torch.allclose(lp.double(), want_lp, rtol=0, atol=2e-5)
        path, n_kept, following = d.accept(tokens, top, choice_stride=3)
        choice = logits.float().view(B, m, V).argmax(2).tolist()
        for b in range(B):
            line = [0] if n_rows[b] else []
            while line:
                nxt = choice[b][line[-1]]
                below = [c for c in range(line[-1] + 1, n_rows[b]) if up[b][c] == line[-1] and int(tokens[b, c]) == nxt]
                if not below:
                    assert int(following[b]) == nxt
                    break
                line.append(below[0])
            assert path[b].tolist() == line + [-1] * (m - len(line)) and int(n_kept[b]) == len(line)
            r = all_rows[b]
            depth = [len(x) - 1 for x in ways(up[b], m)]
            r.k = np.concatenate([r.k, rotate(k64[b], r.pos + np.array(depth), BASE)[line]])
            r.v = np.concatenate([r.v, v64[b][line]])
            r.pos += len(line)
            kept_in_all += len(line)
            assert int(d.len[b]) == len(r.k) and int(d.pos[b]) == r.pos
    assert kept_in_all > 12 * B                                             # (drafts stood)


def test_pages_go_round():
    B, page = 2, 16
    mk = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")
    d = PagedTreeDecoder(B, 6, page, 5, Hq, Hkv, D, BASE, max_rows=4)
    d.load(0, mk(1, Hkv, 30, D), mk(1, Hkv, 30, D), 30)
    with pytest.raises(ValueError, match="not loaded"):
        d.step(mk(B, 1, Hq, D), mk(B, 1, Hkv, D), mk(B, 1, Hkv, D))
    with pytest.raises(ValueError, match="pages"):
        d.load(1, mk(1, Hkv, 65, D), mk(1, Hkv, 65, D), 65)                 # four are free
    d.load(1, mk(1, Hkv, 20, D), mk(1, Hkv, 20, D), 20)
    one = torch.zeros((B, 4), dtype=torch.int32, device="cuda")
    steps = 0
    with pytest.raises(ValueError, match="do not fit"):
        for steps in range(100):                                            # chains that stand: four rows a step each
            d.step(mk(B, 4, Hq, D), mk(B, 4, Hkv, D), mk(B, 4, Hkv, D))
            d.accept(one, one)
    assert d.len.tolist() == [30 + 4 * steps, 20 + 4 * steps] and steps == 4
    d.release(1)
    assert len(d.free) == 3 and (d.table[1] == -1).all() and int(d.len[1]) == 0
    only = torch.tensor([4, 0], dtype=torch.int32, device="cuda")
    for _ in range(5):
        d.step(mk(B, 4, Hq, D), mk(B, 4, Hkv, D), mk(B, 4, Hkv, D), n_rows=only)
        d.accept(one, one)
    assert d.len.tolist() == [66, 0]
    d.load(1, mk(1, Hkv, 16, D), mk(1, Hkv, 16, D), 16)
    used = d.pages[0] + d.pages[1]
    assert len(set(used + d.free)) == 6 and d.table[0, :5].tolist() == d.pages[0]


def test_drafts_that_never_stand_take_no_pages():
    mk = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")
    d = PagedTreeDecoder(1, 3, 16, 3, Hq, Hkv, D, BASE, max_rows=8)
    d.load(0, mk(1, Hkv, 4, D), mk(1, Hkv, 4, D), 4)
    tokens, choice = torch.zeros((1, 8), dtype=torch.int32, device="cuda"), torch.ones((1, 8), dtype=torch.int32, device="cuda")
    for _ in range(20):
        d.step(mk(1, 8, Hq, D), mk(1, 8, Hkv, D), mk(1, 8, Hkv, D))
        d.accept(tokens, choice)
    assert d.len.tolist() == [24] and len(d.pages[0]) == 2


def test_a_captured_step_goes_on():
    gen = torch.Generator(device="cuda").manual_seed(9)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    B, n = 2, 3
    kc, vc = mk(2, Hkv, 20, D), mk(2, Hkv, 20, D)
    data = [(mk(B, n, Hq, D), mk(B, n, Hkv, D), mk(B, n, Hkv, D)) for _ in range(6)]
    parent = torch.tensor([[-1, 0, 0], [-1, 0, 1]], dtype=torch.int32, device="cuda")
    tokens = torch.tensor([[9, 1, 2], [9, 1, 2]], dtype=torch.int32, device="cuda")
    choice = torch.tensor([[2, 0, 4], [1, 2, 5]], dtype=torch.int32, device="cuda")
    made = [PagedTreeDecoder(B, 20, 16, 8, Hq, Hkv, D, BASE, max_rows=n) for _ in range(2)]
    for d in made:
        for b in range(B):
            d.load(b, kc, vc, 40)
    eager, d = made
    want = []
    for q, k, v in data:
        want.append(eager.step(q, k, v, parent=parent).clone())
        eager.accept(tokens, choice)
    q, k, v = (t.clone() for t in data[0])
    for b in range(B):
        d.reserve(b, 40 + 6 * n)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = d.step(q, k, v, parent=parent)
        d.accept(tokens, choice)
    for (a, b, c), w in zip(data, want):
        q.copy_(a); k.copy_(b); v.copy_(c)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)
    assert d.len.tolist() == eager.len.tolist() == [40 + 6 * 2, 40 + 6 * 3]
    d.step(*data[0], parent=parent)                                         # an eager step reads the lengths that the replays left
    assert d.most == d.len.tolist()


def test_a_step_behind_a_load_or_release_is_dropped():
    """Between a step and its acceptance a sequence's lengths may not become another's."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    d = PagedTreeDecoder(2, 12, 16, 4, Hq, Hkv, D, BASE, max_rows=2)
    docs = [mk(1, Hkv, 20, D) for _ in range(3)]
    d.load(0, docs[0], docs[0], 20)
    d.load(1, docs[1], docs[1], 20)
    q, k, v = mk(2, 2, Hq, D), mk(2, 2, Hkv, D), mk(2, 2, Hkv, D)
    tokens = torch.ones((2, 2), dtype=torch.int32, device="cuda")
    want = d.step(q, k, v).clone()
    d.load(1, docs[2], docs[2], 33)
    with pytest.raises(ValueError, match="no step"):
        d.accept(tokens, tokens)
    assert d.len.tolist() == [20, 20] and d.pos.tolist() == [20, 33]
    out = d.step(q, k, v)
    assert torch.equal(out[0], want[0]) and not torch.equal(out[1], want[1])
    d.release(1)
    with pytest.raises(ValueError, match="no step"):
        d.accept(tokens, tokens)
    assert d.len.tolist() == [20, 0]
    one = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    assert torch.equal(d.step(q, k, v, n_rows=one)[0], want[0])
    d.accept(tokens, tokens)
    assert d.len.tolist() == [22, 0] and d.pos.tolist() == [22, 0]
