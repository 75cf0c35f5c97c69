"""Drafted trees over a paged cache, and what tokens are worth, as measurable cases.

A case is a dict of plain sizes; `kind` names the operator:
  append    pc_kv_append_paged: keys (rotated on the way) and values into the pages of their sequences, 16 or 8 bits
  attn      pc_tree_attn: the nodes of a tree of drafted tokens over their sequence's pages and their own ancestors
  logprobs  pc_token_logprobs: log probabilities of given tokens, the entropy, the most likely tokens
  accept    pc_tree_accept: the path of a tree that the target's choices follow, its rows moved to where they stay

Where `own` is false, `run` computes the same in plain torch operations in 32 bits.  Inputs are drawn on the GPU from the
seed: unit-variance keys, values and queries (logits of deviation 1), sequences of unequal lengths from a third of the longest
on, pages in no order, trees in level order with random parents, vocabulary logits of deviation 2.
"""
import math
import random

import torch

own = False

BF16, F8 = torch.bfloat16, torch.float8_e4m3fn
BASE = 5e5                                                              # of the rotation
SHIFT = -1000                                                           # a row's position less its number: documents are compressed


# ------------------------------------------------------------------------------------------ cases
def _named(name, case):
    return dict(case, name=name) if name else case


def _append(name, batch, n, hkv, d, page, fmt="bf16", tree=False, ragged=False):
    return _named(name, {"kind": "append", "batch": batch, "n": n, "hkv": hkv, "d": d, "page": page, "fmt": fmt, "tree": tree,
                         "ragged": ragged})


def _attn(name, batch, n, hq, hkv, d, most, page, fmt="bf16", ragged=False, rotate=True):
    return _named(name, {"kind": "attn", "batch": batch, "n": n, "hq": hq, "hkv": hkv, "d": d, "most": most, "page": page,
                         "fmt": fmt, "ragged": ragged, "rotate": rotate})


def _logprobs(name, rows, vocab, dtype, tokens, top, pad=0):
    return _named(name, {"kind": "logprobs", "rows": rows, "vocab": vocab, "dtype": dtype, "tokens": tokens, "top": top, "pad": pad})


def _accept(name, batch, n, hkv, d, page, fmt="bf16", ragged=False):
    return _named(name, {"kind": "accept", "batch": batch, "n": n, "hkv": hkv, "d": d, "page": page, "fmt": fmt, "ragged": ragged})


def listed():
    return [
        # the next token of two short answers, a small model: launches and latency, not bytes
        _attn("attn_two_short", 2, 1, 8, 8, 64, 512, 16),
        # the next token of 32 answers over compressed documents of 4096 to 12288 rows
        _attn("attn_32_tokens", 32, 1, 32, 8, 128, 12288, 64),
        # sixteen answers, trees of 16 drafted tokens
        _attn("attn_trees", 16, 16, 32, 8, 128, 16640, 64),
        # long documents kept in 8 bits, trees of 32
        _attn("attn_trees_8bit", 8, 32, 32, 8, 128, 65536, 128, fmt="row8"),
        # a KV head for every query head, small trees of unequal sizes, lengths that end inside pages; the logsumexp goes to a
        # caller who joins further keys
        _attn("attn_trees_mha", 12, 7, 32, 32, 128, 4001, 32, ragged=True, rotate=False),
        # one layer's rows of sixteen trees
        _append("append_trees", 16, 16, 8, 128, 64, tree=True),
        # eight long prompts' rows into 8-bit pages
        _append("append_prompts_8bit", 8, 8192, 8, 128, 128, fmt="row8"),
        # the greedy choice at the nodes of a few small trees, the vocabulary of a Llama-2-shaped model
        _logprobs("logprobs_step", 16, 32000, "bf16", 0, 1),
        # drafts of 64 sequences with alternatives, the vocabulary of a Llama-3-shaped model, 32-bit logits
        _logprobs("logprobs_alternatives", 512, 128256, "fp32", 2, 20),
        # a prompt's tokens scored
        _logprobs("logprobs_prompt", 2048, 128256, "bf16", 1, 5),
        # four trees of five
        _accept("accept_four", 4, 5, 8, 128, 16),
        # 64 trees of 64
        _accept("accept_64", 64, 64, 8, 128, 64, fmt="row8", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "logprobs", "logprobs", "accept"])
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 32, 128), (32, 8, 128), (8, 8, 64), (16, 4, 128), (24, 8, 64), (28, 4, 128),
                             (16, 1, 64)])
    page, fmt, ragged = rng.choice([16, 16, 32, 64, 128, 256]), rng.choice(["bf16", "row8"]), rng.random() < 0.4
    if kind == "attn":
        largest = work(listed()[3])
        while True:
            n = rng.choice([1, 1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
            case = _attn(None, _log_int(rng, 1, 64), n, hq, hkv, d, n + _log_int(rng, 32, 65536), page, fmt, ragged, rng.random() < 0.7)
            w = work(case)
            if w["flops"] <= largest["flops"] and w["bytes"] <= 1.1e9:
                return case
    if kind == "append":
        n = _log_int(rng, 1, 8192)
        return _append(None, _log_int(rng, 1, max(1, min(64, 524288 // (n * hkv)))), n, hkv, d, page, fmt,
                       n <= 64 and rng.random() < 0.7, ragged)
    if kind == "logprobs":
        vocab = rng.randint(4000, 128256)
        return _logprobs(None, _log_int(rng, 1, min(2048, 260_000_000 // vocab)), vocab, rng.choice(["bf16", "fp32"]),
                         rng.randint(0, 4), rng.choice([0, 1, 1, 5, 20, rng.randint(2, 32)]), rng.choice([0, 0, rng.randint(1, 200)]))
    return _accept(None, _log_int(rng, 1, 64), _log_int(rng, 2, 64), hkv, d, page, fmt, ragged)


def _rows_of(case):
    """Nodes (rows) of every sequence: all n, or from a third of them on."""
    B, n = case["batch"], case["n"]
    return [n if not case.get("ragged") else max(1, n - (b * 7919 % B) * 2 * n // (3 * B)) for b in range(B)]


def _before_of(case):
    """Rows of every sequence in front of the new ones."""
    return [b * 7919 % 601 for b in range(case["batch"])]


def _lens_of(case):
    """Rows of every sequence's cache, from a third of the most on, its own nodes among them."""
    B, most = case["batch"], case["most"]
    return [max(r, most - (b * 104729 % B) * 2 * most // (3 * B)) for b, r in enumerate(_rows_of(case))]


def work(case):
    """Bytes and flops of one pass: every row that counts read once."""
    kind = case["kind"]
    if kind == "logprobs":
        size = 2.0 if case["dtype"] == "bf16" else 4.0
        return {"bytes": case["rows"] * (size * case["vocab"] + 8.0 * (case["tokens"] + case["top"]) + 4.0), "flops": 0.0}
    hkv, d = case["hkv"], case["d"]
    row, rows = {"bf16": 4.0 * d, "row8": 2.0 * d + 8.0}[case["fmt"]], sum(_rows_of(case))
    if kind == "append":
        return {"bytes": rows * hkv * (4.0 * d + row), "flops": 0.0}
    if kind == "accept":                                                # some three rows a sequence move
        return {"bytes": 12.0 * rows + 2.0 * min(3.0, case["n"] - 1.0) * case["batch"] * hkv * row, "flops": 0.0}
    keys = _lens_of(case)
    return {"bytes": hkv * row * sum(keys) + 4.0 * rows * case["hq"] * d,
            "flops": 4.0 * d * case["hq"] * sum(k * r for k, r in zip(keys, _rows_of(case)))}


# ------------------------------------------------------------------------------------------ inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda").to(BF16)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pages(gen, case, rows, fill):
    """A pool of pages [n_pages, hkv, page, d] and the table of sequences of that many rows: no page twice, none in order."""
    page, hkv, d = case["page"], case["hkv"], case["d"]
    need = [(r + page - 1) // page for r in rows]
    n_pages, width = sum(need) + 3, max(need) + 1
    order, table, at = torch.randperm(n_pages, generator=gen, device="cuda").int().tolist(), [], 0
    for n in need:
        table.append(order[at:at + n] + [-1] * (width - n))
        at += n
    s = {"table": _ints(table)}
    for name in ("k", "v"):
        if case["fmt"] == "bf16":
            s[name] = _normal(gen, n_pages, hkv, page, d) if fill else torch.zeros((n_pages, hkv, page, d), dtype=BF16, device="cuda")
            s[name + "_scale"] = None
        elif fill:
            s[name] = torch.empty((n_pages, hkv, page, d), dtype=torch.uint8, device="cuda")
            s[name + "_scale"] = torch.empty((n_pages, hkv, page), device="cuda")
            for p in range(0, n_pages, 256):                            # (a part at a time)
                x = _normal(gen, min(256, n_pages - p), hkv, page, d).float()
                scale = x.abs().amax(-1) / 448.0
                s[name][p:p + 256] = (x / scale[..., None]).to(F8).view(torch.uint8)
                s[name + "_scale"][p:p + 256] = scale
        else:
            s[name] = torch.zeros((n_pages, hkv, page, d), dtype=torch.uint8, device="cuda")
            s[name + "_scale"] = torch.zeros((n_pages, hkv, page), device="cuda")
    return s


def _tree(rng, n):
    """Parents of n nodes in level order: a level of up to 8 nodes, each below one of the level before."""
    parent, before = [-1], [0]
    while len(parent) < n:
        level = range(len(parent), min(n, len(parent) + rng.randint(2, 8)))
        parent += [rng.choice(before) for _ in level]
        before = list(level)
    return parent


def _followed(rng, parent):
    """A path from the root that the target follows.  No row of it lies where another one moves to, so that a pass can be
    repeated on its own result."""
    n = len(parent)
    while True:
        path = [0]
        for _ in range(rng.randint(0, 6)):
            below = [c for c in range(n) if parent[c] == path[-1]]
            if not below:
                break
            path.append(rng.choice(below))
        if all(p == j or p >= len(path) for j, p in enumerate(path)):
            return path


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = random.Random(int(seed))
    s, kind = {"case": case}, case["kind"]
    if kind == "logprobs":
        rows, V, dtype = case["rows"], case["vocab"], BF16 if case["dtype"] == "bf16" else torch.float32
        whole = torch.empty((rows, V + case["pad"]), dtype=dtype, device="cuda")
        for r in range(0, rows, 256):                                   # (a part at a time)
            whole[r:r + 256] = 2.0 * torch.randn((min(256, rows - r), V + case["pad"]), generator=gen, device="cuda")
        s["logits"] = whole[:, :V]
        new = lambda n, t: torch.empty((rows, n), dtype=t, device="cuda") if n else None
        s["tokens"] = torch.randint(0, V, (rows, case["tokens"]), generator=gen, device="cuda", dtype=torch.int32) if case["tokens"] else None
        s["logprob"], s["entropy"] = new(case["tokens"], torch.float32), torch.empty((rows,), device="cuda")
        s["top"], s["top_logprob"] = new(case["top"], torch.int32), new(case["top"], torch.float32)
        return s
    B, n, hkv, d = (case[k] for k in ("batch", "n", "hkv", "d"))
    rows = _rows_of(case)
    s["n_rows"] = _ints(rows) if case["ragged"] else None
    trees = [_tree(rng, n) for _ in range(B)] if n <= 64 and n > 1 else None
    s["parent"] = _ints(trees) if trees and (kind != "append" or case["tree"]) else None
    if kind == "append":
        before = _before_of(case)
        s["pages"] = _pages(gen, case, [x + r for x, r in zip(before, rows)], False)
        qkv = _normal(gen, B, n, 3 * hkv, d)                            # as one projection leaves them
        s["k_new"], s["v_new"] = qkv[:, :, hkv:2 * hkv], qkv[:, :, 2 * hkv:]
        s["len"], s["len_out"] = _ints(before), _ints([0] * B)
        s["pos"] = s["len"] + 7680
    elif kind == "attn":
        lens = _lens_of(case)
        s["pages"] = _pages(gen, case, lens, True)
        s["q"] = _normal(gen, B, n, case["hq"], d)
        s["len"] = _ints(lens)
        s["pos"] = (s["len"] - _ints(rows) + 7680 + SHIFT) if case["rotate"] else None
        s["out"] = torch.zeros((B, n, case["hq"], d), dtype=BF16, device="cuda")
        s["lse"] = None if case["rotate"] else torch.zeros((B, case["hq"], n), dtype=torch.float32, device="cuda")
    else:
        before = _before_of(case)
        s["pages"] = _pages(gen, case, [x + r for x, r in zip(before, rows)], True)
        token, choice = [[[rng.randrange(32000) for _ in range(n)] for _ in range(B)] for _ in range(2)]
        for b, parent in enumerate(trees):
            path = _followed(rng, parent[:rows[b]])
            for p, c in zip(path, path[1:]):
                choice[b][p] = token[b][c]
        s["tokens"], s["choice"] = _ints(token), _ints(choice)
        s["len"], s["len_out"] = _ints([x + r for x, r in zip(before, rows)]), _ints([0] * B)
        s["path"], s["count"], s["next"] = _ints([[0] * n] * B), _ints([0] * B), _ints([0] * B)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"append": _append_own, "attn": _attn_own, "logprobs": _logprobs_own, "accept": _accept_own}[kind](s)
    return {"append": _append_plain, "attn": _attn_plain, "logprobs": _logprobs_plain, "accept": _accept_plain}[kind](s)


def _some(**outputs):
    return {n: x for n, x in outputs.items() if x is not None}


def _pages_out(s):
    p = s["pages"]
    f8 = s["case"]["fmt"] == "row8"
    return _some(k=p["k"].view(F8) if f8 else p["k"], v=p["v"].view(F8) if f8 else p["v"], k_scale=p["k_scale"], v_scale=p["v_scale"])


def _cache(s):
    import paper_2502_14317_amd as pc
    if "cache" not in s:                                                # what a program makes with its pages
        p = s["pages"]
        s["cache"] = pc.make_page_cache(p["k"], p["v"], p["table"], p["k_scale"], p["v_scale"])
    return s["cache"]


def _append_own(s):
    import paper_2502_14317_amd as pc
    c = s["case"]
    pc.pc_kv_append_paged(s["k_new"], s["v_new"], c["batch"], c["n"], c["hkv"], c["d"], _cache(s), s["len"], s["len_out"],
                          pos=s["pos"], pos0=SHIFT, rope_base=BASE, parent=s["parent"], n_rows=s["n_rows"])
    return dict(_pages_out(s), len=s["len_out"])


def _attn_own(s):
    import paper_2502_14317_amd as pc
    c, cache = s["case"], _cache(s)
    sizes = (c["batch"], c["n"], c["hq"], c["hkv"], c["d"])
    if "ws" not in s:
        s["ws"] = pc.alloc_workspace(pc.pc_tree_attn_workspace_bytes(cache, *sizes))
    pc.pc_tree_attn(s["q"], cache, s["len"], *sizes, s["out"], s["lse"], s["ws"], parent=s["parent"], n_rows=s["n_rows"],
                    pos=s["pos"], rope_base=BASE)
    return _some(out=s["out"], lse=s["lse"])


def _logprobs_own(s):
    import paper_2502_14317_amd as pc
    c = s["case"]
    if "ws" not in s:
        s["ws"] = pc.alloc_workspace(pc.pc_token_logprobs_workspace_bytes(c["rows"], c["vocab"], c["top"]))
    pc.pc_token_logprobs(s["logits"], c["rows"], c["vocab"], s["tokens"], c["tokens"], c["top"], s["logprob"], s["entropy"],
                         s["top"], s["top_logprob"], s["ws"])
    return _some(logprob=s["logprob"], entropy=s["entropy"], top=s["top"], top_logprob=s["top_logprob"])


def _accept_own(s):
    import paper_2502_14317_amd as pc
    c = s["case"]
    pc.pc_tree_accept(s["tokens"], s["parent"], s["choice"], c["batch"], c["n"], s["path"], s["count"], s["next"], cache=_cache(s),
                      n_kv_heads=c["hkv"], head_dim=c["d"], len_in=s["len"], len_out=s["len_out"], n_rows=s["n_rows"])
    return dict(_pages_out(s), path=s["path"], count=s["count"], next=s["next"], len=s["len_out"])


# ------------------------------------------------------------------------------------------ the plain forms
def _ancestors(s):
    """[B, n, n]: is node j the node t or above it; and the depths [B, n]."""
    B, n = s["case"]["batch"], s["case"]["n"]
    at = torch.arange(n, device="cuda").expand(B, n)
    parent = (at - 1 if s["parent"] is None else s["parent"]).long()
    each, seen, depth = torch.arange(n, device="cuda"), torch.zeros((B, n, n), dtype=torch.bool, device="cuda"), -torch.ones_like(at)
    for _ in range(n):
        seen |= at[:, :, None] == each
        depth = depth + (at >= 0)
        at = torch.where(at >= 0, parent.gather(1, at.clamp(min=0)), -1)
    return seen, depth


def _rotated(x, at):
    """x [B, n, H, D] in 32 bits at positions at [B, n], dimension i with i + D / 2 (angles in 64 bits)."""
    half = x.shape[-1] // 2
    theta = BASE ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    angle = (at.double()[..., None] * theta)[:, :, None, :]
    cs, sn = angle.cos().float(), angle.sin().float()
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)


def _places(s, row):
    """Page and row in it of rows [B, n] of the sequences."""
    page = s["case"]["page"]
    return s["pages"]["table"].gather(1, row // page).long(), row % page


def _nodes_here(s):
    """Is node (or row) t one of its sequence's: [B, n]."""
    B, n = s["case"]["batch"], s["case"]["n"]
    t = torch.arange(n, device="cuda").expand(B, n)
    return t < (n if s["n_rows"] is None else s["n_rows"][:, None])


def _append_plain(s):
    c, p = s["case"], s["pages"]
    t = torch.arange(c["n"], device="cuda")
    depth = t if s["parent"] is None else _ancestors(s)[1]
    here = _nodes_here(s)
    at, row = _places(s, torch.where(here, s["len"][:, None] + t, 0))
    at, row = at[here], row[here]
    for name in ("k", "v"):
        x = s[name + "_new"].float()
        if name == "k":
            x = _rotated(x, s["pos"][:, None] + SHIFT + depth)
        x = x[here]                                                     # [rows, hkv, d]
        if c["fmt"] == "bf16":
            p[name][at, :, row] = x.to(BF16)
            continue
        top = x.abs().amax(-1)
        scale = torch.where(top > 0, top / 448.0, 1.0)
        p[name][at, :, row] = (x / scale[..., None]).clamp(-448.0, 448.0).to(F8).view(torch.uint8)
        p[name + "_scale"][at, :, row] = scale
    torch.add(s["len"], here.sum(1), out=s["len_out"])
    return dict(_pages_out(s), len=s["len_out"])


def _attn_plain(s):
    c, p = s["case"], s["pages"]
    n, hq, hkv, d, page = (c[k] for k in ("n", "hq", "hkv", "d", "page"))
    G = hq // hkv
    seen, depth = _ancestors(s)
    q = s["q"].float()
    if s["pos"] is not None:
        q = _rotated(q, s["pos"][:, None] + depth)
    q = q * d ** -0.5
    for b, (m, r) in enumerate(zip(_lens_of(c), _rows_of(c))):
        pages = p["table"][b, :(m + page - 1) // page].long()
        k, v = (p[x][pages] for x in ("k", "v"))                        # [pages, hkv, page, d]
        k, v = (x.float() if c["fmt"] == "bf16" else x.view(F8).float() * p[y][pages][..., None] for x, y in ((k, "k_scale"), (v, "v_scale")))
        k, v = (x.transpose(0, 1).reshape(hkv, -1, d)[:, :m] for x in (k, v))
        x = torch.matmul(q[b, :r].view(r, hkv, G, d).transpose(0, 1).reshape(hkv, r * G, d), k.transpose(1, 2).contiguous())
        x.view(hkv, r, G, m)[..., m - r:].masked_fill_(~seen[b, :r, None, :r], -math.inf)
        top = x.amax(-1)
        x.sub_(top[..., None]).exp_()
        total = x.sum(-1)
        o = torch.matmul(x, v.contiguous()) / total[..., None]
        s["out"][b, :r] = o.view(hkv, r, G, d).transpose(0, 1).reshape(r, hq, d).to(BF16)
        if s["lse"] is not None:
            s["lse"][b, :, :r] = (top + total.log()).view(hkv, r, G).transpose(1, 2).reshape(hq, r)
    return _some(out=s["out"], lse=s["lse"])


def _logprobs_plain(s):
    c, x = s["case"], s["logits"].float()
    top = x.amax(1, keepdim=True)
    lse = top + (x - top).exp().sum(1, keepdim=True).log()
    s["entropy"].copy_(-((x - lse).exp() * (x - lse)).sum(1))
    if c["tokens"]:
        s["logprob"].copy_(x.gather(1, s["tokens"].long()) - lse)
    if c["top"]:
        value, index = (y[:, :c["top"]] for y in x.sort(dim=1, descending=True, stable=True))
        s["top"].copy_(index)
        s["top_logprob"].copy_(value - lse)
    return _some(logprob=s["logprob"], entropy=s["entropy"], top=s["top"], top_logprob=s["top_logprob"])


def _accept_plain(s):
    c, p = s["case"], s["pages"]
    B, n = c["batch"], c["n"]
    here, each = _nodes_here(s), torch.arange(n, device="cuda")
    base = s["len"] - here.sum(1).int()
    at = torch.zeros((B,), dtype=torch.long, device="cuda")
    going, next_token = here[:, 0], torch.full((B,), -1, dtype=torch.int32, device="cuda")
    path, count = torch.full((B, n), -1, dtype=torch.int32, device="cuda"), torch.zeros((B,), dtype=torch.int32, device="cuda")
    for j in range(n):
        path[:, j] = torch.where(going, at, -1)
        count += going
        chosen = s["choice"].gather(1, at[:, None])[:, 0]
        next_token = torch.where(going, chosen, next_token)
        child = here & (s["parent"] == at[:, None]) & (s["tokens"] == chosen[:, None]) & (each > at[:, None])
        going = going & child.any(1)
        at = torch.where(going, child.int().argmax(1), at)
    moves = path >= 0
    page_to, row_to = _places(s, torch.where(moves, base[:, None] + each, 0))
    page_from, row_from = _places(s, torch.where(moves, base[:, None] + path, 0))
    to, frm = (page_to[moves], row_to[moves]), (page_from[moves], row_from[moves])
    for name in ("k", "v", "k_scale", "v_scale"):
        if p[name] is not None:
            p[name][to[0], :, to[1]] = p[name][frm[0], :, frm[1]]
    s["path"].copy_(path); s["count"].copy_(count); s["next"].copy_(next_token)
    torch.add(base, count, out=s["len_out"])
    return dict(_pages_out(s), path=s["path"], count=s["count"], next=s["next"], len=s["len_out"])


# ------------------------------------------------------------------------------------------ in 64 bits
def _exact_e4m3(x):
    """The nearest E4M3 value, ties to the even one; |x| up to the largest."""
    exponent = torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 1
    step = torch.exp2((exponent - 3).double())
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_turn(x, at):
    """Pairs (i, i + D / 2) as complex numbers turned by their row's angles; x [rows, H, D], positions at [rows]."""
    half = x.shape[-1] // 2
    theta = torch.tensor([BASE ** (-2.0 * i / (2 * half)) for i in range(half)], dtype=torch.float64, device="cuda")
    angle = torch.tensor(at, dtype=torch.float64, device="cuda")[:, None] * theta
    z = torch.complex(x[..., :half].double(), x[..., half:].double()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([z.real, z.imag], -1)


def _above(parent, t):
    """The nodes from t up to its root."""
    nodes = [t]
    while parent[nodes[-1]] >= 0:
        nodes.append(parent[nodes[-1]])
    return nodes


def exact(case, seed):
    """Sequence by sequence, a node's ancestors by walking up its tree."""
    kind = case["kind"]
    if kind == "accept":
        return None                                                     # whole numbers and copies
    s = prepare(case, seed)
    if kind == "logprobs":
        rows, parts = case["rows"], []
        for r in range(0, rows, 256):
            x = s["logits"][r:r + 256].double()
            p = torch.log_softmax(x, 1)
            token = None if s["tokens"] is None else p.gather(1, s["tokens"][r:r + 256].long())
            top = p.topk(case["top"], 1).values if case["top"] else None
            parts.append((token, torch.special.entr(p.exp()).sum(1), top))
        join = lambda i: None if parts[0][i] is None else torch.cat([y[i] for y in parts])
        out = _some(logprob=join(0), entropy=join(1))
        if case["top"]:
            out.update(top=None, top_logprob=join(2))
        return out
    B, n, hkv, d, page = (case[k] for k in ("batch", "n", "hkv", "d", "page"))
    rows, table, lens = _rows_of(case), s["pages"]["table"].tolist(), s["len"].tolist()
    chain = list(range(-1, n - 1))
    trees = [chain] * B if s["parent"] is None else s["parent"].tolist()
    if kind == "append":
        new = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        out = {name: new(x) for name, x in _pages_out(s).items()}
        for b in range(B):
            depth = range(n) if s["parent"] is None else [len(_above(trees[b], t)) - 1 for t in range(n)]
            first = int(s["pos"][b]) + SHIFT
            at = torch.tensor([[table[b][(lens[b] + t) // page], (lens[b] + t) % page] for t in range(rows[b])], device="cuda")
            for name in ("k", "v"):
                x = s[name + "_new"][b, :rows[b]]
                x = _exact_turn(x, [first + depth[t] for t in range(rows[b])]) if name == "k" else x.double()
                if case["fmt"] == "row8":
                    scale = x.abs().amax(-1) / 448.0
                    out[name + "_scale"][at[:, 0], :, at[:, 1]] = scale
                    x = _exact_e4m3(x / scale[..., None])
                out[name][at[:, 0], :, at[:, 1]] = x
        return dict(out, len=None)
    hq = case["hq"]
    G, out = hq // hkv, torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, hq, n), dtype=torch.float64, device="cuda")

    def values(name, b):
        pages = table[b][:(lens[b] + page - 1) // page]
        x, scale = s["pages"][name][pages], s["pages"][name + "_scale"]
        if scale is not None:
            code = x.int()
            exponent, mantissa = (code >> 3) & 15, (code & 7).double()
            size = torch.where(exponent == 0, mantissa * 2.0 ** -9, (1.0 + mantissa / 8.0) * torch.exp2((exponent - 7).double()))
            x = torch.where(code >= 128, -size, size) * scale[pages].double()[..., None]
        return x.double().transpose(0, 1).reshape(hkv, -1, d)[:, :lens[b]]
    for b in range(B):
        k, v, r, before = values("k", b), values("v", b), rows[b], lens[b] - rows[b]
        q = s["q"][b, :r].double()
        nodes = [_above(trees[b], t) for t in range(r)]
        if s["pos"] is not None:
            q = _exact_turn(s["q"][b, :r], [int(s["pos"][b]) + len(x) - 1 for x in nodes])
        sees = torch.zeros((r, lens[b]), dtype=torch.bool)
        sees[:, :before] = True
        for t, x in enumerate(nodes):
            sees[t, [before + j for j in x]] = True
        hidden = ~sees.to("cuda")
        for g in range(hkv):                                            # (a head at a time: 64 bits of a long cache)
            x = torch.matmul(q[:, g * G:(g + 1) * G].reshape(r * G, d), k[g].t().contiguous()) / math.sqrt(d)
            x.view(r, G, -1).masked_fill_(hidden[:, None], -math.inf)
            lse[b, g * G:(g + 1) * G, :r] = torch.logsumexp(x, -1).view(r, G).t()
            out[b, :r, g * G:(g + 1) * G] = torch.matmul(torch.softmax(x, -1), v[g]).view(r, G, d)
    return _some(out=out, lse=None if s["lse"] is None else lse)
