"""64-bit statements of the operators of drafted trees over a paged cache, for their tests: written from the definitions in
include/parallelcomp.h, on the CPU, a sequence, a node and a head at a time."""
import numpy as np
import torch

from serving import E4M3, f64, quantize_rows, rotate


def rows_of(case, b):
    return case["n"] if case["n_rows"] is None else min(max(int(case["n_rows"][b]), 0), case["n"])


def above(case, b):
    """For every node: the nodes from it up to its root, itself first."""
    n = case["n"]
    up = list(range(-1, n - 1)) if case["parent"] is None else case["parent"][b].tolist()
    lines = []
    for t in range(n):
        line = [t]
        while 0 <= up[line[-1]] < line[-1]:
            line.append(up[line[-1]])
        lines.append(line)
    return lines


def place(case, b, row):
    """(page, row in it) of a sequence's row; None: it is not there."""
    page, table = case["page"], case["table"]
    if row < 0 or row // page >= table.shape[1]:
        return None
    p = int(table[b, row // page])
    return (p, row % page) if 0 <= p < case["n_pages"] else None


def random_tree(rng, n):
    """Parents: chains, bushes and several roots."""
    return [-1 if t == 0 or rng.random() < 0.08 else int(rng.integers(max(0, t - int(rng.integers(1, n + 1))), t)) for t in range(n)]


def build(B, n, Hq, Hkv, D, page, most, fmt, tree, ragged, rot, seed=0, gain=2.0, lens=None, spare=3):
    """Pools full of NaN but for the sequences' own rows; pages in no order; unequal lengths with the trees' rows at the end."""
    rng = np.random.default_rng([seed, B, n, Hq, D, page, most])
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000 * B + 10 * n + most)
    c = {"B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "base": 1.0e4, "pos0": -7, "spread": gain, "fmt": fmt}
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    c["n_rows"] = i32(rng.integers(0, n + 1, B).tolist()) if ragged else None
    rows = [rows_of(c, b) for b in range(B)]
    lens = [int(rng.integers(0, most + 1)) + r for r in rows] if lens is None else lens
    c["parent"] = i32([random_tree(rng, n) for _ in range(B)]) if tree else None
    need = [(x + page - 1) // page for x in lens]
    c["n_pages"] = sum(need) + spare
    order, width, at, table = rng.permutation(c["n_pages"]).tolist(), max(max(need), 1) + 1, 0, []
    for m in need:
        table.append(order[at:at + m] + [-1] * (width - m))
        at += m
    c["table"], c["len"] = i32(table), i32(lens)
    shape = (c["n_pages"], Hkv, page)
    for name in ("k", "v"):
        if fmt == "bf16":
            c[name], c[name + "_scale"] = torch.full((*shape, D), float("nan"), dtype=torch.bfloat16, device="cuda"), None
        else:
            c[name] = torch.full((*shape, D), 0x7f, dtype=torch.uint8, device="cuda")
            c[name + "_scale"] = torch.full(shape, float("nan"), device="cuda")
    for b in range(B):
        if lens[b] == 0:
            continue
        j = np.arange(lens[b])
        pages, at = torch.tensor([table[b][x] for x in j // page], device="cuda"), torch.tensor(j % page, device="cuda")
        for name in ("k", "v"):
            if fmt == "bf16":
                c[name][pages, :, at] = (gain * torch.randn((lens[b], Hkv, D), generator=gen, device="cuda")).to(torch.bfloat16)
            else:
                sign = torch.randint(0, 2, (lens[b], Hkv, D), generator=gen, device="cuda")
                c[name][pages, :, at] = (torch.randint(0, 127, (lens[b], Hkv, D), generator=gen, device="cuda") + 128 * sign).to(torch.uint8)
                c[name + "_scale"][pages, :, at] = gain * (0.5 + torch.rand((lens[b], Hkv), generator=gen, device="cuda")) / 120.0
    c["q"] = (gain * torch.randn((B, n, Hq, D), generator=gen, device="cuda")).to(torch.bfloat16)
    c["pos"] = i32((np.asarray(lens) - rows + rng.integers(7, 9000)).tolist()) if rot else None
    return c


def attention(case):
    """out, lse and what they may be off; a row that is not a sequence's is NaN in both.  Every term is a rounding of the kernels:
      2^-8 |out|             the output's rounding to bf16 (half a step), with room for the fp32 sums
      2^-8 sum p |v|         the probabilities' rounding
      2 eps sum p |v|, eps   the logits' errors: a rotated q is two bf16 parts and its angle's sine and cosine good to 1e-7, so a
                             logit moves by at most 2^-16 scale sum |q_i k_i|, which moves a probability by twice that,
                             relatively, and the logsumexp by that; fp32 products, sums and exponentials: 1e-5"""
    B, n, Hq, Hkv, D = (case[k] for k in ("B", "n", "Hq", "Hkv", "D"))
    G, scale = Hq // Hkv, case.get("scale") or D ** -0.5
    out, bound = np.full((B, n, Hq, D), np.nan), np.zeros((B, n, Hq, D))
    lse, lse_bound = np.full((B, Hq, n), np.nan), np.zeros((B, Hq, n))
    pools = {x: (case[x].cpu(), None if case[x + "_scale"] is None else case[x + "_scale"].cpu().numpy().astype(np.float64)) for x in "kv"}

    def row(x, at, g):
        pool, s = pools[x]
        return f64(pool[at[0], g, at[1]]) if s is None else E4M3[pool[at[0], g, at[1]].numpy()] * s[at[0], g, at[1]]
    q_all = f64(case["q"])
    for b in range(B):
        r, lines = rows_of(case, b), above(case, b)
        base = max(int(case["len"][b]), 0) - r
        q = q_all[b]
        if case["pos"] is not None:
            q = rotate(q, [int(case["pos"][b]) + case["pos0"] + len(x) - 1 for x in lines], case["base"])
        places = [place(case, b, j) for j in range(base + r)]
        for g in range(Hkv):
            ks, vs = ({j: row(x, at, g) for j, at in enumerate(places) if at is not None} for x in "kv")
            for t in range(r):
                own = {base + u for u in lines[t]}
                seen = [j for j in ks if j < base or j in own]
                hs = slice(g * G, (g + 1) * G)
                out[b, t, hs], lse[b, hs, t] = 0.0, -np.inf
                if not seen:
                    continue
                k, v = np.stack([ks[j] for j in seen]), np.stack([vs[j] for j in seen])
                x = scale * (q[t, hs] @ k.T)                                # [G, keys]
                with np.errstate(invalid="ignore"):
                    m = x.max(1, keepdims=True)
                    e = np.exp(x - m)
                    p = e / e.sum(1, keepdims=True)
                    out[b, t, hs] = p @ v
                    lse[b, hs, t] = m[:, 0] + np.log(e.sum(1))
                    eps = 1e-5 + (2.0 ** -16 * scale * (np.abs(q[t, hs]) @ np.abs(k).T).max(1) if case["pos"] is not None else np.zeros(G))
                    bound[b, t, hs] = 2.0 ** -8 * np.abs(out[b, t, hs]) + (2.0 ** -8 + 2 * eps[:, None]) * (p @ np.abs(v)) + 1e-30
                    lse_bound[b, hs, t] = eps + 1e-6 * np.abs(lse[b, hs, t])
    return out, bound, lse, lse_bound


def check_attention(out, lse, case, what, untouched):
    """untouched: what lies in rows of out and lse that are no sequence's."""
    ref, bound, ref_lse, lse_bound = attention(case)
    o, l = f64(out), None if lse is None else lse.cpu().numpy().astype(np.float64)
    for b in range(case["B"]):
        r = rows_of(case, b)
        assert (o[b, r:] == untouched).all(), f"{what}: rows behind a tree are written"
        assert l is None or (l[b, :, r:] == untouched).all(), f"{what}: logsumexp behind a tree is written"
        fine = np.isfinite(ref[b, :r])
        assert np.array_equal(fine, np.isfinite(o[b, :r])), f"{what}: sequence {b}, not finite in other places"
        same = o[b, :r][~fine], ref[b, :r][~fine]
        assert np.array_equal(*same, equal_nan=True), f"{what}: sequence {b}, infinities and NaN differ"
        err = np.abs(o[b, :r][fine] - ref[b, :r][fine])
        assert np.all(err <= bound[b, :r][fine]), f"{what}: sequence {b}, out off by {err.max():.3e}"
        if l is not None:
            x, y = l[b, :, :r], ref_lse[b, :, :r]
            assert np.array_equal(np.isneginf(x), np.isneginf(y)), f"{what}: lse of empty rows"
            some = np.isfinite(y)
            off = np.abs(x[some] - y[some])
            assert np.all(off <= lse_bound[b, :, :r][some]), f"{what}: lse off by {off.max():.3e}"


def append(case, k_new, v_new, before):
    """The pools after an append behind `before` rows: ({name: values}, {name: bound}, lengths).  bf16: the rotated key's
    rounding, half a step (2^-8), and its sum's of two products in 32 bits, 2^-22 of |x1| + |x2|.  8 bits: codes and scales by
    quantize_rows, where nothing is rotated exactly; else a step of the code (2^-3 of it, at least 2^-9 scales), for a value that
    may lie at a border between two."""
    want = {x: case[x].cpu().clone() for x in ("k", "v", "k_scale", "v_scale") if case[x] is not None}
    want = {x: (f64(t) if t.dtype == torch.bfloat16 else t.numpy()) for x, t in want.items()}
    bound = {x: np.zeros(t.shape) for x, t in want.items()}
    lens = []
    for b in range(case["B"]):
        r, lines = rows_of(case, b), above(case, b)
        lens.append(max(before[b], 0) + r)
        for x, new in (("k", k_new), ("v", v_new)):
            y = f64(new[b])
            size = np.abs(y)
            if x == "k" and case["pos"] is not None:
                half = y.shape[-1] // 2
                size = np.concatenate([size[..., :half] + size[..., half:]] * 2, -1)
                y = rotate(y, [int(case["pos"][b]) + case["pos0"] + len(line) - 1 for line in lines], case["base"])
            for t in range(r):
                at = place(case, b, max(before[b], 0) + t)
                if at is None:
                    continue
                if case["fmt"] == "bf16":
                    want[x][at[0], :, at[1]] = y[t]
                    bound[x][at[0], :, at[1]] = 0.0 if x == "v" or case["pos"] is None else 2.0 ** -8 * np.abs(y[t]) + 2.0 ** -22 * size[t]
                    continue
                code, scale = quantize_rows(y[t])
                want[x][at[0], :, at[1]], want[x + "_scale"][at[0], :, at[1]] = code, scale
                if x == "k" and case["pos"] is not None:
                    bound[x][at[0], :, at[1]] = 1.0
                    bound[x + "_scale"][at[0], :, at[1]] = scale * 2.0 ** -21
    return want, bound, lens


def accept(case, tokens, choice):
    """path, n_kept, next token of every sequence, and the moves of rows (from, to)."""
    B, n = case["B"], case["n"]
    path, kept, following, moves = np.full((B, n), -1, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32), []
    for b in range(B):
        r = rows_of(case, b)
        up = list(range(-1, n - 1)) if case["parent"] is None else case["parent"][b].tolist()
        line = [0] if r else []
        while line:
            following[b] = choice[b][line[-1]]
            below = [c for c in range(line[-1] + 1, r) if up[c] == line[-1] and tokens[b][c] == choice[b][line[-1]]]
            if not below:
                break
            line.append(below[0])
        path[b, :len(line)], kept[b] = line, len(line)
        base = int(case["len"][b]) - r
        moves.append([(place(case, b, base + t), place(case, b, base + j)) for j, t in enumerate(line)])
    return path, kept, following, moves
