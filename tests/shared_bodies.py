"""Calls of pc_shared_attn that reach every body of its kernels, and a statement of the result in 64 bits whose bounds are
close enough to notice a lost part of a query row or a wrong rescaling at large logits."""
import ctypes
import itertools

import numpy as np
import torch

import paper_2502_14317_amd as pc
from serving import row_values, rotate

# B, P, n_q, H_q, H_kv, D, segments (0: no prefix), k_t, tail cap (0: no tail), prefix format, tail format.  The kinds of
# work in each are asserted below: `kinds` asks the library.
CASES = [
    # one launch: nothing shared or little
    (1, 1, 1, 4, 1, 64, 0, 1, 84, "bf16", "bf16"),
    (1, 1, 3, 1, 1, 64, 0, 1, 69, "bf16", "row8"),
    (1, 1, 1, 2, 2, 128, 0, 1, 131, "bf16", "bf16"),
    (2, 1, 1, 2, 2, 128, 0, 1, 65, "row8", "row8"),
    (1, 1, 1, 4, 4, 64, 3, 79, 0, "bf16", "bf16"),
    (2, 1, 2, 1, 1, 64, 1, 162, 0, "row8", "bf16"),
    (1, 1, 3, 1, 1, 128, 2, 138, 0, "bf16", "bf16"),
    (1, 1, 1, 2, 2, 128, 9, 22, 0, "row8", "bf16"),
    (3, 3, 1, 2, 1, 64, 2, 81, 65, "bf16", "bf16"),
    (4, 2, 1, 1, 1, 64, 1, 231, 53, "bf16", "row8"),
    (1, 1, 1, 1, 1, 64, 3, 148, 23, "row8", "bf16"),
    (1, 1, 1, 2, 2, 64, 1, 159, 76, "row8", "row8"),
    (2, 1, 1, 1, 1, 128, 2, 106, 104, "bf16", "bf16"),
    (2, 1, 3, 2, 2, 128, 1, 220, 26, "bf16", "row8"),
    (1, 1, 1, 2, 2, 128, 8, 25, 206, "row8", "bf16"),
    (1, 1, 2, 2, 2, 128, 2, 162, 27, "row8", "row8"),
    # up to 16 rows, the tails behind them with eight, four, two and one wavefronts each
    (1, 1, 1, 2, 2, 64, 2, 311, 507, "bf16", "bf16"),
    (2, 2, 1, 1, 1, 128, 3, 195, 501, "bf16", "bf16"),
    (2, 1, 1, 1, 1, 64, 1, 874, 143, "row8", "row8"),
    (2, 2, 1, 1, 1, 128, 2, 628, 1391, "row8", "row8"),
    (15, 3, 1, 8, 8, 64, 5, 189, 38, "row8", "row8"),
    (3, 3, 1, 16, 8, 128, 2, 867, 38, "bf16", "bf16"),
    (9, 3, 2, 2, 2, 128, 4, 1478, 41, "bf16", "row8"),
    (4, 1, 1, 8, 8, 128, 3, 2052, 27, "bf16", "bf16"),
    # 32, 64 and 256 rows with such tails
    (63, 3, 1, 8, 8, 64, 5, 92, 44, "bf16", "row8"),
    (72, 2, 1, 8, 8, 64, 2, 380, 27, "bf16", "row8"),
    (132, 2, 1, 8, 8, 128, 1, 266, 20, "row8", "row8"),
    (230, 1, 1, 2, 2, 64, 3, 86, 251, "bf16", "bf16"),
    (194, 2, 1, 4, 4, 128, 1, 726, 108, "row8", "row8"),
    (194, 2, 1, 4, 4, 64, 2, 1023, 410, "row8", "bf16"),
    (231, 1, 1, 8, 8, 128, 2, 203, 42, "row8", "bf16"),
    (199, 1, 1, 24, 8, 64, 1, 403, 167, "bf16", "bf16"),
    # tails of more than 16 rows
    (1, 1, 3, 8, 1, 128, 3, 291, 1766, "row8", "bf16"),
    (1, 1, 8, 6, 2, 64, 7, 366, 541, "row8", "bf16"),
    (1, 1, 5, 4, 1, 128, 3, 68, 119, "bf16", "row8"),
    (28, 2, 5, 16, 2, 64, 3, 105, 403, "bf16", "bf16"),
    (9, 3, 5, 28, 4, 128, 2, 375, 321, "bf16", "bf16"),
    (34, 1, 17, 14, 2, 128, 1, 195, 169, "bf16", "row8"),
    (6, 1, 354, 6, 2, 64, 2, 102, 55, "row8", "row8"),
    (31, 1, 37, 8, 4, 64, 3, 100, 77, "row8", "row8"),
    (69, 1, 17, 8, 2, 64, 2, 97, 25, "row8", "row8"),
    (51, 1, 17, 8, 2, 128, 3, 55, 26, "row8", "row8"),
    # tails alone
    (2, 1, 1, 2, 2, 64, 0, 1, 1300, "bf16", "bf16"),
    (3, 1, 1, 2, 2, 64, 0, 1, 1700, "row8", "row8"),
    (3, 3, 1, 2, 2, 128, 0, 1, 2300, "row8", "row8"),
    (2, 1, 1, 2, 1, 64, 0, 1, 727, "row8", "bf16"),
    (1, 1, 1, 4, 1, 64, 0, 1, 833, "row8", "row8"),
    (1, 1, 2, 2, 2, 128, 0, 1, 903, "bf16", "bf16"),
    (1, 1, 1, 2, 2, 128, 0, 1, 1178, "row8", "row8"),
    (1, 1, 5, 8, 1, 64, 0, 1, 100, "row8", "row8"),
    (36, 2, 17, 14, 2, 64, 0, 1, 67, "bf16", "row8"),
    (105, 3, 17, 8, 1, 64, 0, 1, 322, "bf16", "bf16"),
    (51, 3, 17, 16, 2, 128, 0, 1, 344, "bf16", "bf16"),
    (48, 1, 17, 16, 4, 128, 0, 1, 67, "row8", "row8"),
]
# what the cases have to reach: (kind, rows or wavefronts, format, values a row)
EVERY = set(itertools.product(["prefix", "prefix in parts", "tail"], [16, 32, 64, 256], [1, 2], [64, 128])) | \
    set(itertools.product(["behind"], [1, 2, 4, 8], [1, 2], [64, 128])) | \
    set(itertools.product(["tail in parts"], [16, 32, 64, 256], [0], [64, 128])) | \
    set(itertools.product(["merge"], [1, 256], [0], [64, 128])) | \
    {("alone", p, t, d) for p, t, d in itertools.product([0, 1, 2], [0, 1, 2], [64, 128]) if p or t}


def plan(case):
    """How the library does a case; pointers are never followed."""
    B, P, nq, Hq, Hkv, D, S, kt, cap, pf, tf = case
    at = ctypes.c_void_p(256)

    def rows(fmt, n_seg, cap):
        if n_seg == 0:
            return None
        return pc.pc_row_cache(at, at, *([at, at] if fmt == "row8" else [None, None]), at, 0, n_seg, cap)
    return pc.pc_shared_attn_plan(rows(pf, S, kt), rows(tf, int(cap > 0), cap), B, P, nq, Hq, Hkv, D)


def kinds(case):
    p, D, has_tail = plan(case), case[5], case[8] > 0
    if p["alone"]:
        return {("alone", p["prefix_format"], p["tail_format"] * has_tail, D)}
    k = set()
    if p["prefix_rows"]:
        k.add(("prefix", p["prefix_rows"], p["prefix_format"], D))
        if p["prefix_parts"] > 1:
            k.add(("prefix in parts", p["prefix_rows"], p["prefix_format"], D))
    if p["tail_rows"]:
        k.add(("behind", p["tail_waves"], p["tail_format"], D) if p["tails_behind"] else ("tail", p["tail_rows"], p["tail_format"], D))
        if p["tail_parts"] > 1:
            k.add(("tail in parts", p["tail_rows"], 0, D))
    wide = p["prefix_parts"] + p["tail_parts"] > 1024 // D and case[0] * case[2] * case[3] <= 1024
    k.add(("merge", 256 if wide else 1, 0, D))
    return k


def build(case, rotated, gain=2.0, value=1.0, seed=0, device="cuda"):
    """Random rows, a third of the lengths short, `gain` the logits' deviation, `value` the values' size."""
    B, P, nq, Hq, Hkv, D, S, kt, cap, pf, tf = case
    gen = torch.Generator().manual_seed(seed + 7919 * B + 31 * nq + kt + cap)
    normal = lambda *shape: torch.randn(shape, generator=gen)

    def rows(fmt, *shape):
        if fmt == "bf16":
            return [normal(*shape).to(torch.bfloat16), (value * normal(*shape)).to(torch.bfloat16), None, None]
        codes = lambda: torch.randint(0, 127, shape, generator=gen).to(torch.uint8) | (128 * torch.randint(0, 2, shape, generator=gen)).to(torch.uint8)
        scales = lambda size: size * (0.5 + torch.rand(shape[:-1], generator=gen)) / 120.0      # finite codes: deviation 120
        return [codes(), codes(), scales(1.0), scales(value)]
    c = {"case": case, "B": B, "P": P, "nq": nq, "Hq": Hq, "Hkv": Hkv, "D": D, "base": 1.0e4, "pos0": 11, "gain": gain, "pos": None,
         "prefix": None, "tail": None, "seg_len": None, "tail_len": None}
    c["q"] = (gain * normal(B, nq, Hq, D)).to(torch.bfloat16)
    length = lambda n, *shape: torch.where(torch.rand(shape, generator=gen) < 0.67, torch.full(shape, n),
                                           torch.randint(0, n + 1, shape, generator=gen)).to(torch.int32)
    if S:
        c["prefix"], c["seg_len"] = rows(pf, P, S, Hkv, kt, D), length(kt, P, S, Hkv)
    if cap:
        c["tail"], c["tail_len"] = rows(tf, B, 1, Hkv, cap, D), length(cap, B)
    if rotated:
        c["pos"] = torch.randint(0, 9000, (B,), generator=gen).to(torch.int32)
    to = lambda x: x.to(device) if torch.is_tensor(x) else ([to(y) for y in x] if isinstance(x, list) else x)
    return {name: to(x) for name, x in c.items()}


def each_softmax(c):
    """Per sequence and KV head: keys, values, rotated query rows [n_q G, D] in 64 bits, visible keys [n_q G, keys], and the
    head of its first row."""
    B, P, nq, Hq, Hkv, D = (c[k] for k in ("B", "P", "nq", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    values = {n: c[n] and [row_values(x, s) for x, s in zip(c[n][:2], c[n][2:])] for n in ("prefix", "tail")}
    lens = {n: None if c[n] is None else c[n].cpu().numpy() for n in ("seg_len", "tail_len", "pos")}
    q_all = c["q"].float().cpu().numpy().astype(np.float64)
    for b in range(B):
        q = q_all[b] if lens["pos"] is None else rotate(q_all[b], int(lens["pos"][b]) + c["pos0"] + np.arange(nq), c["base"])
        for g in range(Hkv):
            k, v, seen = [], [], []
            if c["prefix"]:
                p = b // (B // P)
                for s in range(c["prefix"][0].shape[1]):
                    n = int(np.clip(lens["seg_len"][p, s, g], 0, c["prefix"][0].shape[3]))
                    k.append(values["prefix"][0][p, s, g, :n]); v.append(values["prefix"][1][p, s, g, :n])
                    seen.append(np.ones((nq, n), bool))
            if c["tail"]:
                n = int(np.clip(lens["tail_len"][b], 0, c["tail"][0].shape[3]))
                k.append(values["tail"][0][b, 0, g, :n]); v.append(values["tail"][1][b, 0, g, :n])
                seen.append(np.arange(n)[None] < n - (nq - 1 - np.arange(nq))[:, None])
            yield (b, g, np.concatenate(k), np.concatenate(v), q[:, g * G:(g + 1) * G].reshape(nq * G, D),
                   np.repeat(np.concatenate(seen, 1), G, 0))


def softmax_rows(k, v, q, seen, scale):
    """out [rows, D], logsumexp [rows], probabilities, logits; rows that see nothing: 0 and -inf."""
    x = np.where(seen, scale * (q @ k.T), -np.inf)
    m = x.max(1, initial=-np.inf)
    e = np.exp(x - np.where(np.isinf(m), 0.0, m)[:, None])
    total = e.sum(1)
    p = e / np.where(total > 0, total, 1.0)[:, None]
    with np.errstate(divide="ignore"):
        return p @ v, np.where(total > 0, m + np.log(total), -np.inf), p, x


def check(out, lse, c, what):
    """Against 64 bits.  Off by no more than (u = 2^-8, the largest relative error of a rounding to bf16)
      u |out|                    the output's rounding
      (u + 2 eps) sum p |v|      the probabilities' rounding, and an error of eps in the logits, which moves a probability by
                                 twice that, relatively, and the logsumexp by that:
      eps = 1e-5 + 3e-7 max |x|  the exponentials, fp32 sums; the scaled logit's rounding
          + 2^-17 sum |q k|      128 fp32 products and sums a logit
          + 2^-17 sum |q k|      a rotated row kept as two bf16 parts (|q|: of a pair, which the rotation leaves)
    In the 2-norm over 64 rows or more these average: a rounding's error is 1.66e-3 of a value, the output's and the
    probabilities' add up to 2.35e-3, bound 2^-8; the queries' parts add 2^-17 at most times the logits' deviation (bound
    2^-16 of it).  (Of few rows whose weight sits on one key each it is few probabilities' rounding, up to u: bound 2 u.)"""
    D, scale, G = c["D"], c["D"] ** -0.5, c["Hq"] // c["Hkv"]
    turned = 2.0 ** -17 if c["pos"] is not None else 0.0
    out, lse = np.asarray(out, np.float64), np.asarray(lse, np.float64)
    off2 = norm2 = 0.0
    for b, g, k, v, q, seen in each_softmax(c):
        heads = slice(g * G, (g + 1) * G)
        got, got_lse = out[b][:, heads].reshape(-1, D), lse[b][heads].T.reshape(-1)
        if not k.shape[0]:
            assert not got.any() and np.isneginf(got_lse).all(), f"{what}: sequence {b} sees nothing"
            continue
        want, want_lse, p, x = softmax_rows(k, v, q, seen, scale)
        r = np.tile(np.hypot(q[:, :D // 2], q[:, D // 2:]), 2) if c["pos"] is not None else np.abs(q)
        most = np.where(seen, r @ np.abs(k).T, 0.0).max(1) * scale
        eps = 1e-5 + 3e-7 * np.where(seen, np.abs(x), 0.0).max(1) + (2.0 ** -17 + turned) * most
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * eps[:, None]) * (p @ np.abs(v)) + 1e-30
        assert np.isfinite(got).all(), f"{what}: sequence {b}, head {g}: not finite"
        err = np.abs(got - want)
        assert np.all(err <= bound), f"{what}: sequence {b}, head {g}: {np.sum(err > bound)} values outside, off by {(err / bound).max():.3g} of the bound"
        empty = ~seen.any(1)
        assert not got[empty].any() and np.isneginf(got_lse[empty]).all(), f"{what}: sequence {b}: rows that see nothing"
        off = np.abs(got_lse[~empty] - want_lse[~empty])
        allowed = (eps + 1e-6 * np.abs(want_lse))[~empty]
        assert np.all(off <= allowed), f"{what}: sequence {b}, head {g}: logsumexp off by {(off / allowed).max():.3g} of the bound"
        off2 += (err ** 2).sum(); norm2 += (want ** 2).sum()
    if norm2 > 0:
        rel = (off2 / norm2) ** 0.5
        limit = (2.0 ** -8 if c["B"] * c["nq"] * c["Hq"] >= 64 else 2.0 ** -7) + c["gain"] * (2.0 ** -16 if turned else 2.0 ** -17)
        assert rel <= limit, f"{what}: {rel:.3e} of the norm, allowed {limit:.3e}"
