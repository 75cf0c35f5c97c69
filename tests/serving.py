"""64-bit statements of the serving operators for their tests: shared-prefix attention, 8-bit rows, draft verification.
Written from the definitions in include/parallelcomp.h, on the CPU, a sequence and a head at a time."""
import numpy as np
import torch

E4M3 = np.array([(-1) ** (c >> 7) * ((c & 7) / 8.0 + (c >> 3 & 15 != 0)) * 2.0 ** max((c >> 3 & 15) - 7, -6) for c in range(256)])
E4M3[[0x7f, 0xff]] = np.nan


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def row_values(x, scale=None):
    """[.., cap, D] rows in 64 bits: bf16 tensors, or codes with a scale a row."""
    return f64(x) if scale is None else E4M3[x.cpu().numpy()] * scale.cpu().numpy().astype(np.float64)[..., None]


def rotate(x, pos, base):
    """x [n, H, D] at positions pos [n]: dimension i turns with i + D / 2."""
    half = x.shape[-1] // 2
    ang = np.asarray(pos, dtype=np.float64)[:, None, None] * float(base) ** (-np.arange(half) / half)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def visible(case, b, g, t):
    """Number of visible keys of every segment of the prefix, and of the tail."""
    p = b // (case["B"] // case["P"])
    segs = []
    if case["prefix"] is not None:
        n_seg, cap = case["prefix"][0].shape[1], case["prefix"][0].shape[3]
        for s in range(n_seg):
            n = cap if case["seg_len"] is None else int(case["seg_len"][p, s, g] if case["per_head"] else case["seg_len"][p, s])
            segs.append(min(max(n, 0), cap))
    tail = 0
    if case["tail"] is not None:
        cap = case["tail"][0].shape[3]
        tail = cap if case["tail_len"] is None else min(max(int(case["tail_len"][b]), 0), cap)
        if case["own"]:
            tail = max(0, tail - (case["nq"] - 1 - t))
    return segs, tail


def attention(case):
    """out, lse and what a result may be off: every term of the bound is a rounding of the kernels.
      2^-8 |out|             the output's rounding to bf16 (2^-9), with room for the fp32 sums
      2^-8 sum p |v|         the probabilities' rounding (2^-9)
      2 eps sum p |v|, eps   the logits' errors: a rotated q rounded to bf16 moves a logit by at most
                             2^-9 scale sum |q_i k_i|, which moves a probability by twice that, relatively, and the
                             logsumexp by that; fp32 products, sums and exponentials: 1e-5"""
    B, P, nq, Hq, Hkv, D = (case[k] for k in ("B", "P", "nq", "Hq", "Hkv", "D"))
    G, scale = Hq // Hkv, case.get("scale") or D ** -0.5
    out, bound = np.zeros((B, nq, Hq, D)), np.zeros((B, nq, Hq, D))
    lse, lse_bound = np.full((B, Hq, nq), -np.inf), np.zeros((B, Hq, nq))
    val = {n: None if case[n] is None else [row_values(x, s) for x, s in zip(case[n][:2], case[n][2:])] for n in ("prefix", "tail")}
    q_all = f64(case["q"])
    for b in range(B):
        q = q_all[b]
        if case["pos"] is not None:
            q = rotate(q, int(case["pos"][b]) + case.get("pos0", 0) + np.arange(nq), case["base"])
        for g in range(Hkv):
            for t in range(nq):
                segs, n_tail = visible(case, b, g, t)
                ks, vs = [], []
                for s, n in enumerate(segs):
                    ks.append(val["prefix"][0][b // (B // P), s, g, :n]); vs.append(val["prefix"][1][b // (B // P), s, g, :n])
                if case["tail"] is not None:
                    ks.append(val["tail"][0][b, 0, g, :n_tail]); vs.append(val["tail"][1][b, 0, g, :n_tail])
                k, v = np.concatenate(ks), np.concatenate(vs)
                if not len(k):
                    continue
                for h in range(g * G, (g + 1) * G):
                    x = scale * (k @ q[t, h])
                    m = x.max()
                    e = np.exp(x - m)
                    p = e / e.sum()
                    with np.errstate(invalid="ignore"):
                        out[b, t, h] = p @ v
                    lse[b, h, t] = m + np.log(e.sum())
                    eps = 1e-5
                    if case["pos"] is not None:
                        eps += 2.0 ** -9 * scale * (np.abs(k) @ np.abs(q[t, h])).max()
                    with np.errstate(invalid="ignore"):
                        spread = p @ np.abs(v)
                    bound[b, t, h] = 2.0 ** -8 * np.abs(out[b, t, h]) + (2.0 ** -8 + 2 * eps) * spread + 1e-30
                    lse_bound[b, h, t] = eps + 1e-6 * abs(lse[b, h, t])
    return out, bound, lse, lse_bound


def check_attention(out, lse, case, what):
    ref, bound, ref_lse, lse_bound = attention(case)
    o, l = f64(out), None if lse is None else lse.cpu().numpy().astype(np.float64)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(ref), np.isnan(o)), f"{what}: NaN in other places"
    assert np.array_equal(ref[~fine & ~np.isnan(ref)], o[~fine & ~np.isnan(ref)]), f"{what}: infinities differ"
    err = np.abs(o[fine] - ref[fine])
    assert np.all(err <= bound[fine]), f"{what}: out off by {err.max():.3e}, {np.sum(err > bound[fine])} values outside"
    # in the 2-norm the roundings above average: each at most 2^-9 a value, q's twice over and times a logit's deviation
    if fine.all() and np.linalg.norm(ref) > 0:
        rel = np.linalg.norm(o - ref) / np.linalg.norm(ref)
        assert rel <= (3.0 * case.get("spread", 1.0) if case["pos"] is not None else 2.0) * 2.0 ** -9, f"{what}: {rel:.3e} of the norm"
    if l is not None:
        empty = np.isneginf(ref_lse)
        assert np.array_equal(empty, np.isneginf(l)), f"{what}: lse of empty rows"
        off = np.abs(l[~empty] - ref_lse[~empty])
        assert np.all(off <= lse_bound[~empty]), f"{what}: lse off by {off.max():.3e}"


def make_rows(gen, fmt, shape, gain=1.0):
    """Random rows as the tuple (k, v, k_scale, v_scale) on the GPU; 8-bit ones directly as codes and scales."""
    if fmt == "bf16":
        mk = lambda: (gain * torch.randn(shape, generator=gen, device="cuda")).to(torch.bfloat16)
        return mk(), mk(), None, None
    codes = lambda: torch.randint(0, 127, shape, generator=gen, device="cuda").to(torch.uint8) | \
        (128 * torch.randint(0, 2, shape, generator=gen, device="cuda")).to(torch.uint8)
    # codes spread over all finite ones have a deviation of about 120: scales bring rows to about `gain`
    scales = lambda: gain * (0.5 + torch.rand(shape[:-1], generator=gen, device="cuda")) / 120.0
    return codes(), codes(), scales(), scales()


def quantize_rows(x):
    """x [.., D] fp32 numpy -> (codes, scales) by the definition in 32-bit steps: a table's nearest value, ties to the
    even code."""
    x = np.asarray(x, dtype=np.float32)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    scale = np.where((top > 0) & ~bad, np.maximum(np.where(bad, 1, top) / np.float32(448), np.float32(2.0 ** -126)), np.float32(1)).astype(np.float32)
    y = np.clip(np.where(bad[..., None], 0, x) / scale[..., None], np.float32(-448), np.float32(448)).astype(np.float64)
    table = E4M3[:127]
    mid = (table[:-1] + table[1:]) / 2
    lo = np.searchsorted(mid, np.abs(y), side="left")               # a tie stays with the lower code
    tie = (lo < 126) & (np.abs(y) == mid[np.minimum(lo, 125)]) & (lo % 2 == 1)
    code = (lo + tie).astype(np.uint8) | np.where(np.signbit(y), 128, 0).astype(np.uint8)
    return np.where(bad[..., None], np.uint8(0x7f), code), scale


def verify(draft, draft_prob, target_prob, u, noise, draft_len=None):
    """One sequence after the other, one 32-bit operation at a time."""
    B, k, V = draft.shape[0], draft.shape[1], target_prob.shape[2]
    tokens, count = np.full((B, k + 1), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        n = k if draft_len is None else min(max(int(draft_len[b]), 0), k)
        a = 0
        while a < n:
            d = int(draft[b, a])
            if not 0 <= d < V:
                break
            qd = np.float32(1) if draft_prob is None else draft_prob[b, a, d]
            if not np.float32(u[b, a] * qd) < target_prob[b, a, d]:
                break
            a += 1
        p = target_prob[b, a]
        q = np.zeros(V, np.float32)
        if a < n:
            if draft_prob is not None:
                q = draft_prob[b, a]
            elif 0 <= draft[b, a] < V:
                q[draft[b, a]] = 1
        token = -1
        for r in ((p - q).astype(np.float32), p):
            with np.errstate(divide="ignore", invalid="ignore"):
                ratio = (r / noise[b]).astype(np.float32)
            ok = (r > 0) & (ratio >= 0)
            if ok.any():
                token = int(np.argmax(np.where(ok, ratio, np.float32(-1))))
                break
        tokens[b, :a], tokens[b, a], count[b] = draft[b, :a], token, a
    return tokens, count
