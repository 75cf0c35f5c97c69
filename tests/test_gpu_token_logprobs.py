"""pc_token_logprobs against 64 bits: types, vocabularies of one token to more than a workgroup's, odd sizes and row strides, ties,
masked entries, rows without a distribution."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc

pytestmark = pytest.mark.gpu


def call(logits, tokens, n_top, entropy=True, top_logprob=True):
    rows, vocab = logits.shape
    n_tokens = 0 if tokens is None else tokens.shape[1]
    new = lambda n, t: torch.full((rows, n), -7, dtype=t, device="cuda")
    token_lp = new(n_tokens, torch.float32) if n_tokens else None
    ent = new(1, torch.float32)[:, 0] if entropy else None
    top, top_lp = new(n_top, torch.int32), new(n_top, torch.float32) if top_logprob else None
    ws = pc.alloc_workspace(pc.pc_token_logprobs_workspace_bytes(rows, vocab, n_top))
    ws.fill_(255)
    run = lambda: pc.pc_token_logprobs(logits, rows, vocab, tokens, n_tokens, n_top, token_lp, ent, top if n_top else None,
                                       top_lp if n_top else None, ws)
    run()
    return token_lp, ent, top, top_lp, run


def reference(logits, tokens, n_top):
    x = logits.float().cpu().numpy().astype(np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(1, keepdims=True)
        lse = m + np.log(np.exp(x - m).sum(1, keepdims=True))
        lp = x - lse
        terms = np.exp(lp) * lp
        ent = -np.where(np.isneginf(lp), 0.0, terms).sum(1)
    lp[np.isneginf(m)[:, 0]] = np.nan
    ent[np.isneginf(m)[:, 0]] = np.nan
    order = np.argsort(np.where(np.isnan(x), np.inf, -x), axis=1, kind="stable")          # NaN behind -inf, the lower token first
    nan_last = np.take_along_axis(np.isnan(x), order, 1)
    order = np.take_along_axis(order, np.argsort(nan_last, axis=1, kind="stable"), 1)[:, :n_top]
    tok = None
    if tokens is not None:
        t = tokens.cpu().numpy()
        tok = np.where((t >= 0) & (t < x.shape[1]), np.take_along_axis(lp, np.clip(t, 0, x.shape[1] - 1), 1), np.nan)
    return tok, ent, order, np.take_along_axis(lp, order, 1)


def check(logits, tokens, n_top, what):
    """A log probability is (x - m) - log l: x log2 e in one rounding relative to the product's size, log2 l good to the
    sum's 2^-20 (a thread's 128 terms at most one after the other, then a tree; an exponential's 2^-22 each), so
    |x - m| 2^-22 + 2^-18 covers it, with m's own rounding, |m| 2^-23.  The entropy sums terms of p log p of one sign: the same
    relative errors, of a number up to log V, and those of the terms' logarithms."""
    token_lp, ent, top, top_lp, _ = call(logits, tokens, n_top)
    want_tok, want_ent, want_top, want_top_lp = reference(logits, tokens, n_top)
    x = logits.float().cpu().numpy().astype(np.float64)
    with np.errstate(invalid="ignore"):
        m = np.abs(np.where(np.isfinite(x), x, 0.0)).max(1)[:, None]

    def near(got, want, name):
        got = got.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: {name}, NaN in other places"
        some = ~np.isnan(want)
        inf = np.isinf(want)
        assert np.array_equal(got[inf], want[inf]), f"{what}: {name}, infinities"
        some &= ~inf
        bound = np.broadcast_to(2.0 ** -18 + (np.abs(np.where(some, want, 0.0)) + 2 * m) * 2.0 ** -22, want.shape)
        off = np.abs(got - want)
        assert np.all(off[some] <= bound[some]), f"{what}: {name} off by {off[some].max():.3e}"
    if tokens is not None:
        near(token_lp, want_tok, "token_logprob")
    near(ent[:, None], want_ent[:, None], "entropy")
    if n_top:
        assert np.array_equal(top.cpu().numpy(), want_top), f"{what}: top_idx"
        near(top_lp, want_top_lp, "top_logprob")


def make(rows, vocab, dtype, seed, pad=0, gain=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed + rows + vocab)
    whole = (gain * torch.randn((rows, vocab + pad), generator=gen, device="cuda")).to(dtype)
    tokens = torch.randint(-1, vocab + 1, (rows, 3), generator=gen, device="cuda", dtype=torch.int32)
    return whole[:, :vocab], tokens


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab,n_top,pad", [(1, 1, 1, 0), (2, 7, 3, 0), (3, 64, 64, 1), (1, 1000, 20, 0), (5, 4097, 5, 3), (40, 32000, 1, 0),
                                                  (2, 128256, 20, 0), (600, 5003, 20, 0), (7, 50257, 64, 5), (300, 20000, 0, 0), (1, 300001, 33, 0),
                                                  (520, 40001, 17, 1), (3, 2100000, 64, 0)])
def test_against_64_bits(rows, vocab, n_top, pad, dtype):
    print("logprobs", rows, vocab, n_top, pad, dtype, flush=True)
    logits, tokens = make(rows, vocab, dtype, 1, pad)
    check(logits, tokens, n_top, "random")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(2, 40000), (300, 9001), (3, 700)])
def test_ties(rows, vocab, dtype):
    """Equal logits: the lower token first; many of them, some, all, in rising and in falling order."""
    logits, tokens = make(rows, vocab, dtype, 2)
    at = torch.arange(vocab, device="cuda")
    kinds = [torch.zeros(vocab), (at % 3 == 1).float(), (at % 1001 == 700).float() * 5, -(at // 64).float(), (at // 64).float(),
             (at // 4096).float(), torch.where(at % 2 == 0, 0.0, -0.0)]
    for i, kind in enumerate(kinds):
        logits[i % rows] = kind.to(logits)
        if i % rows == rows - 1 or i == len(kinds) - 1:
            for n_top in (1, 20, 64):
                check(logits, tokens, n_top, f"ties up to {i}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [33, 5000, 70001])
def test_masked_entries_and_rows_without_a_distribution(vocab, dtype):
    inf, nan = float("inf"), float("nan")
    logits, tokens = make(9, vocab, dtype, 3)
    logits[0, 5:] = -inf                                                    # five tokens left
    logits[1] = -inf
    logits[1, vocab - 2] = 3.0                                              # one left: probability 1, entropy 0
    logits[2] = -inf
    logits[3, vocab // 2] = nan
    logits[4, 3] = inf
    logits[5] = nan
    logits[6, ::2] = -inf
    logits[7] = torch.where(torch.arange(vocab, device="cuda") == 4, 80.0, -80.0).to(dtype)
    tokens[:, 0] = vocab - 2
    for n_top in (1, 20, 33):
        check(logits, tokens, n_top, "masked")


def test_what_is_not_asked_for():
    logits, tokens = make(6, 3001, torch.bfloat16, 4)
    full = call(logits, tokens, 5)
    a, b, c = call(logits, None, 5, entropy=False, top_logprob=False), call(logits, tokens, 0, entropy=False), call(logits, None, 0)
    assert a[0] is None and a[1] is None and a[3] is None and torch.equal(a[2], full[2])
    assert torch.equal(b[0].view(torch.int32), full[0].view(torch.int32)) and torch.equal(c[1], full[1])


def test_rows_beyond_32_bits():
    """A row that starts behind 2^32 elements."""
    small, tokens = make(2, 5001, torch.bfloat16, 5)
    stride = 2 ** 32 + 9
    whole = torch.empty((stride + 5001,), dtype=torch.bfloat16, device="cuda")
    far = whole.as_strided((2, 5001), (stride, 1))
    far.copy_(small)
    for x, y in zip(call(far, tokens, 9)[:4], call(small, tokens, 9)[:4]):
        assert torch.equal(x.view(torch.int32), y.view(torch.int32)) or torch.allclose(x, y, rtol=2 ** -20, atol=2 ** -18, equal_nan=True)


@pytest.mark.parametrize("rows,vocab", [(2, 60000), (600, 3001)])
def test_same_bits_again_a_stream_and_a_graph(rows, vocab):
    logits, tokens = make(rows, vocab, torch.float32, 6)
    *outs, run = call(logits, tokens, 20)
    want = [x.clone() for x in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in outs:
            x.fill_(0)
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        assert all(torch.equal(x.view(torch.int32), y.view(torch.int32)) for x, y in zip(outs, want))
        for x in outs:
            x.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
    assert all(torch.equal(x.view(torch.int32), y.view(torch.int32)) for x, y in zip(outs, want))
