"""pc_token_logprobs over the whole range of its types: masks of the lowest value, some entries and all, logits near the largest, and
large ones in general, where a product with log2 e is out of range or off by more than the logits' differences."""
import numpy as np
import pytest
import torch

from test_gpu_token_logprobs import call, make

pytestmark = pytest.mark.gpu


def reference(x, n_top):
    """log p of every token, the entropy and the top list in 64 bits, from differences to the largest logit; and what the entropy may
    be off: a term p d, d = x - m, moves with d's rounding and the exponential's, 2^-22 + |d| 2^-23 of it, and with the sum's 2^-20."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore", under="ignore"):
        m = x.max(1, keepdims=True)
        d = x - m
        e = np.exp(d)
        l = e.sum(1, keepdims=True)
        lp = d - np.log(l)
        p, some = e / l, np.where(e > 0, d, 0.0)
        ent = np.log(l)[:, 0] - (p * some).sum(1)
        bound = 2.0 ** -18 + (p * np.abs(some)).sum(1) * 2.0 ** -19 + (p * some * some).sum(1) * 2.0 ** -22
    none = ~np.isfinite(m[:, 0])                                            # NaN, +inf or nothing but -inf
    lp[none], ent[none] = np.nan, np.nan
    order = np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -np.where(np.isnan(x), -np.inf, x), np.isnan(x)), axis=1)[:, :n_top]
    return lp, ent, bound, order


def check(logits, tokens, n_top, what):
    """A log probability is (x - m) - log l: the difference's rounding and the result's, 2^-22 of it, and log l's 2^-18."""
    token_lp, ent, top, top_lp, _ = call(logits, tokens, n_top)
    lp, want_ent, ent_bound, want_top = reference(logits.double().cpu().numpy(), n_top)
    t = tokens.cpu().numpy()
    want_tok = np.where((t >= 0) & (t < lp.shape[1]), np.take_along_axis(lp, np.clip(t, 0, lp.shape[1] - 1), 1), np.nan)
    assert np.array_equal(top.cpu().numpy(), want_top), f"{what}: top_idx"
    for got, want, bound, name in ((token_lp, want_tok, None, "token_logprob"), (top_lp, np.take_along_axis(lp, want_top, 1), None, "top_logprob"),
                                   (ent, want_ent, ent_bound, "entropy")):
        got = got.cpu().numpy().astype(np.float64)
        with np.errstate(over="ignore"):
            out = np.isinf(want.astype(np.float32))                         # out of the result's range
        assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: {name}, NaN in other places"
        assert np.array_equal(got[out], np.copysign(np.inf, want[out])), f"{what}: {name}, infinities"
        fine = ~out & ~np.isnan(want)
        off = np.abs(got[fine] - want[fine])
        most = (2.0 ** -18 + 2.0 ** -22 * np.abs(want) if bound is None else bound)[fine]
        assert np.all(off <= most), f"{what}: {name} off by {off.max():.3e}, row {np.argwhere(fine)[np.argmax(off - most)]}"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [33, 5000, 120001])
def test_lowest_and_largest_values(vocab, dtype):
    print("logprobs range", vocab, dtype, flush=True)
    lo, hi = torch.finfo(dtype).min, torch.finfo(dtype).max
    logits, tokens = make(14, vocab, dtype, 7)
    noise = logits.float().clone()
    logits[0, ::3] = lo                                                     # masked with the lowest value: some,
    logits[1] = lo                                                          # all,
    logits[2] = lo
    logits[2, vocab // 2] = 3.0                                             # all but one
    logits[3] = hi                                                          # the largest: all, some
    logits[4, 1::5] = hi
    logits[5], logits[5, 2::4] = lo, hi                                     # a difference beyond the range
    logits[6] = (noise[6] * 1e37).to(dtype)
    logits[7] = (noise[7] * 2.0 ** 31).to(dtype)
    logits[8] = torch.where(noise[8] > 1, 2.0 ** 40, -2.0 ** 50).to(dtype)
    logits[9] = lo
    logits[9, ::2] = float("-inf")                                          # the lowest value is above this
    logits[10] = lo
    logits[10, 7] = float("nan")
    logits[11] = hi
    logits[11, 9] = float("inf")
    logits[12] = (noise[12].abs() * lo / 16).to(dtype)                      # nothing but large negative ones
    tokens[:, 0], tokens[:, 1] = vocab // 2, 0
    for n_top in (1, 20, 33):
        check(logits, tokens, n_top, f"range, {n_top}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [700, 60000])
@pytest.mark.parametrize("offset", [0.0, 300.0, -5e3, 1e6, -3e7, 4e9])
def test_an_offset_of_all_logits(offset, vocab, dtype):
    """A row's numbers hang on the logits' differences alone."""
    logits, tokens = make(5, vocab, torch.float32, 8)
    logits = (logits + offset).to(dtype)
    tokens[:, 0] = 5
    check(logits, tokens, 20, f"offset {offset}")
