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
