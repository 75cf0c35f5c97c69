"""PagedTreeDecoder.load: what it refuses leaves the sequence, its pages and the step at hand as they were."""
import pytest
import torch

import paper_2502_14317_amd as pc
from paper_2502_14317_amd.layer import PagedTreeDecoder

pytestmark = pytest.mark.gpu

B, Hq, Hkv, D, KT, N0 = 2, 4, 2, 64, 20, 3


def mk(*shape, gen=torch.Generator().manual_seed(4)):
    return torch.randn(shape, generator=gen).to(torch.bfloat16).cuda()


def state(d):
    return [d.len.tolist(), d.pos.tolist(), d.table.tolist(), [list(p or []) for p in d.pages], list(d.free), list(d.most)]


def wide(t):
    """The same values with rows 4 values further apart."""
    return torch.cat([t, t[..., :4]], -1)[..., :D]


def odd(t):
    """The same values at an address that is no multiple of 16 bytes."""
    whole = torch.zeros((t.numel() + 1,), dtype=t.dtype, device="cuda")
    whole[1:] = t.flatten()
    return whole[1:].view(t.shape)


turned = lambda t: t.transpose(2, 3).contiguous().transpose(2, 3)           # values of a row apart
other = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)            # rows in another order
one_place = lambda t: t[:1, :1, :1].expand(t.shape)
BAD = {"turned": dict(kc=turned, vc=turned), "kc alone": dict(kc=other), "vc turned": dict(vc=turned), "vc alone": dict(vc=other), "kc elsewhere": dict(kc=torch.Tensor.cpu),
       "vc elsewhere": dict(vc=torch.Tensor.cpu), "both elsewhere": dict(kc=torch.Tensor.cpu, vc=torch.Tensor.cpu), "row strides": dict(kc=wide, vc=wide),
       "kc's address": dict(kc=odd), "vc's address": dict(vc=odd), "one place": dict(kc=one_place, vc=one_place),
       "k_tail elsewhere": dict(k_tail=torch.Tensor.cpu), "v_tail elsewhere": dict(v_tail=torch.Tensor.cpu), "k_tail's address": dict(k_tail=odd),
       "v_tail's address": dict(v_tail=odd), "position": dict(pos=lambda p: 2 ** 31), "no position": dict(pos=lambda p: "first"),
       "no number": dict(pos=lambda p: None), "no sequence": dict(b=lambda b: B)}


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("eight_bit", [False, True], ids=["bf16", "row8"])
def test_a_refused_load_leaves_everything_as_it_was(eight_bit, bad):
    d, same = (PagedTreeDecoder(B, 8, 16, 4, Hq, Hkv, D, 1e4, max_rows=2, eight_bit=eight_bit) for _ in range(2))
    doc, tail, q, k, v = mk(2, Hkv, KT, D), mk(N0, Hkv, D), mk(B, 2, Hq, D), mk(B, 2, Hkv, D), mk(B, 2, Hkv, D)
    tokens = torch.ones((B, 2), dtype=torch.int32, device="cuda")
    for x in (d, same):
        for b in range(B):
            x.load(b, doc + b, doc - b, 40 + b)
        x.step(q, k, v)
    good = dict(b=1, kc=mk(2, Hkv, KT, D), vc=mk(2, Hkv, KT, D), pos=77, k_tail=tail, v_tail=-tail)
    before = state(d)
    with pytest.raises((ValueError, TypeError, IndexError, pc.PcError)):
        d.load(**{name: BAD[bad].get(name, lambda x: x)(x) for name, x in good.items()})
    assert state(d) == before
    for x in (d, same):
        x.accept(tokens, tokens)                                            # the step at hand is still there
    assert state(d) == state(same) and torch.equal(d.step(q, k, v), same.step(q, k, v))
    for x in (d, same):
        x.load(**good)
    assert torch.equal(d.step(q, k, v), same.step(q, k, v)) and d.pos.tolist() == same.pos.tolist()


def test_sequences_counted_from_the_last_one():
    d, same = (PagedTreeDecoder(B, 8, 16, 4, Hq, Hkv, D, 1e4, max_rows=2) for _ in range(2))
    doc, tail, q, k, v = mk(1, Hkv, KT, D), mk(N0, Hkv, D), mk(B, 2, Hq, D), mk(B, 2, Hkv, D), mk(B, 2, Hkv, D)
    for x, last in ((d, -1), (same, 1)):
        x.load(0, doc, doc, 20)
        x.load(last, -doc, doc, 23, k_tail=tail, v_tail=tail)
    assert state(d) == state(same) and torch.equal(d.step(q, k, v), same.step(q, k, v))
