"""SharedPrefixDecoder on the CPU, over a stand-in for the library that keeps the lengths as the calls do: what it refuses,
before anything is written, and which rows it counts."""
import pytest
import torch

from paper_2502_14317_amd import layer

B, P, S, KT, CAP, HQ, HKV, D, V = 4, 2, 3, 16, 12, 8, 2, 64, 50


class Library:
    """Lengths as pc_kv_append_row8 and pc_verify_drafts leave them; `accepted` says how many drafts stand."""

    def __init__(self):
        self.calls, self.accepted = [], None

    def make_row_cache(self, *tensors, **lens):
        return object()

    def alloc_workspace(self, n, device):
        return object()

    def pc_shared_attn_workspace_bytes(self, *sizes):
        return 256

    def pc_kv_append_row8(self, k, v, batch, n, cap, hkv, d, k8, v8, ks, vs, len_in, len_out, **rotation):
        self.calls.append(("append", n))
        if len_out is not None:
            assert len_out.data_ptr() != len_in.data_ptr()
            len_out.copy_((len_in.clamp(0, cap) + n).clamp(max=cap))

    def pc_shared_attn(self, q, *args, **kw):
        self.calls.append(("attention", q.shape[1]))

    def pc_verify_drafts(self, draft, *args, len_in, len_out, **kw):
        self.calls.append(("verify", draft.shape[1]))
        len_out.copy_(len_in + 1 + torch.tensor(self.accepted, dtype=torch.int32))


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def rows(n):
    return bf(B, n, HQ, D), bf(B, n, HKV, D), bf(B, n, HKV, D)


def drafts(k):
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    return dict(draft=i32(B, k), draft_prob=torch.zeros(B, k, V), target_prob=torch.zeros(B, k + 1, V), u=torch.zeros(B, k),
                noise=torch.ones(B, V), tokens=i32(B, k + 1), n_accepted=i32(B), ws=None)


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(layer, "B", lib)
    return lib


def decoder(n0=0, eight_bit_prefix=False, max_rows=4):
    d = layer.SharedPrefixDecoder(B, P, S, KT, CAP, HQ, HKV, D, 1e4, 100, max_rows=max_rows, eight_bit_prefix=eight_bit_prefix, device="cpu")
    kc = bf(P, S, HKV, KT, D)
    d.load(kc, kc, k_tail=bf(B, n0, HKV, D) if n0 else None, v_tail=bf(B, n0, HKV, D) if n0 else None)
    return d


def test_a_step_that_would_pass_the_capacity(lib):
    d = decoder(CAP - 2)
    lib.calls.clear()
    before, new = d.len.clone(), d.len_new.clone()
    for n in (3, 4):
        with pytest.raises(ValueError, match="hold 12 rows"):
            d.step(*rows(n))
    assert lib.calls == [] and torch.equal(d.len, before) and torch.equal(d.len_new, new)
    d.step(*rows(2))                                                        # these fit
    d.accept()
    assert d.len.tolist() == [CAP] * B
    with pytest.raises(ValueError, match="hold 12 rows"):
        d.step(*rows(1))


def test_drafts_that_fell_leave_room(lib):
    """The rows of fallen drafts are written over: the count of rows that may stand is settled by the lengths themselves."""
    d = decoder()
    for step in range(4):                                                   # 4 x 4 rows were written, 3 sequences keep 2 of each 4
        d.step(*rows(4))
        lib.accepted = [1, 1, 0, 1]
        d.verify(**drafts(3))
    assert d.len.tolist() == [8, 8, 4, 8]
    d.step(*rows(4))
    lib.accepted = [3, 0, 0, 0]
    d.verify(**drafts(3))
    assert d.len.tolist() == [CAP, 9, 5, 9]
    with pytest.raises(ValueError, match="hold 12 rows"):                   # one sequence is full
        d.step(*rows(1))


def test_a_query_block_longer_than_the_tails(lib):
    with pytest.raises(ValueError, match="hold 12 rows"):
        decoder(CAP + 1)
    assert lib.calls == []
    assert decoder(CAP).len.tolist() == [CAP] * B


def test_a_second_load_starts_anew(lib):
    d = decoder(CAP)
    kc = bf(P, S, HKV, KT, D)
    d.load(kc, kc)
    d.step(*rows(4))
    d.accept()
    assert d.len.tolist() == [4] * B


def test_lengths_and_workspace_stay_where_they_are(lib):
    """What a captured step has taken in: the same lengths are read and written by every step."""
    d = decoder(2)
    at = d.len.data_ptr(), d.len_new.data_ptr()
    for _ in range(2):
        d.step(*rows(1))
        d.accept()
        assert (d.len.data_ptr(), d.len_new.data_ptr()) == at
    assert d.len.tolist() == [4] * B
    ws = d.ws
    d.load(*[bf(P, S, HKV, KT, D)] * 2)
    d.step(*rows(1))
    assert d.ws is ws is not None


def test_verification_of_rows_that_were_not_written(lib):
    d = decoder(2)
    with pytest.raises(ValueError, match="rows of the step"):               # no step at all
        d.verify(**drafts(0))
    with pytest.raises(ValueError, match="rows of the step"):
        d.accept()
    d.step(*rows(2))
    lib.calls.clear()
    with pytest.raises(ValueError, match="rows of the step"):
        d.verify(**drafts(2))
    assert lib.calls == [] and d.len.tolist() == [2] * B
    lib.accepted = [1, 0, 1, 0]
    d.verify(**drafts(1))
    assert d.len.tolist() == [4, 3, 4, 3]
    with pytest.raises(ValueError, match="rows of the step"):               # once only
        d.verify(**drafts(1))
    d.step(*rows(3))                                                        # fewer drafts than rows are fine
    lib.accepted = [0] * 4
    d.verify(**drafts(0))
    assert d.len.tolist() == [5, 4, 5, 4]


def test_steps_in_a_graph_may_be_verified_outside(lib, monkeypatch):
    """Who replays a captured step verifies its rows after every replay."""
    d = decoder(2)
    monkeypatch.setattr(layer, "_capturing", lambda t: True)
    d.step(*rows(3))
    monkeypatch.setattr(layer, "_capturing", lambda t: False)
    lib.accepted = [0] * 4
    for _ in range(3):
        d.verify(**drafts(2))
    with pytest.raises(ValueError, match="rows of the step"):
        d.verify(**drafts(3))
    assert d.len.tolist() == [5] * B
    d.step(*rows(1))                                                        # an eager step counts for itself
    with pytest.raises(ValueError, match="rows of the step"):
        d.verify(**drafts(2))
    d.accept()
    assert d.len.tolist() == [6] * B


def changed(args, **change):
    return {**args, **change}


@pytest.mark.parametrize("eight_bit", [False, True], ids=["16bit", "8bit"])
def test_documents_of_another_shape_or_type(lib, eight_bit):
    """In 8 bits the segments' addresses go to the library: nothing but its own shape and type does.  16-bit ones are copied,
    which converts types."""
    d = decoder(2, eight_bit)
    d.step(*rows(1))
    lib.calls.clear()
    good, tail = bf(P, S, HKV, KT, D), bf(B, 2, HKV, D)
    held = [x.clone() for x in (*d.prefix, d.len, d.len_new)]
    one = good + 1
    bad = [dict(kc=one[:, :1]), dict(vc=one[:, :, :, :KT - 1]), dict(kc=one[:1]), dict(vc=one.view(P, S, HKV, D, KT)), dict(kc=one[None])]
    if eight_bit:
        bad += [dict(kc=one.float()), dict(vc=one.half())]
    bad += [dict(k_tail=tail[:, :1]), dict(v_tail=tail[:1]), dict(k_tail=tail.float()), dict(v_tail=tail.half()), dict(v_tail=None),
            dict(k_tail=None), dict(k_tail=tail[0]), dict(k_tail=bf(B, 2, HQ, D), v_tail=bf(B, 2, HQ, D))]
    for change in bad:
        with pytest.raises(ValueError):
            d.load(**changed(dict(kc=one, vc=one, k_tail=tail, v_tail=tail), **change))
        assert lib.calls == [] and all(torch.equal(x, y) for x, y in zip(held, (*d.prefix, d.len, d.len_new))), change
    d.accept()                                                              # the step at hand is still there
    assert d.len.tolist() == [3] * B
    d.load(good, good, k_tail=tail, v_tail=tail)
    if not eight_bit:
        d.load(one.float(), one.half(), k_tail=tail, v_tail=tail)
        assert torch.equal(d.prefix[0], one) and torch.equal(d.prefix[1], one)


def test_rows_of_another_type(lib):
    d = decoder(2)
    lib.calls.clear()
    for at in range(3):
        for dtype in (torch.float32, torch.float16):
            args = [x.to(dtype) if i == at else x for i, x in enumerate(rows(2))]
            with pytest.raises(ValueError, match="bfloat16"):
                d.step(*args)
    assert lib.calls == [] and d.len_new.tolist() == [2] * B


def test_verification_of_another_shape_or_type(lib):
    d = decoder(2)
    d.step(*rows(4))
    lib.calls.clear()
    lib.accepted = [1] * 4
    good = drafts(3)
    bad = [dict(draft=good["draft"].long()), dict(draft=good["draft"][:2]), dict(draft_prob=good["draft_prob"][:, :2]),
           dict(draft_prob=good["draft_prob"].half()), dict(target_prob=good["target_prob"][:, :3]), dict(target_prob=good["target_prob"].double()),
           dict(draft_prob=good["draft_prob"][:, :, :V - 1]), dict(u=good["u"][:, :2]), dict(u=good["u"].half()), dict(noise=good["noise"][:2]),
           dict(noise=good["noise"].half()), dict(noise=good["noise"][:, :V - 1]), dict(tokens=good["tokens"][:, :3]), dict(tokens=good["tokens"].long()),
           dict(n_accepted=good["n_accepted"][:3]), dict(n_accepted=good["n_accepted"].long()),
           dict(draft_len=torch.zeros(B)), dict(draft_len=torch.zeros(B - 1, dtype=torch.int32))]
    for change in bad:
        with pytest.raises(ValueError):
            d.verify(**changed(good, **change))
        assert lib.calls == [] and d.len.tolist() == [2] * B, change
    d.verify(**changed(good, draft_prob=None, draft_len=torch.zeros(B, dtype=torch.int32)))
    assert d.len.tolist() == [4] * B
