"""PagedTreeDecoder on the CPU, over a stand-in for the library that keeps the lengths as the calls do: which rows it finds pages for, what
it reads from the device for that, and which steps may be accepted."""
import pytest
import torch

from paper_2502_14317_amd import layer

HQ, HKV, D, PAGE = 4, 2, 64, 16


class Library:
    """Lengths as pc_kv_append_paged and pc_tree_accept leave them; `kept` says how many nodes stand at most."""

    def __init__(self):
        self.calls, self.kept = [], 64

    def make_page_cache(self, *tensors):
        return tensors

    def alloc_workspace(self, n, device):
        return object()

    def pc_tree_attn_workspace_bytes(self, *sizes):
        return 256

    def rows(self, n_rows, n, like):
        return torch.full_like(like, n) if n_rows is None else n_rows.clamp(0, n)

    def pc_kv_append_paged(self, k, v, batch, n, hkv, d, cache, len_in, len_out, n_rows=None, **more):
        self.calls.append(("append", n))
        if len_out is not None:
            len_out.copy_(len_in.clamp(min=0) + self.rows(n_rows, n, len_in))

    def pc_tree_attn(self, q, *args, **more):
        self.calls.append(("attention", q.shape[1]))

    def pc_tree_accept(self, tokens, parent, choice, batch, n, path, n_kept, next_token, len_in, len_out, pos, n_rows=None, **more):
        self.calls.append(("accept", n))
        rows = self.rows(n_rows, n, len_in)
        kept = rows.clamp(max=self.kept)
        len_out.copy_(len_in - rows + kept)
        pos += kept


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(layer, "B", lib)
    return lib


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def decoder(lens, n_pages=12, max_pages=4, max_rows=4):
    d = layer.PagedTreeDecoder(len(lens), n_pages, PAGE, max_pages, HQ, HKV, D, 1e4, max_rows=max_rows, device="cpu")
    for b, x in enumerate(lens):
        if x is not None:
            d.load(b, bf(1, HKV, x, D), bf(1, HKV, x, D), x)
    return d


def step(d, n, n_rows=None, **more):
    d.step(bf(d.B, n, HQ, D), bf(d.B, n, HKV, D), bf(d.B, n, HKV, D), n_rows=None if n_rows is None else i32(n_rows), **more)


def accept(d, n):
    d.accept(torch.zeros((d.B, n), dtype=torch.int32), torch.zeros((d.B, n), dtype=torch.int32))


def i32(x):
    return torch.tensor(x, dtype=torch.int32)


def test_a_full_sequence_that_does_not_take_part(lib):
    """It has no place left, and needs none: the others go on, and no page is taken for it."""
    d = decoder([64, 10])
    for _ in range(9):
        step(d, 4, [0, 4])
        accept(d, 4)
    assert d.len.tolist() == [64, 46] and [len(p) for p in d.pages] == [4, 3] and len(d.free) == 5
    lib.calls.clear()
    with pytest.raises(ValueError, match="do not fit"):                     # it takes part again
        step(d, 4, [1, 4])
    with pytest.raises(ValueError, match="do not fit"):
        step(d, 1)
    assert lib.calls == [] and d.len.tolist() == [64, 46]


def test_idle_sequences_take_no_pages(lib):
    d = decoder([16, 16, 15], n_pages=5)
    for _ in range(3):
        step(d, 4, [0, 4, 1])
        accept(d, 4)
    assert d.len.tolist() == [16, 28, 18] and [len(p) for p in d.pages] == [1, 2, 2] and not d.free
    step(d, 4, [-3, 4, 0])                                                  # (fewer than none)
    accept(d, 4)
    assert d.len.tolist() == [16, 32, 18]


def test_trees_of_fewer_nodes_than_the_widest(lib):
    """Room for a sequence's own nodes, not for as many as the step has."""
    d = decoder([62, 20])
    step(d, 4, [2, 9])                                                      # (more than there are: all four)
    accept(d, 4)
    assert d.len.tolist() == [64, 24] and d.most == [64, 24]
    with pytest.raises(ValueError, match="do not fit"):
        step(d, 4, [1, 1])


def test_lengths_are_read_only_where_a_sequence_could_pass_its_pages(lib, monkeypatch):
    d = decoder([20, 20])
    read = []
    tolist = torch.Tensor.tolist
    monkeypatch.setattr(torch.Tensor, "tolist", lambda t: (read.append(tuple(t.shape)), tolist(t))[1])
    for _ in range(3):                                                      # 12 rows more: 32, the two pages' end
        step(d, 4, [4, 4])
        accept(d, 4)
    assert read == []
    step(d, 4, [4, 4])
    assert read and [len(p) for p in d.pages] == [3, 3]
    read.clear()
    accept(d, 4)
    step(d, 4)
    assert read == []


def test_sequences_that_are_not_loaded_take_no_pages(lib):
    d = decoder([30, None])
    for _ in range(8):
        step(d, 4, [4, 0])
        accept(d, 4)
    assert d.len.tolist() == [62, 0] and d.pages[1] is None


def test_steps_and_acceptances_are_captured_together(lib, monkeypatch):
    """The host does not see replays: an acceptance outside would be one for all of them, and one inside would move lengths unseen."""
    d = decoder([20, 20])
    capture = lambda on: monkeypatch.setattr(layer, "_capturing", lambda t: on)
    capture(True)
    step(d, 3)
    capture(False)
    for _ in range(2):
        lib.calls.clear()
        with pytest.raises(ValueError, match="graph"):
            accept(d, 3)
        assert lib.calls == []
    capture(True)
    accept(d, 3)                                                            # in a graph behind it
    capture(False)
    with pytest.raises(ValueError, match="no step"):
        accept(d, 3)
    before = d.len.tolist()
    step(d, 2)
    capture(True)
    lib.calls.clear()
    with pytest.raises(ValueError, match="graph"):
        accept(d, 2)
    assert lib.calls == []
    capture(False)
    accept(d, 2)                                                            # the step is still at hand
    assert d.len.tolist() == [x + 2 for x in before]
    capture(True)
    step(d, 4)
    capture(False)
    step(d, 1)                                                              # an eager step counts for itself
    accept(d, 1)
    assert d.len.tolist() == [x + 3 for x in before]
    d.len.fill_(47)                                                         # what replays leave behind
    step(d, 4)
    assert d.most == [47, 47] and [len(p) for p in d.pages] == [4, 4]


def test_a_release_of_no_sequence_keeps_the_step_at_hand(lib):
    d = decoder([20, 20])
    step(d, 2)
    with pytest.raises(IndexError):
        d.release(2)
    accept(d, 2)
    assert d.len.tolist() == [22, 22]


def test_a_refused_step_leaves_the_bound_of_the_one_at_hand(lib):
    d = decoder([20, 63])
    step(d, 4, [4, 1])
    with pytest.raises(ValueError, match="do not fit"):
        step(d, 2, [1, 2])
    accept(d, 4)
    assert d.len.tolist() == [24, 64] and all(m >= x for m, x in zip(d.most, d.len.tolist()))
    for _ in range(3):                                                      # 36 rows: a third page
        step(d, 4, [4, 0])
        accept(d, 4)
    assert d.len.tolist() == [36, 64] and len(d.pages[0]) == 3


def test_a_step_whose_rows_are_written_over_is_no_longer_at_hand(lib, monkeypatch):
    """An attention that is refused has its append in front of it; an append that is refused has written nothing."""
    d = decoder([20, 20])
    step(d, 2)
    with monkeypatch.context() as m:
        def refuse(*args, **more):
            raise ValueError("refused")
        m.setattr(lib, "pc_kv_append_paged", refuse)
        with pytest.raises(ValueError, match="refused"):
            step(d, 4)
    accept(d, 2)
    assert d.len.tolist() == [22, 22]
    step(d, 2)
    with monkeypatch.context() as m:
        m.setattr(lib, "pc_tree_attn", refuse)
        with pytest.raises(ValueError, match="refused"):
            step(d, 4)
    with pytest.raises(ValueError, match="no step"):
        accept(d, 2)
    step(d, 3)
    accept(d, 3)
    assert d.len.tolist() == [25, 25] and all(m >= x for m, x in zip(d.most, d.len.tolist()))
