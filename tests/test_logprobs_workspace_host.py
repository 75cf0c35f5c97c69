"""pc_token_logprobs_workspace_bytes: places for rows that are cut into parts alone, no less for fewer rows or a smaller vocabulary."""
import pytest

import paper_2502_14317_amd as pc

NEED = pc.pc_token_logprobs_workspace_bytes


def test_rows_that_are_not_cut_need_none():
    for rows, vocab in ((1, 1), (1 << 21, 1), (1 << 21, 32000), (65, 49152), (4096, 49152)):
        assert 0 < NEED(rows, vocab, min(64, vocab)) <= 512, (rows, vocab)


@pytest.mark.parametrize("n_top", [0, 5, 64])
def test_sizes_grow_with_rows_and_vocabulary(n_top):
    most = 0
    for vocab in (100, 32000, 49152, 49153, 60000, 98304, 128256, 300001, 1 << 20, 1 << 24):
        sizes = [NEED(rows, vocab, n_top) for rows in (1, 2, 3, 5, 12, 22, 43, 51, 63, 64, 65, 100, 256, 257, 2048, 1 << 21)]
        assert sizes == sorted(sizes), vocab
        assert sizes[-1] >= most and sizes[-1] <= 256 * (12 + 8 * n_top) + 3 * 256, vocab       # 256 parts in all
        most = sizes[-1]


def test_places_for_every_part():
    """(A part: a maximum and two sums, and its list.)"""
    for rows, vocab, parts in ((1, 128256, 31), (4, 128256, 31), (8, 300001, 32), (64, 128256, 4), (1, 1 << 24, 256), (3, 1 << 24, 85)):
        for n_top in (0, 20, 64):
            assert NEED(rows, vocab, n_top) >= rows * parts * (12 + 8 * n_top), (rows, vocab)
