"""Pins of the paged-cache oracle: closed forms, tiny cases by hand, reduction to the dense attention oracle."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from oracle import pafu_oracle as orc


def test_tables_by_hand():
    table = np.full((3, 4), -7)
    table[0, 0], table[2, :2] = 5, (9, 2)
    got, slots, row_start, kv_out, end = po.paged_tables([3, 0, 16], [6, 0, 1], [11, 12, 13, 14], 8, table, 9, free_start=1)
    # request 0: tokens 3..8: five on page 5 (places 3..7), one on a new page; request 2: token 16 on a new page
    assert got.tolist() == [[5, 12, -7, -7], [-7] * 4, [9, 2, 13, -7]]
    assert slots.tolist() == [43, 44, 45, 46, 47, 96, 104, -1, -1]
    assert row_start.tolist() == [0, 6, 6, 7] and kv_out.tolist() == [9, 0, 17] and end == 3


def test_tables_when_the_list_or_the_table_ends():
    got, slots, _, _, end = po.paged_tables([0, 0], [9, 9], [3], 8, np.full((2, 1), -9), 18)
    assert got.tolist() == [[3], [-1]] and end == 4                 # four pages wanted, one there; one column
    assert slots.tolist() == list(range(24, 32)) + [-1] * 10


def test_slots_invert_the_table():
    rng = np.random.default_rng(0)
    table = rng.permutation(40).reshape(4, 10)
    slots, row_start = po.paged_slots(table, [0, 5, 79, 80], [80, 11, 1, 2], 8, 94)
    assert row_start.tolist() == [0, 80, 91, 92, 94]
    tokens = [(0, j) for j in range(80)] + [(1, j) for j in range(5, 16)] + [(2, 79)]
    for (b, j), s in zip(tokens, slots):
        assert s // 8 == table[b, j // 8] and s % 8 == j % 8
    assert slots[92:].tolist() == [-1, -1]                          # beyond the table


@pytest.mark.parametrize("window,pinned,want", [(0, 3, list(range(9))), (4, 0, [5, 6, 7, 8]), (4, 2, [0, 1, 5, 6, 7, 8]),
                                                (4, 6, list(range(9))), (20, 1, list(range(9)))])
def test_visible_tokens(window, pinned, want):
    assert po.visible_tokens(9, pinned, window) == want
    assert po.visible_tokens(0, pinned, window) == po.visible_tokens(-3, pinned, window) == []


def test_attention_is_the_dense_oracle_on_the_gathered_rows():
    rng = np.random.default_rng(1)
    K, V = (rng.standard_normal((6, 8, 2, 64)) for _ in range(2))
    Q = rng.standard_normal((2, 2, 64))
    table = np.array([[4, 0, 2], [1, 5, 3]])
    got = po.paged_attention(Q, K, V, table, [19, 8])
    for b, n in ((0, 19), (1, 8)):
        rows = [(table[b, j // 8], j % 8) for j in range(n)]
        k, v = (np.stack([x[p, o] for p, o in rows]) for x in (K, V))
        want = orc.chunk_attention(Q[b:b + 1], k[:-1], v[:-1], k[-1:], v[-1:], 1)   # the last token as a chunk of one
        assert np.allclose(got[b], want[0], rtol=0, atol=1e-12)


def test_attention_closed_forms():
    rng = np.random.default_rng(2)
    K, V = rng.standard_normal((3, 8, 1, 64)), rng.standard_normal((3, 8, 1, 64))
    table = np.array([[2, 7, -1, 0]])
    # shared heads, a zero query: the mean of the visible values; pages 7 and -1 are outside
    got = po.paged_attention(np.zeros((1, 4, 64)), K, V, table, [30])
    want = np.concatenate([V[2, :, 0], V[0, :6, 0]]).mean(0)
    assert np.allclose(got[0], want[None], atol=1e-14)
    assert np.all(po.paged_attention(np.zeros((1, 4, 64)), K, V, table, [0]) == 0)
    assert np.allclose(po.paged_attention(rng.standard_normal((1, 4, 64)), K, V, table, [1])[0], V[2, 0], atol=1e-14)
