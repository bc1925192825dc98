"""The plan of more new tokens than rows, against hand-worked lengths (CPU)."""
import numpy as np

from oracle import chunk as ref


def test_tokens_without_a_row_are_not_in_the_chunk():
    table = np.array([[5, -1, -1], [3, 4, -1], [-1, -1, -1], [0, 1, -1]])
    out = ref.plan_chunk([3, 6, 0, 7], [2, 3, 9, 1], [1, 2, 0, 2], [9, 8, 7, 6, 2], 5, table, 4, 100, 7)
    # rows: 2 and 3 of the first two sequences, two of the third's nine, none of the last's one
    np.testing.assert_array_equal(out["row_start"], [0, 2, 5, 7, 7])
    np.testing.assert_array_equal(out["kv_len"], [5, 9, 2, 7])
    np.testing.assert_array_equal(out["pos"], [3, 4, 6, 7, 8, 0, 1])
    # a row's position is kv_len - rows + j, as the attention reads it
    m = np.diff(out["row_start"])
    np.testing.assert_array_equal(np.concatenate([k - n + np.arange(n) for k, n in zip(out["kv_len"], m)]), out["pos"])
    # the pages are those of all tokens: 6's second page for sequence 0, one for 1, three for 2
    np.testing.assert_array_equal(out["pages_held"], [2, 3, 3, 2])
    assert out["free_count"][0] == 0 and out["missing"][0] == 0
