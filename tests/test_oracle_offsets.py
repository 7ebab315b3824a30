"""The plain attention of several new tokens where some of a row's tokens are not given."""
import numpy as np

from oracle import paged


def test_tokens_that_are_not_given_leave_the_others_their_positions():
    rng = np.random.default_rng(4)
    K, V = rng.normal(size=(2, 9, 2, 3, 16)).astype(np.float32)
    table, kv = np.array([[2, 0, 5], [1, 7, 8]], np.int32), np.array([7, 9])
    q = rng.normal(size=(8, 4, 16)).astype(np.float32)
    off = np.array([0, 3, 8])
    want, _ = paged.paged_chunk_attn(q, K, V, table, kv, off)
    for n in range(1, 8):
        got, _ = paged.paged_chunk_attn(q[:n], K, V, table, kv, off)
        assert np.array_equal(got, want[:n])
    # by hand: the second row's first token, of five, is at position 4 and attends 5
    one = paged.paged_attn(q[3:4], K, V, table[1:], np.array([5]))
    assert np.allclose(want[3], one[0], rtol=0, atol=1e-13)


def test_refused_rows_name_no_page_where_they_wanted_one():
    table = np.array([[1, 0, 0, 0], [2, 0, 0, 0], [3, 0, 0, 0]], np.int32)
    free = np.array([4, 5, 9, 9, 9, 9])
    r = paged.paged_resize(table, np.array([4, 4, 4]), np.array([12, 9, 100]), free, 2, 4, 30)
    assert r["table"].tolist() == [[1, 5, 4, 0], [2, -1, -1, 0], [3, -1, -1, -1]]
    assert r["kv_len"].tolist() == [12, 4, 4] and r["free_count"] == 0
    assert (r["slots"][8:] == -1).all()
