"""The fp64 forms of growing rows, rotary positions and the attention of several new tokens
pinned by hand-worked values, closed forms and invariants."""
import math

import numpy as np

from oracle import paged


def test_resize_by_hand():
    # pages of 2: row 0 holds 3 positions in pages 5, 1; row 1 holds 4 in 0, 3; row 2 none
    table = np.array([[5, 1, -1], [0, 3, -1], [-1, -1, -1]], np.int32)
    free = np.array([2, 4, 9, 9, 9, 9], np.int32)   # 4 on top
    got = paged.paged_resize(table, np.array([3, 4, 0]), np.array([5, 1, 3]), free, 2, 2, 7)
    # row 1 gives back its second page, 3; then row 0 takes one (3), row 2 two (4, 2)
    assert got["table"].tolist() == [[5, 1, 3], [0, -1, -1], [4, 2, -1]]
    assert got["kv_len"].tolist() == [5, 1, 3] and got["free_count"] == 0
    assert got["start"].tolist() == [3, 4, 0] and got["offsets"].tolist() == [0, 2, 2, 5]
    assert got["positions"].tolist() == [3, 4, 0, 1, 2, 0, 0] and got["slots"].tolist() == [3, 6, 8, 9, 4, -1, -1]
    # none is left: row 0 has room for one position more in its last page, row 2 has not
    got = paged.paged_resize(got["table"], got["kv_len"], np.array([6, 1, 5]), free, 0, 2, 3)
    assert got["kv_len"].tolist() == [6, 1, 3] and got["slots"].tolist() == [7, -1, -1] and got["positions"].tolist() == [5, 3, 4]


def test_resize_there_and_back():
    rng = np.random.default_rng(0)
    held, more = rng.integers(0, 50, 9), rng.integers(0, 60, 9)
    need = -(-held // 4)
    ids = rng.permutation(int(need.sum()) + 100).astype(np.int32)
    table = np.full((9, 30), -1, np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    free = np.concatenate([ids[at:], np.zeros(at, np.int32)])
    a = paged.paged_resize(table, held, more, free, len(ids) - at, 4)
    b = paged.paged_resize(a["table"], a["kv_len"], held, a["free_pages"], a["free_count"], 4)
    assert np.array_equal(b["table"], table) and np.array_equal(b["free_pages"][:b["free_count"]], ids[at:])
    used = np.concatenate([a["table"][a["table"] >= 0], a["free_pages"][:a["free_count"]]])
    assert np.array_equal(np.sort(used), np.arange(len(ids)))   # every page once


def test_rotary_by_hand():
    x = np.zeros((2, 1, 16), np.float32)
    x[:, 0, 0], x[:, 0, 1], x[:, 0, 9] = 1, 2, 7
    quarter = np.array([math.pi / 2])
    got = paged.rotary(x, np.array([1, 2]), quarter, interleaved=True)[:, 0]
    assert np.allclose(got[:, :2], [[-2, 1], [-1, -2]]) and (got[:, 9] == 7).all()
    got = paged.rotary(x, np.array([-1, 0]), np.array([math.pi / 2, 0.0]), magnitude=3.0)[:, 0]
    # halves of four elements: pairs (0, 2) and (1, 3); the second does not turn
    assert np.allclose(got[:, :4], [[0, 6, -3, 0], [3, 6, 0, 0]])


def test_rotary_scores_depend_on_the_distance():
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(2, 1, 1, 32)).astype(np.float32)
    f = paged.rotary_frequencies(32)
    at = lambda x, p, i: paged.rotary(x, [p], f, i)[0, 0]
    for i in (False, True):
        assert abs(at(q, 1000, i) @ at(k, 990, i) - at(q, 10, i) @ at(k, 0, i)) < 1e-11
        assert np.allclose(np.linalg.norm(at(q, 77, i)), np.linalg.norm(q))


def test_frequencies():
    f = paged.rotary_frequencies(8, 10000.0)
    assert np.allclose(f, [1, 0.1, 0.01, 0.001])
    assert np.allclose(paged.rotary_frequencies(8, 10000.0, 4.0), f / 4)
    # 628.3 positions: 100, 10, 1 and 0.1 turns; between 1 and 19 turns mixed
    g = paged.rotary_frequencies(8, 10000.0, 4.0, context=628, fast=19.0, slow=1.0)
    turns = 62.8 / (2 * math.pi)
    keep = (turns - 1) / 18
    assert np.allclose(g, [1, 0.1 * keep + 0.025 * (1 - keep), 0.0025, 0.00025], rtol=1e-12)


def test_chunk_attention_against_one_token_at_a_time():
    rng = np.random.default_rng(2)
    K, V = rng.normal(size=(2, 9, 2, 3, 16)).astype(np.float32)
    table = np.array([[2, 0, 5], [1, -1, 8]], np.int32)   # a page is missing
    q = rng.normal(size=(7, 4, 16)).astype(np.float32)
    off, kv = np.array([1, 4, 6]), np.array([7, 9])
    out, mean = paged.paged_chunk_attn(q, K, V, table, kv, off)
    assert np.isnan(out[[0, 6]]).all() and (np.abs(out[1:6]) <= mean[1:6] + 1e-12).all()
    for r in range(2):
        for i, n in enumerate(range(off[r], off[r + 1])):
            p = kv[r] - (off[r + 1] - off[r]) + i
            one = paged.paged_attn(q[n:n + 1], K, V, table[r:r + 1], np.array([p + 1]))
            assert np.allclose(out[n], one[0], rtol=0, atol=1e-13)


def test_chunk_attention_of_nothing():
    K = np.ones((2, 1, 2, 16), np.float32)
    q = np.ones((3, 1, 16), np.float32)
    out, _ = paged.paged_chunk_attn(q, K, K, np.array([[0, 1]]), np.array([1]), np.array([0, 3]))
    assert not out[:2].any() and (out[2] == 1).all()   # tokens before position 0
