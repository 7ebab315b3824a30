"""The fp64 forms of the paged cache and the sampling pinned by hand-worked
values, closed forms and invariants."""
import math

import numpy as np
import pytest

from oracle import paged


def test_append_by_hand():
    K = np.zeros((3, 1, 2, 16), np.float32)
    V = np.zeros_like(K)
    k = np.arange(5, dtype=np.float32)[:, None, None] + np.ones((5, 1, 16), np.float32)
    table = np.array([[2, 0], [1, 7]], np.int32)
    # row 0: tokens 0..2 to positions 1..3; row 1: token 3 to position 2 (a page
    # outside the cache: skipped); token 4 is of no row
    K2, V2 = paged.paged_append(K, V, k, -k, table, np.array([1, 2]), np.array([0, 3, 4]))
    want = np.zeros((3, 2))
    want[2, 1], want[0, 0], want[0, 1] = 1, 2, 3
    assert np.array_equal(K2[:, 0, :, 0], want) and np.array_equal(V2, -K2)
    assert not K.any()


def test_attention_of_one_position_is_its_value():
    rng = np.random.default_rng(0)
    K, V = rng.normal(size=(2, 4, 2, 3, 16)).astype(np.float32)
    out = paged.paged_attn(rng.normal(size=(1, 4, 16)).astype(np.float32), K, V, np.array([[2]]), np.array([1]))
    assert np.array_equal(out[0, 0], V[2, 0, 0].astype(np.float64))
    assert np.array_equal(out[0, 3], V[2, 1, 0].astype(np.float64))


def test_attention_equal_keys_give_the_mean_and_bad_pages_are_left_out():
    rng = np.random.default_rng(1)
    K = np.ones((4, 1, 2, 16), np.float32)
    V = rng.normal(size=K.shape).astype(np.float32)
    q = rng.normal(size=(1, 1, 16)).astype(np.float32)
    out = paged.paged_attn(q, K, V, np.array([[3, -1, 1]]), np.array([5]))
    want = np.mean([V[3, 0, 0], V[3, 0, 1], V[1, 0, 0]], axis=0, dtype=np.float64)
    assert np.allclose(out[0, 0], want, rtol=1e-15, atol=1e-15)
    assert not paged.paged_attn(q, K, V, np.array([[9, -1, 4]]), np.array([5])).any()
    assert not paged.paged_attn(q, K, V, np.array([[3, 2, 1]]), np.array([0])).any()


def test_attention_with_the_new_token_equals_append_then_attend():
    rng = np.random.default_rng(2)
    K, V = rng.normal(size=(2, 6, 2, 4, 16)).astype(np.float32)
    q = rng.normal(size=(2, 4, 16)).astype(np.float32)
    k, v = rng.normal(size=(2, 2, 2, 16)).astype(np.float32)
    table, n = np.array([[0, 1], [5, 3]]), np.array([7, 3])
    out, K2, V2 = paged.paged_attn(q, K, V, table, n, k, v)
    K3, V3 = paged.paged_append(K, V, k, v, table, n - 1)
    assert np.array_equal(K2, K3) and np.array_equal(V2, V3)
    assert np.array_equal(out, paged.paged_attn(q, K3, V3, table, n))


def draw(x, us, **kw):
    R = len(us)
    full = {n: np.full(R, a) for n, a in kw.items()}
    return paged.token_sample(np.tile(np.asarray(x, np.float32), (R, 1)), np.asarray(us), **full)


def test_sampling_by_hand():
    # weights 1/2, 1, 1/4, 1/4 of a total of 2
    x = np.log([2, 4, 1, 1])
    us = [0.0, 0.24, 0.26, 0.74, 0.76, 0.88]
    tok, lp = draw(x, us)
    assert tok.tolist() == [0, 0, 1, 1, 2, 3]
    assert np.allclose(lp, np.log([.25, .25, .5, .5, .125, .125]), atol=1e-7)
    # top-k 3: of the two equal ones the first index; a total of 7/4
    tok, lp = draw(x, [0.0, 0.29, 0.84, 0.87, 0.99], top_k=3)
    assert tok.tolist() == [0, 1, 1, 2, 2] and math.isclose(lp[4], math.log(1 / 7), abs_tol=1e-6)
    # top-p 0.6: 1 lies before the second (less than 0.6 * 2), 1.5 before the third
    tok, _ = draw(x, [0.0, 0.3, 0.4, 0.99], top_p=0.6)
    assert tok.tolist() == [0, 0, 1, 1]
    assert draw(x, [0.99], top_p=0.4)[0].tolist() == [1]
    assert draw(x, [0.99], top_p=0.0)[0].tolist() == [1]
    # min-p 0.4 keeps the weights 1 and 1/2
    assert draw(x, [0.3, 0.99], min_p=0.4)[0].tolist() == [0, 1]
    assert draw(x, [0.0, 0.99], min_p=7.0)[0].tolist() == [1, 1]
    # temperature 2: weights sqrt
    assert math.isclose(draw(x, [0.0], temperature=2.0)[1][0], math.log(2 ** .5 / (2 + 2 ** .5 + 2)), abs_tol=1e-6)
    tok, lp = draw([1, 3, 3, 2], [0.9], temperature=0.0)
    assert tok[0] == 1 and lp[0] == 0


def test_rows_with_no_distribution_and_bans():
    inf = np.inf
    for x, T in (([np.nan, 1], 1), ([inf, 1], 1), ([-inf, -inf], 1), ([0, 1], -1), ([0, 1], np.nan)):
        tok, lp = draw(x, [0.5], temperature=T)
        assert tok[0] == -1 and np.isnan(lp[0])
    assert draw([-inf, 0, -inf, 0], [0.0, 0.49, 0.5, 1.0, np.nan])[0].tolist() == [1, 1, 3, 3, 3]
    low = np.finfo(np.float32).min
    assert draw([low, low], [0.0, 0.6])[0].tolist() == [0, 1]   # masked by the lowest value alone: still a row


@pytest.mark.parametrize("kw", [{}, dict(top_k=5), dict(top_p=0.7), dict(min_p=0.1), dict(top_k=9, top_p=0.8, min_p=0.05)])
def test_frequencies_are_the_kept_probabilities(kw):
    rng = np.random.default_rng(3)
    x = rng.normal(size=20) * 2
    us = (np.arange(20000) + 0.5) / 20000
    tok, lp = draw(x, us, **kw)
    f = np.bincount(tok, minlength=20) / len(us)
    p = np.zeros(20)
    p[tok] = np.exp(lp)
    assert np.abs(f - p).max() <= 1 / 20000 + 1e-12
    # a token of probability 1/20000 or more spans one of the 20000 midpoints at
    # least, so each token that was never drawn has less than that
    assert -1e-9 <= 1 - p.sum() <= np.count_nonzero(p == 0) / 20000 + 1e-9


def test_a_token_past_its_rows_table_is_neither_written_nor_attended():
    """A row of two positions, both held: a new token at length 3 has no place, at
    length 2 it is the second."""
    K = np.arange(4, dtype=np.float32).reshape(1, 1, 2, 2)
    V = K + 10
    q, table = np.zeros((1, 1, 2), np.float32), np.zeros((1, 1), np.int32)
    k, v = np.full((1, 1, 2), 50, np.float32), np.full((1, 1, 2), 70, np.float32)
    out, K3, V3 = paged.paged_attn(q, K, V, table, [3], k, v)
    assert (K3 == K).all() and (V3 == V).all()
    np.testing.assert_array_equal(out[0, 0], [11, 12])   # the mean of [10, 11] and [12, 13]
    out, K2, V2 = paged.paged_attn(q, K, V, table, [2], k, v)
    assert (K2[0, 0, 1] == 50).all() and (V2[0, 0, 1] == 70).all()
    np.testing.assert_array_equal(out[0, 0], [40, 40.5])
