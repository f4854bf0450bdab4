"""Pins of the plain 64-bit forms in oracle/decoding.py: hand values and identities
that do not go through their own formulas (no GPU)."""

import numpy as np

from oracle import decoding as D


def test_path_ends_at_links_that_do_not_point_back():
    assert D.path([-1, 0, 1, 2], 3) == [3, 2, 1, 0]
    assert D.path([-1, 0, 5, 2], 3) == [3, 2]
    assert D.path([-1, 0, -4, 0], 2) == [2]


def test_attention_by_hand():
    """Equal scores average the visible values; a weight of e against 1; a sibling is not seen;
    rows of a page behind the context are not read."""
    par = [-1, 0, 0]
    q = np.zeros((3, 2, 2))
    k_new, v_new = np.zeros((3, 1, 2)), np.arange(6.0).reshape(3, 1, 2)
    cache = np.full((2, 1, 2, 2), np.nan)
    cache[1, 0, 0] = (10.0, 20.0)
    kc = np.where(np.isnan(cache), np.nan, 0.0)
    out, _, _ = D.tree_attention(q, k_new, v_new, par, kc, cache, [1], 1, 1.0)
    assert np.allclose(out[0, 0], (5.0, 10.5)) and np.allclose(out[1, 1], (12 / 3, 24 / 3))
    assert np.allclose(out[2, 0], (14 / 3, 26 / 3))        # values of the cache, node 0, node 2
    q[0, 0] = (2.0, 0.0)
    kc[1, 0, 0] = (1.0, 0.0)
    out, mass, big = D.tree_attention(q, k_new, v_new, par, kc, cache, [1], 1, 0.5)
    assert np.allclose(out[0, 0], (10 * np.e / (np.e + 1), (20 * np.e + 1) / (np.e + 1)))
    assert big[0, 0] == 1.0 and np.allclose(mass[0, 0], out[0, 0])
    out, _, _ = D.tree_attention(q, k_new, v_new, par, kc, cache, [2], 1, 0.5)
    assert np.isnan(out).all()
    out, _, _ = D.tree_attention(q, k_new, v_new, par, kc, cache, [1], 3, 0.5)
    assert np.isnan(out).all()


def test_logits_by_hand():
    z = np.array([[2.0, -2.0, 1.0, 4.0, 0.5]] * 3)
    out = D.process_logits(z, [-1, 0, 1], [3, 1, 1], [0, 2, 2, 9], 1, 2.0, 0.25, 0.5,
                           [(4, 1.0), (4, 3.0), (7, 1.0)], [None, None, np.arange(5) != 3])
    # token 0 in the prompt, 2 generated twice, 4 biased; the path adds token 1 once, then twice
    assert np.array_equal(out[0], [1.0, -2.0, 0.5 - 1.25, 4.0, 3.5])
    assert np.array_equal(out[1], [1.0, -4.0 - 0.75, 0.5 - 1.25, 4.0, 3.5])
    assert np.array_equal(out[2], [1.0, -4.0 - 1.25, 0.5 - 1.25, -np.inf, 3.5])


def test_growth_by_hand():
    table = np.array([[4, -1], [2, 3], [5, -1], [-1, -1]], np.int32)
    free = np.array([0, 1, -1, -1, -1, -1], np.int32)
    slots, seq, t, f, n, st = D.cache_extend(np.array([2, D.RELEASE, -1, 3]),
                                             np.array([15, 17, 9, 0]), table, free, 2, 16, 3)
    # request 1 pushes pages 2 and 3; request 0 pops 3, request 3 pops 2
    assert slots.tolist() == [[4 * 16 + 15, 48, -1], [-1] * 3, [-1] * 3, [32, 33, 34]]
    assert seq.tolist() == [17, 0, 9, 3] and t.tolist() == [[4, 3], [-1, -1], [5, -1], [2, -1]]
    assert n == 2 and f[:4].tolist() == [0, 1, 2, 3] and not st.any()
    _, seq, _, _, n, st = D.cache_extend(np.array([20, 16, 1, 0]), np.array([0, 16, 15, 33]),
                                         table, free, 1, 16, 20)
    assert st.tolist() == [D.FULL, D.FULL, D.OK, D.BAD_LENGTH] and n == 1
    assert seq.tolist() == [0, 16, 16, 33]
    _, _, _, _, _, st = D.cache_extend(np.array([4, 18, 0, 0]), np.array([0, 15, 0, 0]), table,
                                       free, 2, 16, 3)
    assert st.tolist() == [D.OVERFLOW, D.OVERFLOW, D.OK, D.OK]


def test_commit_by_hand():
    k = np.arange(1 * 2 * 3).reshape(1, 2, 3, 1, 1).astype(float)
    cache = np.full((1, 2, 1, 2, 1), -1.0)
    got = D.cache_commit(k, cache, [2, 3], np.array([[3, 0], [1, 9]]), np.array([[2], [5]]))
    assert got.ravel().tolist() == [2.0, 3.0, -1.0, 0.0]
    got = D.cache_commit(k, cache, [2, -1], np.array([[3, 0], [1, 9]]), None)
    assert got.ravel().tolist() == [1.0, -1.0, -1.0, 0.0]
