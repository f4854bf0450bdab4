"""Pins of the plain 64-bit forms of prompt attention and of the cache of 4 bits in
oracle/decoding.py: hand values and identities that do not go through their own formulas
(no GPU)."""

import numpy as np
import pytest

from oracle import decoding as D


def test_prompt_by_hand():
    """Equal scores average the visible values; a weight of e against 1; two heads read one key
    head; earlier keys are seen by all queries, and more queries than keys leave rows of zeros."""
    q, k = np.zeros((2, 2, 2)), np.zeros((3, 1, 2))
    v = np.array([[[1.0, 2.0]], [[3.0, 6.0]], [[8.0, 1.0]]])
    out, mass, big = D.prompt_attention(q, k, v, 1.0)
    assert np.allclose(out[0], [(2.0, 4.0)] * 2) and np.allclose(out[1], [(4.0, 3.0)] * 2)
    assert np.allclose(mass, out) and not big.any()
    q[0, 1] = (2.0, 0.0)
    k[1, 0] = (1.0, -3.0)
    out, _, big = D.prompt_attention(q, k, v, 0.5)
    assert np.allclose(out[0, 1], ((1 + 3 * np.e) / (1 + np.e), (2 + 6 * np.e) / (1 + np.e)))
    assert np.allclose(out[0, 0], (2.0, 4.0)) and big[0, 1] == 1.0
    out, _, _ = D.prompt_attention(np.ones((3, 2, 2)), k[:1], v[:1], 1.0)
    assert not out[:2].any() and np.allclose(out[2], [(1.0, 2.0)] * 2)


def test_prompt_is_a_tree_that_is_a_chain():
    rng = np.random.default_rng(0)
    q, kn, vn = rng.normal(size=(5, 4, 8)), rng.normal(size=(5, 2, 8)), rng.normal(size=(5, 2, 8))
    kc, vc = rng.normal(size=(3, 2, 4, 8)), rng.normal(size=(3, 2, 4, 8))
    old = [D.cached(c, [2, 0], 7) for c in (kc, vc)]
    want, _, _ = D.tree_attention(q, kn, vn, [-1, 0, 1, 2, 3], kc, vc, [2, 0], 7, 0.3)
    got, _, _ = D.prompt_attention(q, np.concatenate([old[0], kn]), np.concatenate([old[1], vn]), 0.3)
    assert np.allclose(got, want, atol=1e-14)


def test_fp4_values_are_those_of_their_bits():
    """Sign, two bits of exponent with bias 1, one of the significand."""
    for c in range(16):
        e, m = c >> 1 & 3, c & 1
        want = (1 + m / 2) * 2.0 ** (e - 1) if e else m / 2
        assert D.fp4_values([c], 130)[0] == (-1) ** (c >> 3) * want * 8
    assert np.isnan(D.fp4_values([0, 7], 255)).all()


def test_fp4_encode_by_hand():
    pad = [0.0] * 24
    x = [6.0, 0.25, 0.75, 1.25, 1.75, -2.5, -3.5, 5.0]           # ties
    codes, e = D.fp4_encode(x + pad)
    assert e == 127 and codes[:8] == [7, 0, 2, 2, 4, 8 + 4, 8 + 6, 6] and codes[8:] == [0] * 24
    codes, e = D.fp4_encode([7.0, -0.0, 0.26, -0.2] + [0.0] * 28)
    assert e == 127 and codes[:4] == [7, 8, 1, 8]
    codes, e = D.fp4_encode([np.nextafter(7.0, 8.0)] + [0.0] * 31)
    assert e == 128 and codes[0] == 6                              # 3.5 of two: to 4
    assert D.fp4_encode([0.0] * 32) == ([0] * 32, 1)
    assert D.fp4_encode([2.0 ** -133] + [0.0] * 31)[1] == 1
    assert D.fp4_encode([1.0, np.inf] + [0.0] * 30) == ([0] * 32, 255)
    assert D.fp4_encode([np.nan] + [0.0] * 31) == ([0] * 32, 255)
    codes, e = D.fp4_encode([65504.0] + [0.0] * 31, 140)
    assert (codes[0], e) == (7, 140) and D.fp4_encode([65504.0] + [0.0] * 31)[1] == 141


def test_fp4_encode_is_the_nearest():
    """No value of the exponent's grid is nearer, none of the exponents below holds the largest."""
    rng = np.random.default_rng(1)
    for _ in range(50):
        x = rng.normal(size=32) * 2.0 ** rng.integers(-20, 20)
        codes, e = D.fp4_encode(x)
        got = D.fp4_values(codes, e)
        grid = np.array([s * t for s in (1, -1) for t in D.FP4_VALUES]) * 2.0 ** (e - 127)
        assert np.allclose(np.abs(got - x), np.abs(grid[None] - x[:, None]).min(1), atol=0)
        assert np.abs(x).max() <= 7 * 2.0 ** (e - 127) and np.abs(x).max() > 7 * 2.0 ** (e - 128)


@pytest.mark.parametrize("ps,dim", [(4, 32), (2, 64), (3, 96)])
def test_fp4_rows_written_are_read_back(ps, dim):
    """Numbers of the grid come back as they are, and no other row of the page changes."""
    rng = np.random.default_rng(2)
    page = rng.integers(0, 256, ps * dim // 32 * 17).astype(np.uint8)
    page[ps * dim // 2:] = 127
    before = [D.fp4_row(page, ps, dim, r) for r in range(ps)]
    x = np.concatenate([np.append(6.0, rng.choice(D.FP4_VALUES, 31)) * s * 2.0 ** k
                        for s, k in zip((1, -1, 1, -1), rng.integers(-9, 9, dim // 32))])
    D.fp4_put(page, ps, dim, ps - 2, x)
    for r in range(ps):
        assert np.array_equal(D.fp4_row(page, ps, dim, r), x if r == ps - 2 else before[r])


def test_commit_and_read_by_hand():
    cache = np.zeros((1, 3, 1, 2 * 17), np.uint8)
    k_new = np.zeros((1, 1, 3, 1, 32))
    k_new[0, 0, 0], k_new[0, 0, 2, 0, 1] = 3.0, -12.0
    got = D.cache_commit_fp4(k_new, cache, 2, [2], np.array([[4, 1, 0]]), np.array([[2, 1]]))
    # node 0 to page 2, row 0; node 2 to page 0, row 1
    assert got[0, 2, 0, :16].tolist() == [0x77] * 16 and got[0, 2, 0, 32] == 126
    assert got[0, 0, 0, 16:32].tolist() == [0xf0] + [0] * 15 and got[0, 0, 0, 33] == 128
    assert not got[0, 1].any()
    out = D.cache_read_fp4(got, 2, 32, np.array([[2, 0, 9]]), [0], [6], [1], np.full((1, 6, 1, 32), 5.0))
    assert (out[0, 0] == 5.0).all() and (out[0, 1] == 3.0).all() and not out[0, 2].any()
    assert out[0, 4, 0, 1] == -12.0 and np.isnan(out[0, 5]).all()
