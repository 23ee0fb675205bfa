"""The 64-bit oracle of the row operators against published known answers, closed forms,
the oracle of the compressed products, and finite differences (CPU)."""

import numpy as np
import pytest

import oracle as O
from oracle import rows as R


def test_generator_known_answers():
    # the known-answer vectors published with the generator
    ones = 0xFFFFFFFF
    assert R.philox4x32((0, 0, 0, 0), (0, 0)) == (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)
    assert R.philox4x32((ones,) * 4, (ones,) * 2) == (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)
    assert R.philox4x32((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) \
        == (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)


def test_mask_shares_and_ends():
    n, d = 64, 200
    for p in (0.1, 0.5, 0.9):
        k = R.kept(n, d, (p, 5, 6))
        # a share of n d independent draws: within five standard deviations
        assert abs(k.mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / (n * d))
    assert R.kept(3, 9, (0.0, 1, 2)).all() and not R.kept(3, 9, (1.0, 1, 2)).any()
    X = np.ones((5, 11))
    assert np.array_equal(R.dropout(X, (0.0, 1, 2)), X)
    assert np.array_equal(R.dropout(X, (1.0, 1, 2)), 0 * X)
    assert set(np.unique(R.dropout(X, (0.5, 1, 2)))) == {0.0, 2.0}
    a, b, c = (R.kept(8, 64, m) for m in ((0.5, 1, 2), (0.5, 1, 3), (0.5, 2, 2)))
    assert (a != b).any() and (a != c).any()
    # a wider matrix has the same mask in its first columns
    assert np.array_equal(R.kept(8, 64, (0.5, 1, 2))[:, :13], R.kept(8, 13, (0.5, 1, 2)))


def test_embed_is_the_product_of_one_pair_tuples():
    rng = np.random.default_rng(1)
    ids, V, d, scale = rng.integers(0, 9, 40), 9, 5, 0.5
    tuples = [[(int(v), O.f32_bits(scale))] for v in ids]
    E, G = rng.standard_normal((V, d)), rng.standard_normal((40, d))
    assert np.allclose(R.embed(ids, E, scale), O.dense_right(tuples, V, E)[0], rtol=0, atol=1e-14)
    dE, S, count = R.embed_grad(ids, G, V, scale)
    want, scale_of = O.dense_left(tuples, V, G)
    assert np.allclose(dE, want, rtol=0, atol=1e-13) and np.allclose(S, scale_of, rtol=0, atol=1e-13)
    assert np.array_equal(count, np.bincount(ids, minlength=V))


def test_embed_outside_and_duality():
    rng = np.random.default_rng(2)
    ids = np.array([-1, 0, 7, 6, 3, 3, 2 ** 40, -2 ** 40])
    E, G = rng.standard_normal((7, 19)), rng.standard_normal((8, 19))
    drop = (0.3, 11, 12)
    out = R.embed(ids, E, 1.5, drop)
    assert not out[[0, 2, 6, 7]].any() and out[1].any()
    dE = R.embed_grad(ids, G, 7, 1.5, drop)[0]
    assert np.isclose(np.sum(out * G), np.sum(dE * E), rtol=1e-12)
    assert not dE[[1, 2, 4, 5]].any()


def test_norm_closed_forms():
    h, y = R.rmsnorm(np.array([[3.0, 4.0]]), eps=1e-30)
    assert np.allclose(y, np.array([[3.0, 4.0]]) / np.sqrt(12.5))
    h, y = R.rmsnorm(np.ones((2, 8)), R=np.ones((2, 8)), w=np.arange(8.0), eps=1e-30)
    assert np.array_equal(h, 2 * np.ones((2, 8))) and np.allclose(y, np.arange(8.0)[None, :])
    h, y = R.rmsnorm(np.zeros((1, 5)))
    assert not y.any()


@pytest.mark.parametrize("drop", [None, (0.4, 3, 9)])
@pytest.mark.parametrize("d", [1, 2, 9])
def test_norm_gradients_by_differences(d, drop):
    """Central differences of loss = <y, dY> + <h, dR> in X, R and w."""
    rng = np.random.default_rng(d)
    n = 4
    X, Rs, dY, dR = (rng.standard_normal((n, d)) for _ in range(4))
    w = rng.standard_normal(d)

    def loss(X, Rs, w):
        h, y = R.rmsnorm(X, Rs, w, 1e-3, drop)
        return np.sum(y * dY) + np.sum(h * dR)

    h = R.rmsnorm(X, Rs, w, 1e-3, drop)[0]
    dH, dX, dw = R.rmsnorm_grad(h, dY, w, 1e-3, dR, drop)
    e = 1e-6
    for name, at, grad in (("X", X, dX), ("R", Rs, dH), ("w", w, dw)):
        for i in np.ndindex(at.shape):
            lo, hi = at.copy(), at.copy()
            lo[i] -= e
            hi[i] += e
            args = {"X": (X, Rs, w), "R": (X, Rs, w), "w": (X, Rs, w)}[name]
            k = "XRw".index(name)
            diff = (loss(*[hi if j == k else a for j, a in enumerate(args)])
                    - loss(*[lo if j == k else a for j, a in enumerate(args)])) / (2 * e)
            # rounding of the two losses (1e-16 of a few tens, over 2e) and the third
            # derivative's e^2 (up to eps^-1.5 = 3e4 where a row is nearly zero)
            assert abs(diff - grad[i]) < 1e-7 * (1 + abs(grad[i])), (name, i)


def test_e4m3_numbers():
    v = R.e4m3_values()
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and np.sum(np.isnan(v)) == 2
    assert v[0x7E] == 448.0 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0] == 0.0
    assert np.all(np.diff(v[:0x7F]) > 0) and np.array_equal(v[0x80:0xFF], -v[:0x7F])
    for b in range(1, 0x7E):
        gap = min(v[b + 1] - v[b], v[b] - v[b - 1])
        assert R.e4m3_half_step(v[b]) >= gap / 2
