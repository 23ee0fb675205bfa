"""The 64-bit oracle of the operators on rows of logits against closed forms and finite
differences (CPU)."""

import numpy as np
import pytest

from oracle import logits as L

INF = np.inf


def test_uniform_and_two_columns():
    for d in (1, 2, 7, 1000):
        out = L.logprob(np.full((1, d), 3.0), [d - 1], 0.7, 1)
        assert np.isclose(out["logp"][0], -np.log(d), atol=1e-14)
        assert np.isclose(out["entropy"][0], np.log(d), atol=1e-12)
        assert np.isclose(out["lse"][0], 0.7 * 3 + np.log(d), atol=1e-14)
        assert out["top_ids"][0, 0] == 0
    # p = 1 / (1 + e^-x) of two columns x / scale apart
    x = 0.9
    out = L.logprob([[x / 2.0, 0.0]], [0], 2.0, 2)
    p = 1 / (1 + np.exp(-x))
    assert np.isclose(out["logp"][0], np.log(p))
    assert np.isclose(out["entropy"][0], -p * np.log(p) - (1 - p) * np.log(1 - p))
    assert np.allclose(out["top_logp"][0], np.log([p, 1 - p]))


def test_masked_and_empty_rows():
    Z = np.array([[1.0, -INF, 2.0, -INF], [-INF] * 4, [0.0, np.nan, 0.0, 0.0], [0.0, INF, 0.0, 0.0]])
    out = L.logprob(Z, [0, 1, 0, 0], 1.0, 3)
    assert np.isclose(out["logp"][0], -np.log(1 + np.e)) and out["logp"][1] == -INF
    assert out["entropy"][1] == 0 and out["lse"][1] == -INF
    assert np.isnan(out["logp"][2:]).all() and np.isnan(out["entropy"][2:]).all()
    assert out["top_ids"].tolist() == [[2, 0, -1], [-1] * 3, [0, 2, 3], [1, 0, 2]]
    g = L.logprob_grad(Z, [0, 1, 0, 0], 1.0, np.ones(4), None, np.ones(4))
    assert not g[1].any() and g[0, 1] == 0 and np.isnan(g[2:]).all()
    assert not L.logprob_grad(Z, [-1, 4, -1, 9], 1.0, np.ones(4)).any()


def test_alternatives_break_ties_low():
    assert L.alternatives(np.array([1.0, 5, 5, -0.0, 0.0, 5]), 6).tolist() == [1, 2, 5, 0, 3, 4]


@pytest.mark.parametrize("scale", [1.0, 0.4, 1.7])
def test_gradients_are_differences(scale):
    rng = np.random.default_rng(7)
    n, d, k, h = 3, 11, 5, 1e-6
    Z = rng.standard_normal((n, d)) * 2
    Z[0, 4] = -INF
    ids = np.array([2, -1, 10])
    w = rng.standard_normal((3, n))
    tid = np.stack([rng.permutation(d)[:k] for _ in range(n)])
    tid[0] = [1, 1, 3, -1, 1]                     # equal entries, one that is no token
    t = rng.standard_normal((n, k)) * 2
    t_lse = np.log(np.exp(0.8 * t).sum(1) * 1.3)

    def scored(Z):
        o = L.logprob(Z, ids, scale)
        return (w[0] * o["logp"] + w[1] * o["lse"] + w[2] * o["entropy"]).sum()

    def taught(Z, lse):
        return (w[0] * L.distill(Z, tid, t, scale, 0.8, lse)).sum()

    cases = [(scored, L.logprob_grad(Z, ids, scale, *w))]
    cases += [(lambda Z, l=l: taught(Z, l), L.distill_grad(Z, tid, t, w[0], scale, 0.8, l)) for l in (None, t_lse)]
    for f, grad in cases:
        for i in range(n):
            for j in range(d):
                if Z[i, j] == -INF:
                    continue
                up, down = Z.copy(), Z.copy()
                up[i, j] += h
                down[i, j] -= h
                # differences of numbers of size 10 over 2 h: 1e-15 * 10 / 2e-6, and h^2 of the third derivative
                assert abs((f(up) - f(down)) / (2 * h) - grad[i, j]) < 1e-7


def test_teacher():
    log_q, q = L.teacher([3, -1, 0, 9], [1.0, 50.0, 0.0, 50.0], 9, 2.0)
    assert np.allclose(q, [1 / (1 + np.exp(-2)), 0, 1 / (1 + np.exp(2)), 0]) and np.isclose(q.sum(), 1)
    log_q, q = L.teacher([3, 4], [1.0, -INF], 9, 2.0, 2.5)
    assert np.allclose(log_q[0], -0.5) and q[1] == 0
    # a teacher equal to the row has distance 0, any other has more
    z = np.random.default_rng(1).standard_normal((1, 6))
    ids = np.arange(6)[None]
    assert abs(L.distill(z, ids, z)[0]) < 1e-14 and L.distill(z, ids, 2 * z)[0] > 1e-3
    assert np.abs(L.distill_grad(z, ids, z, [1.0])).max() < 1e-14
    assert L.distill(z, [[-1] * 6], z)[0] == 0 and L.distill(np.full((1, 3), -INF), [[0]], [[0.0]])[0] == INF
