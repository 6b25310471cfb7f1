"""Pins of oracle/relpos_oracle.py and oracle/muon_oracle.py (CPU): hand-worked
buckets, the gradient against finite differences, and the orthogonalisation
against the singular value decomposition."""
import numpy as np
import pytest

from oracle import muon_oracle as mo
from oracle import relpos_oracle as ro


def test_buckets_by_hand():
    # offsets 0, 2, 5 against 0, 1, clipped at +-1: edges 0, 1
    n = ro.buckets([[0, 2, 5]], [[0, 1]], [0, 1])
    assert n.tolist() == [[[1, 0], [2, 2], [2, 2]]]
    n = ro.buckets([[0, 2]], [[0, 2]], [0, 1], [[7, 8]], [[7, 8]])
    assert n.tolist() == [[[1, 3], [3, 1]]]
    assert ro.buckets([[4]], [[9]], []).tolist() == [[[0]]]


def test_clipped_buckets_match_one_hot_of_clipped_difference():
    rng = np.random.default_rng(0)
    pi, pj = rng.integers(-50, 50, (2, 9)), rng.integers(-50, 50, (2, 13))
    K = 8
    edges = np.arange(1 - K, K + 1)
    want = np.clip(pi[:, :, None] - pj[:, None, :], -K, K) + K
    assert np.array_equal(ro.buckets(pi, pj, edges), want)


def test_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(1)
    pi, pj, edges = rng.integers(0, 20, (2, 6)), rng.integers(0, 20, (2, 5)), np.array([-6, -1, 0, 3])
    si, sj = rng.integers(0, 2, (2, 6)), rng.integers(0, 2, (2, 5))
    t, w = rng.standard_normal((3, 6)), rng.standard_normal((2, 3, 6, 5))
    d = ro.backward(pi, pj, edges, w, si, sj)
    f = lambda t: (ro.forward(pi, pj, edges, t, None, si, sj) * w).sum()
    for h in range(3):
        for n in range(6):
            e = np.zeros_like(t)
            e[h, n] = 0.5  # the form is linear in the table: any step is exact but for rounding
            assert abs((f(t + e) - f(t - e)) - d[h, n]) < 1e-12 * np.abs(w).sum()


@pytest.mark.parametrize("m,n", [(5, 5), (3, 8), (9, 4), (1, 6)])
def test_orthogonalize_maps_the_singular_values(m, n):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((m, n))
    U, s, V = np.linalg.svd(x, full_matrices=False)
    want = (U * mo.singular_map(s / np.linalg.norm(s))) @ V
    assert np.abs(mo.orthogonalize(x) - want).max() < 1e-12
    assert np.abs(mo.orthogonalize(np.stack([x, 3 * x]))[1] - want).max() < 1e-12


def test_orthogonalize_of_zero_and_of_an_orthogonal_matrix():
    assert not mo.orthogonalize(np.zeros((3, 4))).any()
    q = np.linalg.qr(np.random.default_rng(3).standard_normal((6, 6)))[0]
    o = mo.orthogonalize(q)
    k = mo.singular_map(1 / np.sqrt(6))
    assert np.abs(o - k * q).max() < 1e-12 and 0.6 < k < 1.3


def test_muon_step_by_hand():
    # a 1 x 1 matrix: the update is the sign times the map of 1
    k = mo.singular_map(1.0)
    p, m, w = mo.muon_step([[2.0]], [[-0.5]], [[0.0]], [[1.0]], lr=0.1, momentum_decay=0.9, nesterov=True,
                           weight_decay=0.5, swa_decay=0.75, update_scale=2.0)
    assert abs(m[0, 0] + 0.05) < 1e-15
    assert abs(p[0, 0] - (2.0 * 0.95 + 0.2 * k)) < 1e-14
    assert abs(w[0, 0] - (0.75 + 0.25 * p[0, 0])) < 1e-14
