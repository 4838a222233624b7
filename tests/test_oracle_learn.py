"""Pins of the fp64 definitions of the learning operators (CPU): closed forms, enumeration, finite differences; and what the
library computes on the host."""
import numpy as np
import pytest

import paper_1910_10892_amd as mrf
from oracle import mrf_learn_oracle as lo


def _differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


def test_layer_norm_has_mean_and_variance_of_the_parameters():
    rng = np.random.default_rng(1)
    x = rng.normal(3.0, 2.0, (5, 9))
    y, mu, rstd = lo.layer_norm(x, np.full(9, 1.5), np.full(9, 0.25), eps=1e-12)
    np.testing.assert_allclose(y.mean(1), 0.25, atol=1e-12)
    np.testing.assert_allclose(y.std(1), 1.5, rtol=1e-9)
    np.testing.assert_allclose(mu, x.mean(1))
    # two values: +-1 whatever they are
    np.testing.assert_allclose(lo.layer_norm(np.array([[3.0, 7.0]]), eps=1e-12)[0], [[-1.0, 1.0]], rtol=1e-9)
    # one value, or equal ones: 0
    assert (lo.layer_norm(np.full((2, 1), 5.0))[0] == 0).all() and (lo.layer_norm(np.full((2, 4), 5.0))[0] == 0).all()


@pytest.mark.parametrize("N,C", [(1, 1), (3, 2), (4, 7)])
def test_layer_norm_gradients_are_differences(N, C):
    rng = np.random.default_rng(2)
    x, gamma, beta, w = rng.normal(size=(N, C)), rng.normal(1, 0.3, C), rng.normal(size=C), rng.normal(size=(N, C))
    gx, gg, gb = lo.layer_norm_grad(w, x, gamma, eps=1e-3)
    f = lambda x, g, b: float((lo.layer_norm(x, g, b, eps=1e-3)[0] * w).sum())
    np.testing.assert_allclose(gx, _differences(lambda v: f(v, gamma, beta), x), atol=2e-7)
    np.testing.assert_allclose(gg, _differences(lambda v: f(x, v, beta), gamma), atol=2e-7)
    np.testing.assert_allclose(gb, _differences(lambda v: f(x, gamma, v), beta), atol=2e-7)


@pytest.mark.parametrize("NB,far,two_sided", [(32, 128, True), (32, 128, False), (16, 16, True), (2, 5, True), (1, 4, True), (3, 9, True),
                                              (7, 40, False), (64, 1000, True), (8, 3, True), (65536, 128, True)])
def test_distance_buckets_are_those_of_the_integer_rule(NB, far, two_sided):
    # (with many buckets the integers of the rule get long: a few offsets do)
    offsets = [-1 << 40, -70000, -40000] if NB > 1000 else list(range(-1100, 1100, 1 if far < 200 else 7))
    for d in offsets:
        got = int(mrf.mrf_distance_buckets(NB, far, d, 1, two_sided)[0])
        want = lo.distance_bucket(d, NB, far, two_sided) if NB <= 1000 else NB // 2 - 1
        assert got == want, d
    got = mrf.mrf_distance_buckets(NB, far, -50, 101, two_sided)
    assert got.dtype == np.int32 and got.min() >= 0 and got.max() < NB
    assert [int(mrf.mrf_distance_buckets(NB, far, d, 1, two_sided)[0]) for d in range(-50, 51)] == got.tolist()


def test_distance_buckets_small_distances_have_their_own():
    assert mrf.mrf_distance_buckets(32, 128, -7, 15).tolist() == [7, 6, 5, 4, 3, 2, 1, 0, 17, 18, 19, 20, 21, 22, 23]
    assert mrf.mrf_distance_buckets(32, 128, -1000, 1)[0] == 15 and mrf.mrf_distance_buckets(32, 128, 1000, 1)[0] == 31


def test_bucket_pairwise_by_hand():
    # offsets -2..3 in buckets 0 0 1 2 2 3
    m = np.array([0, 0, 1, 2, 2, 3])
    out = lo.bucket_pairwise(np.array([[10.0, 11.0, 12.0, 13.0]]), 3, 3, m, -2)
    np.testing.assert_array_equal(out[0], [[11, 12, 12], [10, 11, 12], [10, 10, 11]])
    # the last row alone, as a row of a longer matrix
    np.testing.assert_array_equal(lo.bucket_pairwise(np.array([[10.0, 11.0, 12.0, 13.0]]), 1, 3, m, -2, query_offset=2)[0], out[0, 2:])
    g, size = lo.bucket_pairwise_grad(np.arange(9.0).reshape(1, 3, 3), 4, m, -2)
    np.testing.assert_array_equal(g[0], [3 + 6 + 7, 0 + 4 + 8, 1 + 2 + 5, 0])
    np.testing.assert_array_equal(size, g)


def test_bucket_gradient_is_the_transposed_map():
    rng = np.random.default_rng(3)
    m = rng.integers(0, 5, 12)
    t, w = rng.normal(size=(2, 5)), rng.normal(size=(2, 4, 9))
    g, _ = lo.bucket_pairwise_grad(w, 5, m, -3)
    assert float((lo.bucket_pairwise(t, 4, 9, m, -3) * w).sum()) == pytest.approx(float((t * g).sum()), rel=1e-12)


def test_softmin_logp_closed_forms():
    c = np.array([[0.0, 0.0], [1.0, 3.0], [np.inf, 2.0], [np.inf, np.inf]])
    np.testing.assert_allclose(lo.softmin_logp(c, np.array([0, 0, 1, 1])), [-np.log(2), -np.log1p(np.exp(-2)), 0.0, -np.inf])
    assert lo.softmin_logp(c, np.array([0, 0, 0, 0]))[2] == -np.inf
    # labels outside the range are clamped
    assert lo.softmin_logp(c[1:2], np.array([9]))[0] == lo.softmin_logp(c[1:2], np.array([1]))[0]


@pytest.mark.parametrize("kl,with_old", [(0.0, True), (0.3, True), (0.3, False)])
def test_policy_gradient_is_that_of_the_loss_by_differences(kl, with_old):
    rng = np.random.default_rng(4)
    N, L = 7, 5
    c, a, A = rng.normal(size=(N, L)), rng.integers(0, L, N), rng.normal(size=4) + 0.3
    lp = lo.softmin_logp(c, a)
    # ratios on both sides of both bounds, none within 0.02 of one
    old = lp - np.log(np.array([0.5, 0.78, 0.83, 1.0, 1.17, 1.23, 2.0]))
    ref = lp + rng.normal(0, 0.4, N)
    mask = np.array([1, 1, 0, 1, 1, 1, 1])
    loss, _, grad = lo.policy(c, a, A, old if with_old else None, ref if kl else None, mask, 0.2, 0.2, kl, per=2)

    def f(v):
        # (without old log-probabilities those of the present costs stand in for them, held fixed)
        return lo.policy(v, a, A, old if with_old else lp, ref if kl else None, mask, 0.2, 0.2, kl, per=2)[0][0]

    np.testing.assert_allclose(grad, _differences(f, c), atol=1e-8)
    assert (grad[2] == 0).all()
    np.testing.assert_allclose(grad.sum(1), 0.0, atol=1e-15)      # probabilities sum to one


def test_policy_limits():
    c, a = np.zeros((2, 4)), np.array([1, 2])
    lp = np.full(2, -np.log(4.0))
    # at the old costs: the loss is minus the mean advantage, no divergence from an equal reference
    loss, logp, grad = lo.policy(c, a, np.array([1.0, 3.0]), lp, lp, None, 0.2, 0.2, 0.5)
    np.testing.assert_allclose(loss, [-2.0, -2.0, 0.0])
    np.testing.assert_allclose(grad[0], [-0.125, 0.375, -0.125, -0.125])
    # ratio far above the bound: the loss is held there and the gradient is 0 for A > 0, but not for A < 0
    loss, _, grad = lo.policy(c, a, np.array([1.0, -1.0]), lp - 1.0, None, None, 0.2, 0.2)
    np.testing.assert_allclose(loss[0], -(1.2 - np.e) / 2)
    assert (grad[0] == 0).all() and grad[1, 2] < 0
    # nothing counts
    loss, logp, grad = lo.policy(c, a, np.ones(2), lp, None, np.zeros(2))
    assert (loss == 0).all() and (logp == 0).all() and (grad == 0).all()


def test_distance_buckets_that_no_offset_has():
    """Two-sided: the upper half's distance 0, where a half has more than one bucket, and the middle bucket of an odd number."""
    for NB, empty in ((8, {4}), (9, {4, 5}), (32, {16}), (33, {16, 17}), (4, {2}), (3, {1}), (2, set()), (1, set())):
        got = set(mrf.mrf_distance_buckets(NB, 200, -5000, 10001).tolist())
        assert got == set(range(NB)) - empty, (NB, sorted(got))
    # one-sided: every bucket has a distance
    for NB in (1, 2, 9):
        assert set(mrf.mrf_distance_buckets(NB, 15, -15, 16, two_sided=False).tolist()) == set(range(NB))
