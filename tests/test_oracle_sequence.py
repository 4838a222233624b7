"""The fp64 definitions of the sequence operators: hand-made cases, and their gradients against differences."""
import numpy as np
import pytest

from oracle import mrf_sequence_oracle as so


def _differences(f, x, g, step=1e-5):
    """d sum(g f(x)) / dx by central differences."""
    out = np.zeros_like(x)
    for n in np.ndindex(*x.shape):
        keep = x[n]
        x[n] = keep + step
        up = (g * f(x)).sum()
        x[n] = keep - step
        out[n] = (up - (g * f(x)).sum()) / (2 * step)
        x[n] = keep
    return out


def test_attention_of_one_key_returns_its_value_and_of_none_nothing():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 2, 4)), rng.normal(size=(1, 1, 4)), rng.normal(size=(1, 1, 4))
    ok = np.array([[True], [False], [True]])
    out, lse, p = so.attention(q, k, v, 0.5, ok)
    np.testing.assert_allclose(out[0], np.repeat(v[0], 2, 0))
    assert (out[1] == 0).all() and (lse[:, 1] == -np.inf).all() and (p[:, 1] == 0).all()
    np.testing.assert_allclose(lse[:, 2], 0.5 * (q[2] * k[0]).sum(1))


def test_attention_bands_and_lengths():
    ok, d = so.attention_pairs(3, 5, first=-1, last=0, offset=2)
    assert ok.astype(int).tolist() == [[0, 1, 1, 0, 0], [0, 0, 1, 1, 0], [0, 0, 0, 1, 1]] and d[0].tolist() == [-2, -1, 0, 1, 2]
    ok, _ = so.attention_pairs(3, 5, last=0, offset=2, q_length=2, k_length=3)
    assert ok.astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 0, 0], [0, 0, 0, 0, 0]]


@pytest.mark.parametrize("band", [(None, None), (None, 0), (-2, 1)])
def test_attention_gradients_by_differences(band):
    rng = np.random.default_rng(1)
    Q, K, Hq, Hk, D = 4, 5, 4, 2, 3
    q, k, v, g = rng.normal(size=(Q, Hq, D)), rng.normal(size=(K, Hk, D)), rng.normal(size=(K, Hk, D)), rng.normal(size=(Q, Hq, D))
    ok, d = so.attention_pairs(Q, K, *band, offset=-1, k_length=4)
    table, bucket_of = rng.normal(size=(Hq, 3)), np.array([2, 0, 1, 1, 0], np.int32)
    bias = lambda t: so.attention_bias(d, t, bucket_of, -2)[0]  # noqa: E731
    gq, gk, gv, ds, _ = so.attention_grad(g, q, k, v, 0.7, ok, bias(table))
    out = lambda: so.attention(q, k, v, 0.7, ok, bias(table))[0]  # noqa: E731
    np.testing.assert_allclose(gq, _differences(lambda _: out(), q, g), atol=1e-8)
    np.testing.assert_allclose(gk, _differences(lambda _: out(), k, g), atol=1e-8)
    np.testing.assert_allclose(gv, _differences(lambda _: out(), v, g), atol=1e-8)
    which = so.attention_bias(d, table, bucket_of, -2)[1]
    np.testing.assert_allclose(so.table_grad(ds, which, 3), _differences(lambda _: out(), table, g), atol=1e-8)


def test_rotation_turns_pairs_and_leaves_the_rest():
    x = np.array([[[3.0, 0.0, 4.0, 1.0, 2.0]]])
    n = np.sqrt(30 / 5)
    y = so.head_rotation(x, np.ones(5), 1e-30, [np.pi / 2], positions=np.array([[1]]))
    np.testing.assert_allclose(y[0, 0] * n, [0.0, 3.0, 4.0, 1.0, 2.0], atol=1e-12)
    y = so.head_rotation(x, np.ones(5), 1e-30, [np.pi, np.pi / 2], positions=np.array([[1, 3]]))      # by two axes: pairs (0, 2), (1, 3)
    np.testing.assert_allclose(y[0, 0] * n, [-3.0, 1.0, -4.0, 0.0, 2.0], atol=1e-12)
    y = so.head_rotation(x, np.ones(5), 1e-30, [np.pi / 2, 0.0], offset=1, interleaved=True)
    np.testing.assert_allclose(y[0, 0] * n, [0.0, 3.0, 4.0, 1.0, 2.0], atol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_gradients_by_differences(interleaved):
    rng = np.random.default_rng(2)
    x, gamma, g = rng.normal(size=(3, 2, 6)), rng.normal(1.0, 0.3, 6), rng.normal(size=(3, 2, 6))
    at = rng.integers(0, 9, (3, 2))
    f = lambda: so.head_rotation(x, gamma, 1e-2, [0.7, 0.2], at, 1, interleaved)  # noqa: E731
    gx, gg = so.head_rotation_grad(g, x, gamma, 1e-2, [0.7, 0.2], at, 1, interleaved)
    np.testing.assert_allclose(gx, _differences(lambda _: f(), x, g), atol=1e-8)
    np.testing.assert_allclose(gg, _differences(lambda _: f(), gamma, g), atol=1e-8)


def test_recurrence_by_hand():
    z = np.log(np.array([[3.0], [1.0], [1.0 / 3.0]]))      # gates 3/4, 1/2, 1/4
    x = np.array([[4.0], [8.0], [16.0]])
    y, h = so.gated_scan(x, z, initial=[8.0])
    np.testing.assert_allclose(y[:, 0], [7.0, 7.5, 13.875])
    y, h = so.gated_scan(x, z, complement=False, reverse=True, length=2)
    np.testing.assert_allclose(y[:, 0], [10.0, 8.0, 0.0])
    np.testing.assert_allclose(h, [10.0])
    y, h = so.gated_scan(x, z, initial=[5.0], length=0)
    assert (y == 0).all() and h[0] == 5.0


@pytest.mark.parametrize("complement,reverse,length", [(True, False, None), (False, False, 3), (True, True, 4), (False, True, None)])
def test_recurrence_gradients_by_differences(complement, reverse, length):
    rng = np.random.default_rng(3)
    x, z, h0, g, gf = rng.normal(size=(5, 2)), rng.normal(size=(5, 2)), rng.normal(size=2), rng.normal(size=(5, 2)), rng.normal(size=2)
    if length is not None:
        g[length:] = 0.0

    def f(_):
        y, h = so.gated_scan(x, z, h0, complement, reverse, length)
        return np.concatenate([y, h[None]])
    both = np.concatenate([g, gf[None]])
    gx, gz, gi = so.gated_scan_grad(g, x, z, h0, gf, complement, reverse, length)
    np.testing.assert_allclose(gx, _differences(f, x, both), atol=1e-8)
    np.testing.assert_allclose(gz, _differences(f, z, both), atol=1e-8)
    np.testing.assert_allclose(gi, _differences(f, h0, both), atol=1e-8)
