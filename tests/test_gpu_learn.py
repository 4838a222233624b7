"""GPU parity of the learning operators (layer norm, bucketed pairwise function, policy loss) with their fp64 definitions, through
the C ABI.

Tolerances follow from the arithmetic, with u = 2^-24: a sum of terms t in single precision, whatever tree or chains form it, is
taken to be off by at most SUM u sum |t|.  Roundings are independent, so a chain of m of them is off by about sqrt(m) u sum |t|, and
no layout has chains of more than 1,024; SUM = 32.  A value stored in 16 bits is off by half a unit in its last place more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U, SUM = 2.0 ** -24, 32.0
HALF_ULP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}
PAD = 1024      # elements in front of and behind a buffer


def _torch():
    import torch
    return torch


def _guarded(shape, dtype, shift=0):
    """A buffer of that shape inside a larger one, `shift` elements behind its start's alignment; returns it and a check that nothing around
    it was written."""
    torch = _torch()
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * PAD + shift,), 77, dtype=dtype, device="cuda:0")
    inner = whole[PAD + shift:PAD + shift + n]
    if dtype.is_floating_point:
        inner.fill_(float("nan"))

    def check():
        around = torch.cat([whole[:PAD + shift], whole[PAD + shift + n:]])
        assert (around == 77).all(), "written outside of the buffer"
    return inner.view(shape), check


def _put(a, dtype, shift=0):
    torch = _torch()
    t, _ = _guarded(np.shape(a), getattr(torch, dtype), shift)
    return t.copy_(torch.from_numpy(np.ascontiguousarray(a)))


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, bound, dtype="float32"):
    """|got - want| <= bound (in 32 bits) and the rounding of the stored type."""
    got = _np(got)
    assert np.isfinite(got).all()
    off = np.abs(got - want)
    limit = bound + (np.abs(want) + bound) * HALF_ULP[dtype] * 1.01 + TINY[dtype]
    worst = np.unravel_index(np.argmax(off - limit), off.shape) if off.size else ()
    assert (off <= limit).all(), "off by %g at %s, allowed %g" % (off[worst], worst, limit[worst])


# ---- layer norm

NORM_SHAPES = [(1, 1), (3, 1), (7, 2), (5, 3), (64, 8), (1536, 16), (1, 21), (2, 21), (1001, 21), (300, 24), (37, 31), (50, 32), (9, 33), (66, 48),
               (40, 63), (33, 64), (90, 65), (411, 70), (129, 96), (17, 100), (31, 127), (65, 128), (20, 129), (70, 192), (33, 200), (18, 255), (64, 256),
               (9, 257), (21, 300), (11, 511), (16, 512), (7, 513), (13, 768), (10, 1000), (19, 1024), (5, 1025), (6, 2048), (5, 2050), (3, 4096),
               (4, 5001), (2, 8192), (3, 8193), (2, 12289), (1, 20000), (2, 40004)]
TYPE_PAIRS = [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float16"), ("bfloat16", "float32"), ("float16", "float32")]


def _norm_bounds(x, rstd, gamma):
    """Bound of the error of h = (x - mu) s in units of u: mu's and that of the difference, over the standard deviation, and s's."""
    h = (x - x.mean(1, keepdims=True)) * rstd[:, None]
    size = np.abs(x).mean(1, keepdims=True) * rstd[:, None]
    return h, SUM * U * (size + 2 * np.abs(h)) + U * np.abs(x) * rstd[:, None]


def _check_norm(N, C, x_type, y_type, shift=0, affine=True, level=1.0):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    print("case layer norm", N, C, x_type, y_type, shift, affine, flush=True)
    rng = np.random.default_rng(1000 * N + C)
    x = _put(rng.normal(level, 2.0, (N, C)), x_type, shift)
    dy = _put(rng.normal(0.0, 1.0, (N, C)), y_type, shift)
    gamma = _put(rng.normal(1.0, 0.3, C), "float32", shift) if affine else None
    beta = _put(rng.normal(0.0, 0.5, C), "float32", shift) if affine else None
    y, y_check = _guarded((N, C), getattr(torch, y_type), shift)
    gx, gx_check = _guarded((N, C), x.dtype, shift)
    stats = [_guarded((N,), torch.float32) for _ in range(2)]
    gg, gb = _guarded((C,), torch.float32, shift), _guarded((C,), torch.float32, shift)
    ws, ws_check = _guarded((mrf.mrf_layer_norm_workspace_bytes(N, C),), torch.uint8)
    mrf.mrf_layer_norm_forward(x, gamma, beta, 1e-5, y, stats[0][0], stats[1][0])
    mrf.mrf_layer_norm_backward(dy, x, gamma, stats[0][0], stats[1][0], gx, gg[0], gb[0], ws)
    torch.cuda.synchronize()
    for check in (y_check, gx_check, ws_check, stats[0][1], stats[1][1], gg[1], gb[1]):
        check()
    xd, dyd = _np(x), _np(dy)
    g = _np(gamma) if affine else np.ones(C)
    b = _np(beta) if affine else np.zeros(C)
    want, mu, rstd = lo.layer_norm(xd, g, b)
    h, dh = _norm_bounds(xd, rstd, g)
    _close(y, want, np.abs(g) * dh + U * (2 * np.abs(g * h) + np.abs(b)), y_type)
    _close(stats[0][0], mu, SUM * U * np.abs(xd).mean(1))
    _close(stats[1][0], rstd, SUM * U * rstd)
    wx, wg, wb = lo.layer_norm_grad(dyd, xd, g)
    a = dyd * g
    ma, mah = np.abs(a).mean(1, keepdims=True), np.abs(a * h).mean(1, keepdims=True)
    bound = rstd[:, None] * (U * np.abs(a) + SUM * U * ma + np.abs(h) * SUM * U * mah + dh * np.abs((a * h).mean(1, keepdims=True)) +
                             np.abs(h) * (np.abs(a) * dh).mean(1, keepdims=True) + 4 * U * (np.abs(a) + ma + np.abs(h) * mah))
    _close(gx, wx, bound + SUM * U * np.abs(wx), x_type)
    _close(gg[0], wg, (np.abs(dyd) * dh).sum(0) + SUM * U * np.abs(dyd * h).sum(0))
    _close(gb[0], wb, SUM * U * np.abs(dyd).sum(0))


@pytest.mark.parametrize("types", TYPE_PAIRS, ids="-".join)
@pytest.mark.parametrize("N,C", NORM_SHAPES)
def test_layer_norm_matches_definition(N, C, types):
    _check_norm(N, C, *types)


@pytest.mark.parametrize("types", TYPE_PAIRS, ids="-".join)
@pytest.mark.parametrize("N,C,shift", [(33, 16, 1), (70, 96, 2), (20, 256, 3), (9, 2048, 1), (5, 4096, 4), (1000, 21, 5)])
def test_layer_norm_at_odd_addresses(N, C, shift, types):
    _check_norm(N, C, *types, shift=shift)


@pytest.mark.parametrize("types", TYPE_PAIRS, ids="-".join)
@pytest.mark.parametrize("C", [12, 20, 28, 36, 40, 44, 48, 52, 60, 68])
def test_layer_norm_of_whole_chunks_that_leave_lanes_idle(C, types):
    _check_norm(203, C, *types)
    _check_norm(1, C, *types, shift=1)


@pytest.mark.parametrize("N,C", [(40000, 21), (70001, 16), (9000, 192), (20003, 70), (3001, 1024), (1100, 2048)])
def test_layer_norm_of_many_rows(N, C):
    """More rows than a launch has room for at once."""
    _check_norm(N, C, "float32", "float32")
    _check_norm(N, C, "bfloat16", "float32", affine=False)


def test_layer_norm_of_a_large_mean_keeps_the_variance():
    """Mean 300 standard deviations away: the second pass over the row takes differences."""
    _check_norm(33, 96, "float32", "float32", level=600.0)
    _check_norm(5, 2048, "float32", "float32", level=600.0)
    _check_norm(3, 20000, "float32", "float32", level=600.0)


@pytest.mark.parametrize("C", [16, 21, 300, 2048, 9001])
def test_layer_norm_outputs_that_are_left_out_and_rows_that_are_not_finite(C):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    N = 37
    rng = np.random.default_rng(C)
    x, dy, gamma, beta = (_put(rng.normal(size=s), "float32") for s in ((N, C), (N, C), (C,), (C,)))
    full = [torch.empty_like(x), torch.empty(N, device="cuda:0"), torch.empty(N, device="cuda:0"), torch.empty_like(x),
            torch.empty_like(gamma), torch.empty_like(beta)]
    ws = torch.empty(mrf.mrf_layer_norm_workspace_bytes(N, C), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_layer_norm_forward(x, gamma, beta, 1e-5, *full[:3])
    mrf.mrf_layer_norm_backward(dy, x, gamma, full[1], full[2], *full[3:], ws)
    y, gx, gg, gb = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    mrf.mrf_layer_norm_forward(x, gamma, beta, 1e-5, y, None, None)
    assert torch.equal(y, full[0])
    mrf.mrf_layer_norm_backward(dy, x, gamma, full[1], full[2], gx, None, None, None)
    assert torch.equal(gx, full[3])
    mrf.mrf_layer_norm_backward(dy, x, gamma, full[1], full[2], None, gg, None, ws)
    assert torch.equal(gg, full[4])
    mrf.mrf_layer_norm_backward(dy, x, gamma, full[1], full[2], None, None, gb, ws)
    assert torch.equal(gb, full[5])
    mrf.mrf_layer_norm_backward(dy, x, gamma, full[1], full[2], None, None, None, None)
    # a weight without a bias
    mrf.mrf_layer_norm_forward(x, gamma, None, 1e-5, y, None, None)
    torch.testing.assert_close(y + beta, full[0], rtol=1e-6, atol=1e-6)
    # a row with NaN, one with infinity: theirs alone
    x[5, C // 2], x[11, 0] = float("nan"), float("inf")
    mrf.mrf_layer_norm_forward(x, gamma, beta, 1e-5, y, None, None)
    keep = [i for i in range(N) if i not in (5, 11)]
    assert torch.equal(y[keep], full[0][keep]) and y[5].isnan().all() and y[11].isnan().any()
    # a constant row is 0 before the parameters, and its gradient finite
    x[:] = 3.25
    mrf.mrf_layer_norm_forward(x, None, None, 1e-5, y, full[1], full[2])
    assert (y == 0).all()


def test_layer_norm_without_rows():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    x = torch.empty((0, 21), device="cuda:0")
    gg, gb = torch.full((21,), 5.0, device="cuda:0"), torch.full((21,), 5.0, device="cuda:0")
    ws = torch.empty(mrf.mrf_layer_norm_workspace_bytes(0, 21), dtype=torch.uint8, device="cuda:0")
    e = torch.empty((0,), device="cuda:0")
    mrf.mrf_layer_norm_forward(x, None, None, 1e-5, x, e, e)
    mrf.mrf_layer_norm_backward(x, x, None, e, e, x, gg, gb, ws)
    assert (gg == 0).all() and (gb == 0).all()


# ---- bucketed pairwise function

BUCKET_SHAPES = [  # G, Q, K, NB
    (1, 1, 1, 1), (3, 1, 1, 2), (2, 2, 1, 3), (2, 1, 2, 3), (5, 3, 7, 4), (4, 7, 3, 4), (1, 16, 16, 8), (300, 5, 5, 7), (1001, 21, 21, 16), (77, 21, 21, 41),
    (64, 32, 32, 16), (50, 33, 31, 9), (130, 64, 64, 32), (31, 63, 64, 64), (9, 64, 63, 5), (20, 65, 65, 32), (1, 256, 256, 32), (3, 100, 300, 32),
    (2, 300, 100, 32), (12, 1, 4099, 32), (5, 4099, 1, 32), (2, 513, 1025, 64), (2, 1025, 511, 16), (1, 700, 2049, 200), (16, 3, 5, 32), (1, 2, 5000, 5001),
    (7, 9, 64, 1000), (40, 16, 8, 1), (3, 1, 64, 33), (6, 256, 2, 12), (1, 1, 70001, 32), (4, 130, 257, 512)]


def _check_bucket(G, Q, K, NB, dtype, heads_last=False, query_offset=0, spare=0, shift=0, random_map=False):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    print("case bucket", G, Q, K, NB, dtype, heads_last, query_offset, spare, shift, flush=True)
    rng = np.random.default_rng(G + 10 * Q + 100 * K + NB)
    first = -(Q - 1) - query_offset - spare
    n = Q + K - 1 + 2 * spare
    # (entries outside the buckets are clamped)
    m = rng.integers(-2, NB + 2, n).astype(np.int32) if random_map else mrf.mrf_distance_buckets(NB, max(K // 2, 4), first, n)
    shape = (NB, G) if heads_last else (G, NB)
    table = _put(rng.normal(size=shape), "float32", shift)
    bucket_of = _put(m, "int32", shift)
    out, out_check = _guarded((G, Q, K), getattr(torch, dtype), shift)
    mrf.mrf_bucket_pairwise_forward(table, bucket_of, first, out, query_offset=query_offset, heads_last=heads_last)
    torch.cuda.synchronize()
    out_check()
    t = _np(table).T if heads_last else _np(table)
    want = torch.from_numpy(lo.bucket_pairwise(t, Q, K, m, first, query_offset)).float().to(getattr(torch, dtype))
    assert torch.equal(out.cpu(), want)
    dout = _put(rng.normal(0.3, 1.0, (G, Q, K)), dtype, shift)
    grad, grad_check = _guarded(shape, torch.float32, shift)
    ws, ws_check = _guarded((mrf.mrf_bucket_pairwise_workspace_bytes(G, Q, K, NB),), torch.uint8)
    mrf.mrf_bucket_pairwise_backward(dout, bucket_of, first, grad, ws, query_offset=query_offset, heads_last=heads_last)
    torch.cuda.synchronize()
    grad_check()
    ws_check()
    want, size = lo.bucket_pairwise_grad(_np(dout), NB, m, first, query_offset)
    if heads_last:
        want, size = want.T, size.T
    _close(grad, want, SUM * U * size)
    again, _ = _guarded(shape, torch.float32, shift)
    ws.fill_(0xFF)
    mrf.mrf_bucket_pairwise_backward(dout, bucket_of, first, again, ws, query_offset=query_offset, heads_last=heads_last)
    assert torch.equal(again, grad)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("G,Q,K,NB", BUCKET_SHAPES)
def test_bucket_pairwise_matches_definition(G, Q, K, NB, dtype):
    _check_bucket(G, Q, K, NB, dtype)
    _check_bucket(G, Q, K, NB, dtype, heads_last=True, query_offset=max(K - Q, 0), spare=3, random_map=True)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("shape,shift", [((101, 21, 21, 16), 1), ((40, 32, 32, 8), 3), ((3, 260, 256, 32), 1), ((2, 64, 1024, 32), 5), ((7, 8, 8, 8), 2)])
def test_bucket_pairwise_at_odd_addresses(shape, shift, dtype):
    _check_bucket(*shape, dtype, shift=shift, query_offset=-7, random_map=True)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("G,Q,K,NB", [(4097, 21, 21, 16), (4099, 5, 7, 3), (4100, 33, 31, 9), (4103, 56, 56, 8), (4500, 1, 1, 1), (4098, 3, 1, 2), (6000, 1, 100, 20),
                                      (4097, 4, 256, 300), (4099, 32, 64, 1000), (4096, 16, 16, 1025), (600, 64, 64, 32), (513, 40, 64, 20), (512, 64, 40, 20),
                                      (511, 33, 32, 600), (40, 70, 300, 64), (3, 300, 260, 700)])
def test_bucket_pairwise_of_thousands_of_groups(G, Q, K, NB, dtype):
    """On both sides of the numbers of groups at which the launches change."""
    _check_bucket(G, Q, K, NB, dtype)
    _check_bucket(G, Q, K, NB, dtype, heads_last=True, query_offset=3, spare=1, shift=1, random_map=True)


def test_bucket_pairwise_of_many_nearly_largest_matrices():
    _check_bucket(16385, 56, 56, 8, "float32")
    _check_bucket(5001, 63, 63, 16, "float32", heads_last=True)


@pytest.mark.parametrize("shape", [(70001, 9, 9, 8), (20011, 21, 21, 16), (3, 2048, 2048, 32), (9001, 64, 64, 40), (100003, 3, 4, 2)])
def test_bucket_pairwise_of_many_entries(shape):
    _check_bucket(*shape, "float32")
    _check_bucket(*shape, "bfloat16", heads_last=True)


def test_bucket_pairwise_of_nothing():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    m = torch.zeros(16, dtype=torch.int32, device="cuda:0")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda:0")
    for G, Q, K in ((0, 3, 3), (2, 0, 3), (2, 3, 0)):
        table, grad = torch.ones((G, 4), device="cuda:0"), torch.ones((G, 4), device="cuda:0")
        out = torch.empty((G, Q, K), device="cuda:0")
        mrf.mrf_bucket_pairwise_forward(table, m, -8, out)
        mrf.mrf_bucket_pairwise_backward(out, m, -8, grad, ws)
        assert (grad == 0).all()


def test_bucket_gradient_keeps_nan_in_its_group():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    for G, L in ((9, 21), (3, 300)):
        g = torch.ones((G, L, L), device="cuda:0")
        g[1, 2, 2] = float("nan")
        m = torch.from_numpy(mrf.mrf_distance_buckets(8, 16, -(L - 1), 2 * L - 1)).cuda()
        grad = torch.empty((G, 8), device="cuda:0")
        ws = torch.empty(mrf.mrf_bucket_pairwise_workspace_bytes(G, L, L, 8), dtype=torch.uint8, device="cuda:0")
        mrf.mrf_bucket_pairwise_backward(g, m, -(L - 1), grad, ws)
        bad = torch.zeros((G, 8), dtype=torch.bool, device="cuda:0")
        bad[1, 0] = True
        assert torch.equal(grad.isnan(), bad)


# ---- log-probabilities and policy loss

POLICY_SHAPES = [(1, 1), (2, 1), (5, 2), (7, 3), (1, 21), (1961, 21), (100, 5), (64, 8), (77, 12), (333, 16), (50, 24), (33, 31), (65, 32), (90, 33), (41, 48),
                 (70, 63), (66, 64), (67, 65), (411, 70), (129, 96), (31, 127), (37, 128), (45, 192), (20, 200), (13, 255), (40, 256), (9, 257), (15, 500),
                 (8, 512), (12, 1000), (7, 1024), (5, 1025), (3, 2048), (6, 3001), (4, 4096), (3, 5003), (2, 8192), (3, 10001), (2, 32000), (1, 32771),
                 (2, 50257)]


def _check_policy(N, L, dtype, shift=0, masked=False, barred=False, with_old=True, kl=0.05, per=1, scale=1.0, spread=2.0, label_dtype=None):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    print("case policy", N, L, dtype, shift, masked, barred, with_old, kl, per, flush=True)
    rng = np.random.default_rng(N + 1000 * L)
    label_dtype = label_dtype or ("uint8" if L <= 256 else "int32")
    a = rng.integers(0, L, N)
    c = rng.normal(0.0, spread, (N, L))
    if barred:
        bar = rng.random((N, L)) < 0.3
        bar[np.arange(N), a] = False
        c[bar] = np.inf
    mask = (rng.random(N) < 0.7).astype(np.uint8) if masked else None
    if masked:
        c[mask == 0] = np.where(rng.random(((mask == 0).sum(), 1)) < 0.5, np.nan, np.inf)
    cost = _put(c, dtype, shift)
    cd = _np(cost)
    counted = np.ones(N, bool) if mask is None else mask != 0
    lp = np.zeros(N)
    lp[counted] = lo.softmin_logp(cd[counted], a[counted])
    # log ratios on both sides of the bounds, none within 0.005 of one (the gradient jumps there)
    delta = rng.normal(0.0, 0.25, N)
    for edge in (np.log(0.8), np.log(1.3)):
        near = np.abs(delta - edge) < 0.005
        delta[near] += 0.02
    old = (lp - delta).astype(np.float32) if with_old else None
    ref = (lp + rng.normal(0.0, 0.4, N)).astype(np.float32) if kl > 0 else None
    A = rng.normal(0.2, 1.0, -(-N // per)).astype(np.float32)
    put = lambda v, t: None if v is None else _put(v, t, shift)
    args = (cost, put(a, label_dtype), put(A, "float32"), put(old, "float32"), put(ref, "float32"), put(mask, "uint8"), 0.2, 0.3, kl)
    loss, loss_check = _guarded((3,), torch.float32)
    logp, logp_check = _guarded((N,), torch.float32, shift)
    grad, grad_check = _guarded((N, L), cost.dtype, shift)
    ws, ws_check = _guarded((mrf.mrf_softmin_policy_workspace_bytes(),), torch.uint8)
    mrf.mrf_softmin_policy(*args, loss, logp, grad, ws, pixels_per_advantage=per, grad_scale=scale)
    torch.cuda.synchronize()
    for check in (loss_check, logp_check, grad_check, ws_check):
        check()
    want, _, wgrad = lo.policy(cd, a, A, old, ref, mask, 0.2, 0.3, kl, per)
    # log-probability: an exponential of -z is off by (z + 2) u relative, the sum by SUM u, the logarithm and the differences by a rounding each
    low = np.where(counted, np.min(np.where(np.isnan(cd), np.inf, cd), 1, initial=np.inf), 0.0)
    z = np.where(counted[:, None], cd, 0.0) - low[:, None]
    with np.errstate(invalid="ignore"):
        e = np.exp(-z)
        ze = np.where(np.isinf(z), 0.0, z) * e
    f = e / e.sum(1, keepdims=True)
    mean_z = (ze / e.sum(1, keepdims=True)).sum(1)
    top = z[np.arange(N), a]
    lp_bound = np.where(counted, U * (mean_z + 2 + SUM + 3 * np.abs(top) + 3 * np.abs(np.log(e.sum(1))) + np.abs(lp)), 0.0)
    _close(logp, lp, lp_bound)
    n = max(int(counted.sum()), 1)
    Ai = np.abs(A[np.arange(N) // per].astype(np.float64))
    r = np.exp(lp - old) if with_old else np.ones(N)
    rel = lp_bound + 8 * U + (U * np.abs(lp - old) if with_old else 0.0)
    g_size, g_off, k_off = Ai * r, Ai * r * rel, np.zeros(N)
    if ref is not None:
        d = ref - lp
        d_off = lp_bound + U * np.abs(d)
        g_size = g_size + kl * np.abs(np.expm1(d))
        g_off = g_off + kl * (np.exp(d) * d_off + 4 * U * np.abs(np.expm1(d)))
        k_off = np.abs(np.expm1(d)) * d_off + 4 * U * (np.abs(np.expm1(d)) + np.abs(d))
    hot = np.zeros((N, L))
    hot[np.arange(N), a] = 1.0
    zf = np.where(np.isinf(z), 0.0, z)
    bound = scale / n * (g_off[:, None] * np.abs(f - hot) + g_size[:, None] * (f * U * (zf + mean_z[:, None] + 6 + SUM) + 4 * U * (f + hot)))
    bound[~counted] = 0.0
    _close(grad, wgrad * scale, bound, dtype)
    pg = (g_off * counted).sum() / n + U * (Ai * r * counted).sum() / n
    kd = (k_off * counted).sum() / n
    _close(loss, want, np.array([pg + kl * kd, pg, kd]) + 4 * U * (np.abs(want) + kl * abs(want[2])))
    # the same without gradient and without log-probabilities, and on the same buffers again
    loss2, _ = _guarded((3,), torch.float32)
    mrf.mrf_softmin_policy(*args, loss2, None, None, ws, pixels_per_advantage=per, grad_scale=scale)
    assert torch.equal(loss2, loss)
    grad2, _ = _guarded((N, L), cost.dtype, shift)
    ws.fill_(0xFF)
    mrf.mrf_softmin_policy(*args, loss2, None, grad2, ws, pixels_per_advantage=per, grad_scale=scale)
    assert torch.equal(grad2, grad) and torch.equal(loss2, loss)
    # log-probabilities alone
    if not masked:
        lp2, lp2_check = _guarded((N,), torch.float32, shift)
        mrf.mrf_softmin_logp(cost, args[1], lp2)
        torch.cuda.synchronize()
        lp2_check()
        _close(lp2, lp, lp_bound)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,L", POLICY_SHAPES)
def test_policy_matches_definition(N, L, dtype):
    _check_policy(N, L, dtype, scale=float(2 ** int(np.log2(N))) if dtype == "float16" else 1.0)
    _check_policy(N, L, dtype, masked=True, barred=True, per=max(1, N // 3), scale=float(N) if dtype == "float16" else 1.0)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,L,shift", [(70, 16, 1), (33, 96, 2), (41, 256, 3), (500, 21, 5), (9, 2048, 1), (3, 8192, 4), (2, 32000, 1)])
def test_policy_at_odd_addresses(N, L, shift, dtype):
    _check_policy(N, L, dtype, shift=shift, masked=True)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("L", [4, 6, 9, 20, 28, 36, 40, 44, 48, 52, 60, 80, 100, 112, 148, 152, 160, 176, 224])
def test_policy_of_labels_in_whole_chunks(L, dtype):
    _check_policy(131, L, dtype, scale=128.0 if dtype == "float16" else 1.0)
    _check_policy(67, L, dtype, shift=1, masked=True, barred=True, per=20)


@pytest.mark.parametrize("N,L", [(70001, 21), (20000, 16), (40003, 70), (9001, 192), (2100, 1024), (600, 4099)])
def test_policy_of_many_pixels(N, L):
    """More pixels than a launch has room for at once."""
    _check_policy(N, L, "float32", masked=True, per=N // 4)
    _check_policy(N, L, "bfloat16", with_old=False, kl=0.0)


@pytest.mark.parametrize("with_old,kl", [(False, 0.0), (False, 0.1), (True, 0.0)])
def test_policy_terms_that_are_left_out(with_old, kl):
    _check_policy(300, 21, "float32", with_old=with_old, kl=kl)
    _check_policy(20, 1500, "float32", with_old=with_old, kl=kl)


def test_policy_of_wide_costs_and_32_bit_labels():
    """Costs hundreds apart (probabilities underflow), labels in 32 bits for few labels."""
    _check_policy(200, 40, "float32", spread=100.0, kl=0.0, label_dtype="int32")
    _check_policy(20, 700, "float32", spread=100.0, kl=0.0)


@pytest.mark.parametrize("L", [5, 16, 21, 192, 300, 1024, 5000, 33000])
def test_policy_pixels_without_labels_and_labels_that_are_barred(L):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    N = 9
    rng = np.random.default_rng(L)
    c = rng.normal(size=(N, L)).astype(np.float32)
    c[2] = np.inf                       # no label allowed
    c[4, 3] = np.inf                    # its own label barred
    c[5] = 1e30                         # all alike, far up
    c[6] = np.finfo(np.float32).max     # the type's largest value everywhere
    a = torch.full((N,), 3, dtype=torch.int32, device="cuda:0")
    a[7], a[8] = -5, 1 << 30            # clamped
    cost = torch.from_numpy(c).cuda()
    A = torch.ones(N, device="cuda:0")
    old = torch.full((N,), -1.0, device="cuda:0")
    loss, logp, grad = torch.empty(3, device="cuda:0"), torch.empty(N, device="cuda:0"), torch.empty_like(cost)
    ws = torch.empty(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_softmin_policy(cost, a, A, old, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws)
    from oracle import mrf_learn_oracle as lo
    want, wlp, wgrad = lo.policy(c, a.cpu().numpy(), np.ones(N), old.cpu().numpy(), None, None, 0.2, 0.2)
    assert logp[2] == -float("inf") and logp[4] == -float("inf")
    assert (grad[2] == 0).all() and (grad[4] == 0).all() and torch.isfinite(grad).all()
    rows = [0, 1, 3, 5, 6, 7, 8]
    np.testing.assert_allclose(_np(logp)[rows], wlp[rows], rtol=1e-5, atol=1e-5)
    np.testing.assert_allclose(_np(grad), wgrad, rtol=1e-4, atol=1e-7)
    np.testing.assert_allclose(_np(loss), want, rtol=1e-5)
    lp = torch.empty_like(logp)
    mrf.mrf_softmin_logp(cost, a, lp)
    np.testing.assert_allclose(_np(lp)[rows], wlp[rows], rtol=1e-5, atol=1e-5)
    assert lp[2] == -float("inf") and lp[4] == -float("inf")
    # with a KL term the pixel whose own label is barred has an infinite k: the loss is infinite, the other pixels' gradients are as ever
    ref = torch.full((N,), -2.0, device="cuda:0")
    mrf.mrf_softmin_policy(cost, a, A, old, ref, None, 0.2, 0.2, 0.1, loss, logp, grad, ws)
    assert loss[0] == float("inf") and loss[2] == float("inf") and torch.isfinite(loss[1])
    allowed = c.copy()
    allowed[4, 3] = 0.0
    _, _, wgrad = lo.policy(allowed, a.cpu().numpy(), np.ones(N), old.cpu().numpy(), ref.cpu().numpy(), None, 0.2, 0.2, 0.1)
    others = [0, 1, 2, 3, 5, 6, 7, 8]
    np.testing.assert_allclose(_np(grad)[others], wgrad[others], rtol=1e-4, atol=1e-6)
    # nothing counts: no loss, no gradient
    mrf.mrf_softmin_policy(cost, a, A, old, None, torch.zeros(N, dtype=torch.uint8, device="cuda:0"), 0.2, 0.2, 0.0, loss, logp, grad, ws)
    assert (loss == 0).all() and (logp == 0).all() and (grad == 0).all()
    # NaN stays in its pixel
    cost[1, L - 1] = float("nan")
    mrf.mrf_softmin_policy(cost, a, A, old, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws)
    assert grad[1].isnan().all() and torch.isfinite(grad[[0, 2, 3, 4, 5, 6, 7, 8]]).all()
    # ... and reaches the loss, from the costs, an advantage or an old log-probability
    assert loss[:2].isnan().all()
    cost[1, L - 1] = 0.0
    for given in (A, old):
        kept = given.clone()
        given[7] = float("nan")
        mrf.mrf_softmin_policy(cost, a, A, old, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws)
        assert loss[:2].isnan().all() and grad[7].isnan().all() and torch.isfinite(grad[[0, 1, 2, 3, 4, 5, 6, 8]]).all()
        given.copy_(kept)
    mrf.mrf_softmin_policy(cost, a, A, old, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws)
    assert torch.isfinite(loss).all()


def test_policy_without_pixels():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    e, i = torch.empty((0,), device="cuda:0"), torch.empty((0,), dtype=torch.uint8, device="cuda:0")
    c = torch.empty((0, 21), device="cuda:0")
    loss = torch.ones(3, device="cuda:0")
    ws = torch.empty(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_softmin_policy(c, i, e, e, e, i, 0.2, 0.2, 0.1, loss, e, c, ws)
    assert (loss == 0).all()
    mrf.mrf_softmin_logp(c, i, e)


# ---- gradients against differences of the definitions, along random directions

def test_gradients_of_the_kernels_are_differences_of_the_definitions():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    rng = np.random.default_rng(9)
    N, C, h = 23, 21, 1e-5
    x, gamma, w = rng.normal(size=(N, C)), rng.normal(1, 0.3, C), rng.normal(size=(N, C))
    xt, gt, wt = (_put(v, "float32") for v in (x, gamma, w))
    x, gamma, w = _np(xt), _np(gt), _np(wt)
    y, mean, rstd, gx, gg, gb = (torch.empty(s, device="cuda:0") for s in ((N, C), (N,), (N,), (N, C), (C,), (C,)))
    ws = torch.empty(mrf.mrf_layer_norm_workspace_bytes(N, C), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_layer_norm_forward(xt, gt, None, 1e-5, y, mean, rstd)
    mrf.mrf_layer_norm_backward(wt, xt, gt, mean, rstd, gx, gg, gb, ws)
    f = lambda x, g: float((lo.layer_norm(x, g)[0] * w).sum())
    for grad, value, at in ((gx, x, 0), (gg, gamma, 1)):
        for _ in range(5):
            v = rng.normal(size=value.shape)
            move = lambda s: f(x + s * v, gamma) if at == 0 else f(x, gamma + s * v)
            assert float((_np(grad) * v).sum()) == pytest.approx((move(h) - move(-h)) / (2 * h), rel=1e-4, abs=1e-4)
    L = 12
    c, a, A = rng.normal(size=(N, L)), rng.integers(0, L, N), rng.normal(size=N)
    lp = lo.softmin_logp(c, a)
    old, ref = (lp - np.linspace(-0.9, 0.9, N)).astype(np.float32), (lp + rng.normal(0, 0.3, N)).astype(np.float32)
    put = lambda v, t="float32": _put(v, t)
    ct = put(c)
    c = _np(ct)
    loss, grad = torch.empty(3, device="cuda:0"), torch.empty((N, L), device="cuda:0")
    pws = torch.empty(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_softmin_policy(ct, put(a, "uint8"), put(A), put(old), put(ref), None, 0.2, 0.3, 0.1, loss, None, grad, pws)
    A = A.astype(np.float32)
    f = lambda c: lo.policy(c, a, A, old, ref, None, 0.2, 0.3, 0.1)[0][0]
    for _ in range(5):
        v = rng.normal(size=c.shape)
        assert float((_np(grad) * v).sum()) == pytest.approx((f(c + h * v) - f(c - h * v)) / (2 * h), rel=1e-4, abs=1e-5)


# ---- more than 2^32 entries: a block of rows (groups, pixels) repeated, so that every block has to come out like one alone

def _repeated(block, k):
    torch = _torch()
    out = torch.empty((k, *block.shape), dtype=block.dtype, device="cuda:0")
    out.copy_(block.expand(k, *block.shape))
    return out


def _blocks_alike(many, block):
    torch = _torch()
    for i in (0, len(many) // 2, len(many) - 2, len(many) - 1):
        assert torch.equal(many[i], block), i


@pytest.fixture
def _memory_back():
    yield
    _torch().cuda.empty_cache()


@pytest.mark.parametrize("M,C", [(1000003, 21), (100003, 208), (7001, 2050)])
def test_layer_norm_beyond_32_bit_offsets(M, C, _memory_back):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    k = (1 << 32) // (M * C) + 2
    print("case norm", k * M, C, flush=True)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(C)
    x = torch.randn((M, C), generator=gen, device="cuda:0").to(torch.bfloat16)
    dy = torch.randn((M, C), generator=gen, device="cuda:0").to(torch.bfloat16)
    gamma = torch.rand(C, generator=gen, device="cuda:0") + 0.5

    def both(x, dy):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(x.shape[:-1], device="cuda:0"), torch.empty(x.shape[:-1], device="cuda:0")
        gg, gb = torch.empty(C, device="cuda:0"), torch.empty(C, device="cuda:0")
        ws = torch.empty(mrf.mrf_layer_norm_workspace_bytes(mean.numel(), C), dtype=torch.uint8, device="cuda:0")
        mrf.mrf_layer_norm_forward(x, gamma, None, 1e-5, y, mean, rstd)
        mrf.mrf_layer_norm_backward(dy, x, gamma, mean, rstd, dx, gg, gb, ws)
        return y, dx, mean, rstd, gg, gb

    one = both(x, dy)
    many = both(_repeated(x, k), _repeated(dy, k))
    for a, b in zip(many[:4], one[:4]):
        _blocks_alike(a, b)
    # sums over rows: at most k M rows one after the other over 256 workgroups (the least), then the workgroups'
    h = (x.double() - one[2].double()[:, None]) * one[3].double()[:, None]
    size = [(dy.double() * h).abs().sum(0), dy.double().abs().sum(0)]
    for a, b, s in zip(many[4:], one[4:], size):
        bound = (k * M / 256 + 512) * U * k * s
        assert ((a.double() - k * b.double()).abs() <= bound).all()


def test_bucket_pairwise_beyond_32_bit_offsets_many_matrices(_memory_back):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    M, Q, NB = 100003, 21, 16
    k = (1 << 32) // (M * Q * Q) + 2
    print("case bucket", k * M, Q, flush=True)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    m = torch.from_numpy(mrf.mrf_distance_buckets(NB, 20, -(Q - 1), 2 * Q - 1)).cuda()
    table = torch.randn((M, NB), generator=gen, device="cuda:0")
    dout = torch.randn((M, Q, Q), generator=gen, device="cuda:0").to(torch.bfloat16)

    def both(table, dout):
        out, grad = torch.empty_like(dout), torch.empty_like(table)
        ws = torch.empty(mrf.mrf_bucket_pairwise_workspace_bytes(table.numel() // NB, Q, Q, NB), dtype=torch.uint8, device="cuda:0")
        mrf.mrf_bucket_pairwise_forward(table, m, -(Q - 1), out)
        mrf.mrf_bucket_pairwise_backward(dout, m, -(Q - 1), grad, ws)
        return out, grad

    one, many = both(table, dout), both(_repeated(table, k), _repeated(dout, k))
    for a, b in zip(many, one):
        _blocks_alike(a, b)


def test_bucket_pairwise_beyond_32_bit_offsets_one_matrix(_memory_back):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    L, NB = 66001, 32
    print("case bucket", 1, L, flush=True)
    host = mrf.mrf_distance_buckets(NB, 40000, -(L - 1), 2 * L - 1)
    m = torch.from_numpy(host).cuda()
    table = torch.arange(NB, dtype=torch.float32, device="cuda:0")[None]
    out = torch.empty((1, L, L), dtype=torch.bfloat16, device="cuda:0")
    mrf.mrf_bucket_pairwise_forward(table, m, -(L - 1), out)
    rows = [0, 31000, 65074, 65075, 65076, L - 1]      # (row 65,075 holds entry 2^32)
    for q in rows:
        want = table[0].index_select(0, m[L - 1 - q:2 * L - 1 - q].long()).to(torch.bfloat16)
        assert torch.equal(out[0, q], want), q
    out.zero_()
    for q in rows:
        out[0, q] = 1.0
    grad = torch.empty_like(table)
    ws = torch.empty(mrf.mrf_bucket_pairwise_workspace_bytes(1, L, L, NB), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_bucket_pairwise_backward(out, m, -(L - 1), grad, ws)
    # (sums of ones below 2^24: exact)
    want = sum(np.bincount(host[L - 1 - q:2 * L - 1 - q], minlength=NB) for q in rows)
    np.testing.assert_array_equal(grad.cpu().numpy()[0], want)


@pytest.mark.parametrize("M,L", [(1000003, 21), (130001, 128), (2003, 9000), (301, 40001)])
def test_policy_beyond_32_bit_offsets(M, L, _memory_back):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    k = (1 << 32) // (M * L) + 2
    print("case policy", k * M, L, flush=True)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(L)
    cost = torch.randn((M, L), generator=gen, device="cuda:0").to(torch.bfloat16)
    labels = torch.randint(0, L, (M,), generator=gen, device="cuda:0", dtype=torch.int32)
    A = torch.randn(M, generator=gen, device="cuda:0")
    ws = torch.empty(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device="cuda:0")

    def both(cost, labels, A):
        loss, logp, grad, alone = torch.empty(3, device="cuda:0"), torch.empty_like(A), torch.empty_like(cost), torch.empty_like(A)
        # (scaled by the number of pixels: 1 / n cancels exactly)
        mrf.mrf_softmin_policy(cost, labels, A, None, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws, grad_scale=float(np.float32(A.numel())))
        mrf.mrf_softmin_logp(cost, labels, alone)
        return loss, logp, grad, alone

    one, many = both(cost, labels, A), both(_repeated(cost, k), _repeated(labels, k), _repeated(A, k))
    for a, b in zip(many[1:], one[1:]):
        _blocks_alike(a, b)
    # the mean over k times the same pixels, in 64 bits, rounded once
    assert abs(float(many[0][0]) - float(one[0][0])) <= 4 * U * float(A.abs().mean())


# ---- streams, graphs, refusals

def test_learning_operators_replayed_from_a_graph_on_a_stream_of_its_own():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    N, C = 3000, 21
    side = torch.cuda.Stream()
    rng = np.random.default_rng(12)
    x, dy, gamma, beta = (_put(rng.normal(size=s), "float32") for s in ((N, C), (N, C), (C,), (C,)))
    table = _put(rng.normal(size=(1, 16)), "float32")
    m = torch.from_numpy(mrf.mrf_distance_buckets(16, 16, -(C - 1), 2 * C - 1)).cuda()
    labels = _put(rng.integers(0, C, N), "uint8")
    mask = _put(rng.integers(0, 2, N), "uint8")
    old, A = _put(rng.normal(-3, 0.3, N), "float32"), _put(rng.normal(size=N), "float32")
    new = lambda *s: torch.empty(s, device="cuda:0")
    y, mean, rstd, gx, gg, gb, V, gV, loss, logp, gc = (new(N, C), new(N), new(N), new(N, C), new(C), new(C), new(1, C, C), new(1, 16), new(3),
                                                        new(N), new(N, C))
    ws = torch.empty(max(mrf.mrf_layer_norm_workspace_bytes(N, C), mrf.mrf_bucket_pairwise_workspace_bytes(1, C, C, 16),
                         mrf.mrf_softmin_policy_workspace_bytes()), dtype=torch.uint8, device="cuda:0")

    def step():
        mrf.mrf_layer_norm_forward(x, gamma, beta, 1e-5, y, mean, rstd)
        mrf.mrf_bucket_pairwise_forward(table, m, -(C - 1), V)
        mrf.mrf_softmin_policy(y, labels, A, old, None, mask, 0.2, 0.2, 0.0, loss, logp, gc, ws)
        mrf.mrf_layer_norm_backward(gc, x, gamma, mean, rstd, gx, gg, gb, ws)
        mrf.mrf_bucket_pairwise_backward(V, m, -(C - 1), gV, ws)

    outs = (y, gx, gg, gb, V, gV, loss, logp, gc)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for replay in range(3):
        x.add_(0.25 * torch.randn_like(x))
        table.mul_(-1.5)
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, v in zip(outs, want):
            assert torch.equal(o, v), "replay %d differs from the eager calls" % replay


def test_binding_refuses_tensors_that_do_not_fit():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda:0")
    x = z(4, 8)
    with pytest.raises(ValueError, match="gamma"):
        mrf.mrf_layer_norm_forward(x, z(7), None, 1e-5, x, None, None)
    with pytest.raises(ValueError, match="y has shape"):
        mrf.mrf_layer_norm_forward(x, None, None, 1e-5, z(4, 7), None, None)
    with pytest.raises(ValueError, match="float"):
        mrf.mrf_layer_norm_forward(z(4, 8, dtype=torch.float64), None, None, 1e-5, x, None, None)
    with pytest.raises(ValueError, match="contiguous"):
        mrf.mrf_layer_norm_forward(z(8, 4).t(), None, None, 1e-5, x, None, None)
    with pytest.raises(ValueError, match="contiguous"):
        mrf.mrf_layer_norm_forward(torch.zeros(4, 8), None, None, 1e-5, x, None, None)
    with pytest.raises(mrf.MrfError) as e:
        mrf.mrf_layer_norm_forward(x, None, None, 1e-5, z(4, 8, dtype=torch.float16), None, None)
    assert e.value.status == -12
    with pytest.raises(mrf.MrfError) as e:
        mrf.mrf_layer_norm_backward(x, x, None, z(4), z(4), x, z(8), z(8), z(8, dtype=torch.uint8))
    assert e.value.status == -6
    m = z(9, dtype=torch.int32)
    with pytest.raises(ValueError, match="table"):
        mrf.mrf_bucket_pairwise_forward(z(2, 4), m, -4, z(3, 5, 5))
    with pytest.raises(mrf.MrfError) as e:
        mrf.mrf_bucket_pairwise_forward(z(3, 4), m, -3, z(3, 5, 5))
    assert e.value.status == -12
    with pytest.raises(mrf.MrfError) as e:
        mrf.mrf_bucket_pairwise_forward(z(3, 4), m, -4, z(3, 5, 5), query_offset=1)
    assert e.value.status == -12
    with pytest.raises(ValueError, match="labels"):
        mrf.mrf_softmin_logp(x, z(4, dtype=torch.int64), z(4))
    with pytest.raises(ValueError, match="labels"):
        mrf.mrf_softmin_logp(x, z(5, dtype=torch.uint8), z(4))
    with pytest.raises(mrf.MrfError) as e:
        mrf.mrf_softmin_logp(z(4, 257), z(4, dtype=torch.uint8), z(4))
    assert e.value.status == -3
    lab, ws = z(4, dtype=torch.uint8), z(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8)
    with pytest.raises(ValueError, match="advantage"):
        mrf.mrf_softmin_policy(x, lab, z(3), None, None, None, 0.2, 0.2, 0.0, z(3), None, x, ws)
    with pytest.raises(mrf.MrfError) as e:
        mrf.mrf_softmin_policy(x, lab, z(4), None, None, None, 0.2, 0.2, 0.1, z(3), None, x, ws)
    assert e.value.status == -1


# ---- the policy loss's gradient alone

@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,L", [(1, 1), (2000, 2), (1961, 21), (3001, 16), (66, 64), (411, 70), (37, 128), (9, 257), (5, 1025), (6, 3001), (2, 32000), (1500, 1500), (2, 50257)])
def test_policy_gradient_alone(N, L, dtype):
    """That of the call with the loss, bit for bit: its factor comes from device memory instead."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    print("case policy gradient", N, L, dtype, flush=True)
    rng = np.random.default_rng(N + L)
    cost = _put(rng.normal(size=(N, L)), dtype, 1)
    a = _put(rng.integers(0, L, N), "int32")
    A, old, ref = (_put(rng.normal(m, 0.5, N), "float32") for m in (0.1, -1.0, -1.0))
    mask = _put(rng.random(N) < 0.7, "uint8", 3)
    ws, ws_check = _guarded((mrf.mrf_softmin_policy_workspace_bytes(),), torch.uint8)
    loss, want = torch.empty(3, device="cuda:0"), torch.empty_like(cost)
    for m, scale in ((None, 1.0), (mask, 0.375)):
        mrf.mrf_softmin_policy(cost, a, A, old, ref, m, 0.2, 0.3, 0.1, loss, None, want, ws, grad_scale=scale)
        grad, grad_check = _guarded((N, L), cost.dtype, 1)
        ws.fill_(0xFF)
        mrf.mrf_softmin_policy_backward(cost, a, A, old, ref, m, 0.2, 0.3, 0.1, torch.tensor([scale], device="cuda:0"), grad, ws)
        torch.cuda.synchronize()
        grad_check()
        ws_check()
        assert torch.equal(grad, want)


def test_policy_gradient_alone_of_nothing_and_refusals():
    torch = _torch()
    import paper_1910_10892_amd as mrf
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda:0")
    ws = z(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8)
    mrf.mrf_softmin_policy_backward(z(0, 5), z(0, dtype=torch.uint8), z(0), None, None, None, 0.2, 0.2, 0.0, z(1), z(0, 5), ws)
    c, a = z(4, 5), z(4, dtype=torch.uint8)
    with pytest.raises(ValueError, match="grad_loss"):
        mrf.mrf_softmin_policy_backward(c, a, z(4), None, None, None, 0.2, 0.2, 0.0, z(2), z(4, 5), ws)
    with pytest.raises(ValueError, match="grad_cost"):
        mrf.mrf_softmin_policy_backward(c, a, z(4), None, None, None, 0.2, 0.2, 0.0, z(1), z(4, 5, dtype=torch.float16), ws)
    with pytest.raises(ValueError, match="advantage"):
        mrf.mrf_softmin_policy_backward(c, a, z(3), None, None, None, 0.2, 0.2, 0.0, z(1), z(4, 5), ws)
    for kept in ((None, ws), (z(4, 5), None)):
        with pytest.raises(mrf.MrfError) as e:
            mrf.mrf_softmin_policy_backward(c, a, z(4), None, None, None, 0.2, 0.2, 0.0, z(1), *kept)
        assert e.value.status == -1


# ---- rows so long that a launch has not a thread for each of their columns

@pytest.mark.parametrize("C,dtype", [((1 << 25) - 3, "float32"), ((1 << 25) + 5, "float32"), ((1 << 25) + 5, "bfloat16"), ((1 << 30) + 67, "bfloat16")])
def test_layer_norm_parameter_gradients_of_the_longest_rows(C, dtype, _memory_back):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    print("case layer norm, parameters", C, dtype, flush=True)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(5)
    piece = torch.randn((2, 1, 1000003), generator=gen, device="cuda:0").to(getattr(torch, dtype))
    x, dy = (v.repeat(1, C // 1000003 + 1)[:, :C].contiguous() for v in piece)
    mean, rstd = torch.tensor([0.25], device="cuda:0"), torch.tensor([1.5], device="cuda:0")
    gg, gb = (torch.full((C,), float("nan"), device="cuda:0") for _ in range(2))
    ws = torch.empty(mrf.mrf_layer_norm_workspace_bytes(1, C), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_layer_norm_backward(dy, x, None, mean, rstd, None, gg, gb, ws)
    # (one row: products, no sums)
    assert torch.equal(gb, dy[0].float())
    del gb
    for a in range(0, C, 1 << 28):
        assert torch.equal(gg[a:a + (1 << 28)], dy[0, a:a + (1 << 28)].float() * ((x[0, a:a + (1 << 28)].float() - 0.25) * 1.5)), a


@pytest.mark.parametrize("C", [20001, 300001, 3000001])
def test_layer_norm_backward_of_long_rows_of_one_sign(C):
    """Sums over a row of values that are all alike: every rounding of a long chain would go the same way."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    print("case layer norm, long rows", C, flush=True)
    N = 3
    rng = np.random.default_rng(C)
    x = rng.normal(0.5, 1.0, (N, C)).astype(np.float32)
    dy = np.repeat(np.array([[0.1], [-0.7], [123.4]], np.float32), C, 1)
    dy[2] += x[2]
    gamma = np.full(C, 1.1, np.float32)
    xt, dyt, gt = _put(x, "float32"), _put(dy, "float32"), _put(gamma, "float32")
    y, mean, rstd, gx, gg, gb = (torch.empty(s, device="cuda:0") for s in ((N, C), (N,), (N,), (N, C), (C,), (C,)))
    ws = torch.empty(mrf.mrf_layer_norm_workspace_bytes(N, C), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_layer_norm_forward(xt, gt, None, 1e-5, y, mean, rstd)
    mrf.mrf_layer_norm_backward(dyt, xt, gt, mean, rstd, gx, gg, gb, ws)
    want, mu, rs = lo.layer_norm(x, gamma)
    h, dh = _norm_bounds(x.astype(np.float64), rs, gamma)
    _close(y, want, 1.1 * dh + U * 2 * np.abs(want))
    _close(mean, mu, 2 * U * np.abs(mu))
    _close(rstd, rs, 8 * U * rs)
    wx, wg, wb = lo.layer_norm_grad(dy, x, gamma)
    # h is off by a few roundings, and its sum with dy by no more: all sums as good as exact
    a = np.abs(dy.astype(np.float64) * gamma)
    dh = 4 * U * (1.0 + np.abs(h))
    bound = rs[:, None] * (4 * U * a + 2 * U * a.mean(1, keepdims=True) + 4 * U * np.abs(h) * (a * np.abs(h)).mean(1, keepdims=True) +
                           np.abs(h) * (a * dh).mean(1, keepdims=True) + dh * np.abs((dy * gamma * h).mean(1, keepdims=True)))
    _close(gx, wx, bound)
    _close(gg, wg, (np.abs(dy) * dh).sum(0) + SUM * U * np.abs(dy * h).sum(0))
    _close(gb, wb, SUM * U * np.abs(dy).sum(0))


# ---- rows whose level is far above their contrast

@pytest.mark.parametrize("level", [1000.1, -30000.3, 0.1])
@pytest.mark.parametrize("C", [3, 16, 21, 24, 36, 70, 192, 300, 1000, 2048, 5000, 12000, 20000, 300001])
def test_layer_norm_of_rows_with_little_contrast(C, level):
    """What single precision loses in a row's mean is found again in the differences from it: a constant row is 0, whatever its value."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    print("case layer norm, level", C, level, flush=True)
    N = 7
    rng = np.random.default_rng(C)
    x = np.full((N, C), level, np.float32)
    x[3:] += rng.normal(0.0, 0.02, (N - 3, C)).astype(np.float32)
    dy = rng.normal(0.3, 1.0, (N, C)).astype(np.float32)
    xt, dyt = _put(x, "float32"), _put(dy, "float32")
    y, mean, rstd, gx = (torch.empty(s, device="cuda:0") for s in ((N, C), (N,), (N,), (N, C)))
    mrf.mrf_layer_norm_forward(xt, None, None, 1e-5, y, mean, rstd)
    mrf.mrf_layer_norm_backward(dyt, xt, None, mean, rstd, gx, None, None, None)
    want, mu, rs = lo.layer_norm(x)
    # the mean is off by SUM u of the level at first, then by as much of that and of the contrast (the terms of the second sum), and where it is
    # stored by a rounding
    left = (SUM * U) ** 2 * np.abs(x).max()
    h = np.abs(want)
    bound = (left + SUM * U * (SUM * U * np.abs(x).max()) ** 2 * rs[:, None]) * rs[:, None] + SUM * U * (h + h.mean(1, keepdims=True))
    assert (np.abs(_np(y) - want) <= bound).all(), "off by %g" % np.abs(_np(y) - want).max()
    assert (_np(y)[:3] == 0).all() or np.abs(_np(y)[:3]).max() <= left * rs.max()
    assert (np.abs(_np(mean) - mu) <= 1.01 * U * np.abs(mu) + left + SUM * U * h.mean(1) / rs).all()
    _close(rstd, rs, SUM * U * rs + 0.5 * rs ** 3 * SUM * U * (SUM * U * np.abs(x).max()) ** 2)
    # backward reads the stored mean
    dh = (U * np.abs(x).max() + left) * rs[:, None] + SUM * U * (h + h.mean(1, keepdims=True))
    wx, _, _ = lo.layer_norm_grad(dy, x)
    a = np.abs(dy)
    ma, mah = a.mean(1, keepdims=True), (a * (h + dh)).mean(1, keepdims=True)
    bound = rs[:, None] * (U * a + SUM * U * ma + (h + dh) * SUM * U * mah + dh * mah + h * (a * dh).mean(1, keepdims=True) + 4 * U * (a + ma + h * mah))
    _close(gx, wx, bound + SUM * U * np.abs(wx))


@pytest.mark.parametrize("types", TYPE_PAIRS, ids="-".join)
@pytest.mark.parametrize("C", [21, 24, 300, 2049, 20001])
def test_layer_norm_of_constant_rows_in_each_type(C, types):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    x = _put(np.array([1000.1, -4321.7, 0.3, 6.1e4])[:, None].repeat(C, 1), types[0])
    y, mean, rstd = torch.empty((4, C), dtype=getattr(torch, types[1]), device="cuda:0"), torch.empty(4, device="cuda:0"), torch.empty(4, device="cuda:0")
    mrf.mrf_layer_norm_forward(x, None, None, 1e-5, y, mean, rstd)
    left = (SUM * U) ** 2 * np.abs(_np(x))
    assert (np.abs(_np(y)) <= left / np.sqrt(1e-5)).all(), np.abs(_np(y)).max(1)
    assert torch.equal(mean, x[:, 0].float())


@pytest.mark.parametrize("M,C", [(1000003, 21), (100003, 208), (7001, 2050)])
def test_layer_norm_parameter_gradients_beyond_32_bit_offsets(M, C, _memory_back):
    """Sums over rows that do not cancel, so that a missing block of rows, or a sign, is far outside of the bound; those of the bias exactly."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    k = (1 << 32) // (M * C) + 2
    print("case norm, parameters", k * M, C, flush=True)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(C)
    x = torch.randn((M, C), generator=gen, device="cuda:0").to(torch.bfloat16)
    # towards x: dy h is positive for the most part
    dy = (x.float() + 0.5 * torch.randn((M, C), generator=gen, device="cuda:0")).to(torch.bfloat16)
    mean, rstd = torch.empty(M, device="cuda:0"), torch.empty(M, device="cuda:0")
    y = torch.empty_like(x)
    mrf.mrf_layer_norm_forward(x, None, None, 1e-5, y, mean, rstd)
    del y
    t = dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])
    want, size = k * t.sum(0), k * t.abs().sum(0)
    del t
    xs, ms, rs = _repeated(x, k).view(-1, C), _repeated(mean, k).view(-1), _repeated(rstd, k).view(-1)
    gg, gb = torch.empty(C, device="cuda:0"), torch.empty(C, device="cuda:0")
    ws = torch.empty(mrf.mrf_layer_norm_workspace_bytes(k * M, C), dtype=torch.uint8, device="cuda:0")
    dys = _repeated(dy, k).view(-1, C)
    mrf.mrf_layer_norm_backward(dys, xs, None, ms, rs, None, gg, gb, ws)
    # a lane has every (workgroups x rows of a workgroup)-th row, 256 rows at a time at least: a chain of m of k M rows, whose roundings
    # are independent of each other, and trees
    m = k * M / 256
    bound = (np.sqrt(m) + SUM) * U * size
    assert (bound < 0.05 * want.abs()).all()
    assert ((gg.double() - want).abs() <= bound).all()
    # ones in few rows, first and last among them: exact sums
    dys.zero_()
    rows = torch.cat([torch.tensor([0, 1, k * M // 2, k * M - 2, k * M - 1], device="cuda:0"), torch.randint(0, k * M, (5000,), generator=gen, device="cuda:0")]).unique()
    dys[rows] = 1.0
    mrf.mrf_layer_norm_backward(dys, xs, None, ms, rs, None, gg, gb, ws)
    assert (gb == float(rows.numel())).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("L", [5, 16, 21, 300, 5000, 33000])
def test_policy_labels_that_no_costs_allow(L, dtype):
    """A counted pixel whose label is barred under the present, the old and the reference costs alike: r = 0 and an infinite k, not the
    difference of two infinities."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    N, inf = 6, float("inf")
    rng = np.random.default_rng(L)
    c = rng.normal(size=(N, L))
    c[2, 3] = c[4, 3] = inf
    cost = _put(c, dtype)
    c = _np(cost)
    a = torch.full((N,), 3, dtype=torch.int32, device="cuda:0")
    A = torch.tensor([1.0, -1.0, 1.0, 0.5, -2.0, 0.25], device="cuda:0")
    given = torch.full((N,), -1.0, device="cuda:0")
    mrf.mrf_softmin_logp(cost, a, given)
    assert given[2] == -inf and given[4] == -inf
    old = given.clone()
    loss, logp, grad = torch.empty(3, device="cuda:0"), torch.empty(N, device="cuda:0"), torch.empty_like(cost)
    ws = torch.empty(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_softmin_policy(cost, a, A, old, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws, grad_scale=float(N))
    # (r of such a pixel is 0: it is as if its old log-probability were any finite one)
    finite = np.where(np.isinf(_np(old)), -1.0, _np(old))
    want, _, wgrad = lo.policy(c, a.cpu().numpy(), _np(A), finite, None, None, 0.2, 0.2)
    np.testing.assert_allclose(_np(loss), want, rtol=1e-5, atol=1e-6)
    np.testing.assert_allclose(_np(grad), wgrad * N, rtol=2.0 ** -7 if dtype == "bfloat16" else 2.0 ** -10 if dtype == "float16" else 1e-4, atol=1e-6)
    # the reference bars it too: k is infinite, the other pixels' gradients are as ever
    mrf.mrf_softmin_policy(cost, a, A, old, given, None, 0.2, 0.2, 0.1, loss, logp, grad, ws, grad_scale=float(N))
    assert loss[0] == inf and loss[2] == inf and torch.isfinite(loss[1])
    rows = [0, 1, 3, 5]
    np.testing.assert_allclose(_np(grad)[rows], wgrad[rows] * N, rtol=2.0 ** -7 if dtype == "bfloat16" else 2.0 ** -10 if dtype == "float16" else 1e-4, atol=1e-6)
    # NaN is still NaN
    old[2] = float("nan")
    mrf.mrf_softmin_policy(cost, a, A, old, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws)
    assert loss[0].isnan()


# ---- 16-bit matrices of nearly 64 x 64, on both sides of the number of groups at which the forward launch changes

@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("G,L", [(8192, 56), (8193, 56), (8193, 64), (16385, 64)])
def test_bucket_pairwise_of_thousands_of_16_bit_matrices(G, L, dtype):
    _check_bucket(G, L, L, 16, dtype)


def test_policy_gradient_alone_replayed_from_a_graph():
    """The factor is read when the graph runs, not when it is captured."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    N, L = 3000, 21
    rng = np.random.default_rng(13)
    cost = _put(rng.normal(size=(N, L)), "bfloat16")
    a, A, old = _put(rng.integers(0, L, N), "uint8"), _put(rng.normal(size=N), "float32"), _put(rng.normal(-3, 0.3, N), "float32")
    mask = _put(rng.integers(0, 2, N), "uint8")
    up, grad = torch.ones(1, device="cuda:0"), torch.empty_like(cost)
    ws = torch.empty(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device="cuda:0")
    step = lambda: mrf.mrf_softmin_policy_backward(cost, a, A, old, None, mask, 0.2, 0.2, 0.0, up, grad, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for factor in (1.0, 65536.0, -0.3):
        up.fill_(factor)
        mask.copy_(1 - mask)
        step()
        torch.cuda.synchronize()
        want = grad.clone()
        grad.fill_(float("nan"))
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, want), factor


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("C", [5, 21, 63, 100, 250, 257, 1000, 2047, 4095, 8191, 8193, 10001, 16383, 16384])
def test_layer_norm_of_16_bit_rows_that_are_nearly_constant(C, dtype):
    """Values with all bits of their type set, and a neighbour of theirs in one place (or in every other): the mean lies between two numbers of the
    type, and its rounding in 32 bits would be as large as the contrast."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_learn_oracle as lo
    print("case layer norm, nearly constant", C, dtype, flush=True)
    top, step = (2047.0, 1.0) if dtype == "float16" else (255.0, 1.0)
    x = np.full((6, C), top, np.float32)
    x[1, C // 2] -= step
    x[2, ::2] -= step
    x[3] = -x[1]
    x[4] = 16 * x[0]
    x[5, 0] = 0.0
    xt = _put(x, dtype)
    assert (_np(xt) == x).all()
    y, mean, rstd = (torch.empty(s, device="cuda:0") for s in ((6, C), (6,), (6,)))
    mrf.mrf_layer_norm_forward(xt, None, None, 1e-5, y, mean, rstd)
    want, mu, rs = lo.layer_norm(x)
    # what is left of the mean's error is SUM u of it, or of the contrast
    left = (SUM * U) ** 2 * np.abs(x).max(1, keepdims=True) * rs[:, None]
    h = np.abs(want)
    bound = left + SUM * U * (h + h.mean(1, keepdims=True)) + h * SUM * U * (SUM * U * np.abs(x).max(1, keepdims=True) * rs[:, None]) ** 2
    off = np.abs(_np(y) - want)
    assert (off <= bound).all(), "off by %g, allowed %g" % (off[off > bound][0], bound[off > bound][0])
    assert (np.abs(_np(mean) - mu) <= 1.01 * U * np.abs(mu) + (left + SUM * U * h.mean(1, keepdims=True))[:, 0] / rs).all()
    _close(rstd, rs, SUM * U * rs * (1.0 + (SUM * U * np.abs(x).max(1) * rs) ** 2))


# ---- the longest sums, of values that are all alike: every rounding of a chain in 32 bits would go the same way

@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("L", [40001, 3000001, 30000001])
def test_policy_of_long_rows_of_like_costs(L, dtype):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    print("case policy, like costs", L, dtype, flush=True)
    cost = torch.full((2, L), 0.1, device="cuda:0").to(getattr(torch, dtype))
    cost[:, L // 3] = 0.0
    a = torch.tensor([L // 3, L - 1], dtype=torch.int32, device="cuda:0")
    A = torch.ones(2, device="cuda:0")
    loss, logp, grad, alone = torch.empty(3, device="cuda:0"), torch.empty(2, device="cuda:0"), torch.empty_like(cost), torch.empty(2, device="cuda:0")
    ws = torch.empty(mrf.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_softmin_policy(cost, a, A, None, None, None, 0.2, 0.2, 0.0, loss, logp, grad, ws, grad_scale=2.0)
    mrf.mrf_softmin_logp(cost, a, alone)
    c = float(cost[0, 0])
    s = 1.0 + (L - 1) * np.exp(-c)
    want = np.array([0.0, -c]) - np.log(s)
    # one exponential (2 u and its argument's rounding), a sum as good as exact, a logarithm and two roundings of results of that size
    bound = U * (4 + 4 * np.abs(want))
    for got in (logp, alone):
        assert (np.abs(_np(got) - want) <= bound).all(), (np.abs(_np(got) - want) / U, np.abs(want))
    # slope -1 for both pixels: the probabilities of the labels that were not taken, but for the sign
    f = np.array([1.0, np.exp(-c)]) / s
    g = -_np(grad)
    for row, at, other in ((0, L // 3, L - 2), (1, L - 1, L // 3)):
        p = f[1] if row == 0 else f[0]
        assert abs(g[row, other] - p) <= p * (16 * U + HALF_ULP[dtype] * 1.01)
        assert abs(g[row, at] - (f[0 if row == 0 else 1] - 1.0)) <= 4 * U + HALF_ULP[dtype] * 1.01


@pytest.mark.parametrize("Q,K", [(1, 70001), (1, 3000001), (1, 30000001), (3000001, 1), (30000001, 1), (5, 3000001)])
def test_bucket_gradient_of_long_rows_of_like_entries(Q, K):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    print("case bucket, like entries", Q, K, flush=True)
    NB = 8
    host = mrf.mrf_distance_buckets(NB, 1000, -(Q - 1), Q + K - 1)
    m = torch.from_numpy(host).cuda()
    g = torch.full((1, Q, K), 0.1, device="cuda:0")
    grad = torch.empty((1, NB), device="cuda:0")
    ws = torch.empty(mrf.mrf_bucket_pairwise_workspace_bytes(1, Q, K, NB), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_bucket_pairwise_backward(g, m, -(Q - 1), grad, ws)
    d = np.arange(-(Q - 1), K)
    entries = np.minimum(np.minimum(d + Q, K - d), min(Q, K))      # of a diagonal
    want = np.bincount(host, weights=entries, minlength=NB) * float(np.float32(0.1))
    _close(grad[0], want, 16 * U * want)
