"""Long sums of the sequence operators: many terms of one sign and size, whose roundings all fall the same way, so that a single chain of n of them is off by up to a
quarter of n units in the last place.  Held to the same SUM u as every other sum (see test_gpu_sequence.py, whose bounds these are)."""
import numpy as np
import pytest

from test_gpu_sequence import SUM, TYPES, U, _attention_bounds, _close, _np

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _values(x, dtype):
    """64-bit values as the type holds them, and the tensor."""
    torch = _torch()
    t = torch.from_numpy(np.ascontiguousarray(x)).to(getattr(torch, dtype)).to("cuda:0")
    return t, _np(t)


def _many_keys(D, level, same, dtype):
    """One key ahead, 16,383 others at one level; values all the same, or all of one sign.  Results, and what they should be within."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_sequence_oracle as so
    print("case many keys", D, level, same, dtype, flush=True)
    K, Q, H = 16384, 70, 512      # (so many heads that the keys are not divided among workgroups)
    rng = np.random.default_rng(D)
    q, k = np.zeros((1, 1, 1, D)), np.zeros((1, K, 1, D))
    q[..., 0] = 1.0
    k[0, 1:, 0, 0] = np.log(level) / 0.35
    v = np.broadcast_to(0.5 + rng.random((1, 1, 1, D)), k.shape) if same else 0.5 + rng.random(k.shape)
    (q, qn), (k, kn), (v, vn) = (_values(x, dtype) for x in (q, k, v))
    att = mrf.MrfAttention(q.expand(1, Q, H, D), k, v, 0.35)
    assert mrf.mrf_attention_workspace_bytes(att, False) == 0
    out, lse = torch.empty(1, Q, H, D, dtype=q.dtype, device="cuda:0"), torch.empty(1, H, Q, device="cuda:0")
    mrf.mrf_attention_forward(att, out, lse, None)
    ok, _ = so.attention_pairs(1, K)
    want, _, _ = _attention_bounds(qn[0], kn[0], vn[0], qn[0], float(att.c.scale), ok, None, dtype, so)
    spread = lambda t, shape: np.broadcast_to(t[0, 0], shape)  # noqa: E731
    return (out, *(spread(t, out.shape) for t in want["out"])), (lse, *(spread(t, lse.shape) for t in want["lse"]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("level", [0.7, 0.9, 0.45])
@pytest.mark.parametrize("D", [8, 64, 128])
def test_sum_over_many_keys_of_one_probability(D, level, dtype):
    _, lse = _many_keys(D, level, False, dtype)
    _close(*lse, what="lse")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("same", [True, False])
@pytest.mark.parametrize("level", [0.7, 0.9])
@pytest.mark.parametrize("D", [8, 64, 128])
def test_values_of_many_keys_of_one_probability(D, level, same, dtype):
    out, _ = _many_keys(D, level, same, dtype)
    _close(*out, dtype, "out")


def _backward(att, g, Q, K, D, dtype, grad_table=None):
    torch = _torch()
    import paper_1910_10892_amd as mrf
    T = getattr(torch, dtype)
    out, lse = torch.empty(1, Q, 1, D, dtype=T, device="cuda:0"), torch.empty(1, 1, Q, device="cuda:0")
    ws = torch.empty(max(mrf.mrf_attention_workspace_bytes(att, b) for b in (False, True)), dtype=torch.uint8, device="cuda:0")
    grads = [torch.empty(1, n, 1, D, dtype=T, device="cuda:0") for n in (Q, K, K)]
    mrf.mrf_attention_forward(att, out, lse, ws)
    mrf.mrf_attention_backward(att, g, out, lse, *grads, grad_table, ws)
    return [t[0] for t in grads]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [8, 64, 128])
def test_gradient_of_a_query_from_many_keys(D, dtype):
    """dS of one size, of the keys' own sign, on the way to grad_q; it rises and falls again on the way to its own sum, of which nothing is left."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_sequence_oracle as so
    print("case one query's gradient", D, dtype, flush=True)
    K, Q = 32768, 3
    sign = np.where(np.arange(K) < K // 2, 1.0, -1.0)
    q, k, v, g = np.zeros((1, Q, 1, D)), np.zeros((1, K, 1, D)), np.zeros((1, K, 1, D)), np.zeros((1, Q, 1, D))
    k[0, :, 0, 1:], v[0, :, 0, 0], g[..., 0] = 1.3 * sign[:, None], 1.1 * sign, 0.9
    (q, qn), (k, kn), (v, vn), (g, gn) = (_values(x, dtype) for x in (q, k, v, g))
    att = mrf.MrfAttention(q, k, v, 0.35)
    ok, _ = so.attention_pairs(Q, K)
    want, _, _ = _attention_bounds(qn[0], kn[0], vn[0], gn[0], float(att.c.scale), ok, None, dtype, so)
    for name, got in zip(("grad_q", "grad_k", "grad_v"), _backward(att, g, Q, K, D, dtype)):
        _close(got, *want[name], dtype, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_table", [False, True])
@pytest.mark.parametrize("D", [8, 64, 128])
def test_gradients_of_keys_from_many_queries(D, with_table, dtype):
    """All queries are the same: grad_k and grad_v are sums of 32,768 terms of one size and sign."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_sequence_oracle as so
    print("case gradients of keys", D, with_table, dtype, flush=True)
    K, Q = 70, 32768
    rng = np.random.default_rng(D)
    k, v = rng.normal(size=(1, K, 1, D)) * (1.0 / np.sqrt(D)), rng.normal(size=(1, K, 1, D))
    q, g = np.broadcast_to(0.5 + rng.random((1, 1, 1, D)), (1, Q, 1, D)), np.broadcast_to(0.5 + rng.random((1, 1, 1, D)), (1, Q, 1, D))
    (q, qn), (k, kn), (v, vn), (g, gn) = (_values(x, dtype) for x in (q, k, v, g))
    table = bucket_of = grad_table = None
    if with_table:      # (a bucket, whose value so changes nothing, and which has no gradient)
        table, bucket_of = torch.zeros(1, 1, device="cuda:0"), torch.zeros(1, dtype=torch.int32, device="cuda:0")
        grad_table = torch.empty_like(table)
    att = mrf.MrfAttention(q, k, v, 0.35, table=table, bucket_of=bucket_of)
    got = _backward(att, g, Q, K, D, dtype, grad_table)
    # a query's share, Q times
    ok, _ = so.attention_pairs(1, K)
    want, ds, eds = _attention_bounds(qn[0, :1], kn[0], vn[0], gn[0, :1], float(att.c.scale), ok, None, dtype, so)
    for name, t in zip(("grad_k", "grad_v"), got[1:]):
        _close(t, Q * want[name][0], Q * want[name][1], dtype, name)
    _close(got[0], *(np.broadcast_to(t[0], got[0].shape) for t in want["grad_q"]), dtype, "grad_q")
    if with_table:
        _close(grad_table, np.zeros((1, 1)), Q * (eds + SUM * U * np.abs(ds)).sum() * np.ones((1, 1)), what="grad_table")


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_of_a_norm_from_many_tokens(dtype):
    """All tokens are the same: the gradients of gamma are sums of 4,194,304 terms of one size and sign."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    from oracle import mrf_sequence_oracle as so
    print("case gamma", dtype, flush=True)
    T, H, D = 262144, 16, 512
    rng = np.random.default_rng(5)
    (x, xn), (g, gn) = (_values(0.5 + rng.random((1, 1, 1, D)), dtype) for _ in range(2))
    gamma, _ = _values(np.ones(D), "float32")
    none = torch.empty(1, T, 0, D, dtype=x.dtype, device="cuda:0")
    grad_gamma = torch.empty(D, device="cuda:0")
    ws = torch.empty(mrf.mrf_head_rotation_workspace_bytes(T, H, 0, D), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_head_rotation_backward(g.expand(1, T, H, D).contiguous(), none, x.expand(1, T, H, D), none, gamma, None, 1e-6, None, None, None, grad_gamma, None, ws)
    _, want = so.head_rotation_grad(gn[0], xn[0], np.ones(D), 1e-6, np.zeros(0))
    _close(grad_gamma, T * H * want, T * H * SUM * U * np.abs(want), what="grad_gamma")


def test_parts_of_a_long_cache_that_are_all_alike():
    """A row of 131,072 keys of one probability and one value, in 1,024 parts.  Probabilities are exact (1 before they are divided by their sum), so the rest is the sums' own."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    K, D = 131072, 128
    rng = np.random.default_rng(3)
    q = torch.zeros(1, 1, 1, D, device="cuda:0")
    k = torch.zeros(1, K, 1, D, device="cuda:0")
    v, vn = _values(np.broadcast_to(1.0 + rng.random((1, 1, 1, D)), (1, K, 1, D)), "float32")
    att = mrf.MrfAttention(q, k, v, 0.35)
    n = mrf.mrf_attention_workspace_bytes(att, False)
    assert n == 1024 * (D + 2) * 4
    out, lse = torch.empty_like(q), torch.empty(1, 1, 1, device="cuda:0")
    mrf.mrf_attention_forward(att, out, lse, torch.empty(n, dtype=torch.uint8, device="cuda:0"))
    _close(out, vn[:, :1], SUM * U * vn[:, :1], what="out")


def test_heads_that_share_keys_and_are_all_alike():
    """512 heads on one, each summed by a workgroup of its own: 512 times what one of them gives (whose bits these are)."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    torch.manual_seed(1)
    Q, K, H, D = 40, 100, 512, 64
    q, k, v, g = (torch.randn(1, n, 1, D, device="cuda:0") for n in (Q, K, K, Q))
    results = []
    for heads in (1, H):
        att = mrf.MrfAttention(q.expand(1, Q, heads, D), k, v, 0.125)
        out, lse = torch.empty(1, Q, heads, D, device="cuda:0"), torch.empty(1, heads, Q, device="cuda:0")
        ws = torch.empty(max(mrf.mrf_attention_workspace_bytes(att, b) for b in (False, True)), dtype=torch.uint8, device="cuda:0")
        grads = [torch.empty_like(k), torch.empty_like(v)]
        mrf.mrf_attention_forward(att, out, lse, ws)
        mrf.mrf_attention_backward(att, g.expand(1, Q, heads, D).contiguous(), out, lse, None, *grads, None, ws)
        results.append(grads)
    for one, all_heads in zip(*results):
        want = H * _np(one)
        _close(all_heads, want, SUM * U * np.abs(want))


def test_offsets_of_a_long_band_that_are_all_alike():
    """Queries see the four keys around them, with a probability of 1/4 (to 4 u: lse and the exponential); gradients and values turn by a quarter from one to the next, so dP, and
    with it dS, is the same for all pairs of an offset."""
    torch = _torch()
    import paper_1910_10892_amd as mrf
    n, H, D = 131072, 8, 4
    turn = np.array([[1.0, 0.0], [0.0, 1.0], [-1.0, 0.0], [0.0, -1.0]])[np.arange(n) % 4]
    size = 1.0 + np.random.default_rng(2).random(H)
    v, g = np.zeros((1, n, 1, D)), np.zeros((1, n, H, D))
    v[0, :, 0, :2], g[0, :, :, :2] = turn, turn[:, None] * size[:, None]
    (v, _), (g, gn) = (_values(x, "float32") for x in (v, g))
    size = gn[0, 0, :, 0]
    table, bucket_of = torch.zeros(H, 4, device="cuda:0"), torch.arange(4, dtype=torch.int32, device="cuda:0")
    q = torch.zeros(1, n, H, D, device="cuda:0")
    att = mrf.MrfAttention(q, torch.zeros_like(v), v, 0.5, first_offset=-2, last_offset=1, table=table, bucket_of=bucket_of, map_offset=-2)
    out, lse, grad_table = torch.empty_like(q), torch.empty(1, H, n, device="cuda:0"), torch.empty_like(table)
    ws = torch.empty(max(mrf.mrf_attention_workspace_bytes(att, b) for b in (False, True)), dtype=torch.uint8, device="cuda:0")
    mrf.mrf_attention_forward(att, out, lse, ws)
    mrf.mrf_attention_backward(att, g, out, lse, None, None, None, grad_table, ws)
    # whole rows are queries 2 .. n - 2, whose dP sums to 0; the others, one by one
    d = np.arange(-2, 2)
    dp = np.cos(np.pi / 2 * d).round()
    want, sizes = (n - 3) * dp / 4, (n - 3) * np.abs(dp) / 4
    for i in (0, 1, n - 1):
        ok = (i + d >= 0) & (i + d < n)
        p = ok / ok.sum()
        ds = p * (dp - (p * dp).sum())
        want, sizes = want + ds, sizes + np.abs(ds)
    # dS is off by the probability's 4 u, delta's (a sum of four) and its own roundings: 16 u of 1/4 (1 + |dP|)
    bound = (16 * (n / 4 + sizes) + SUM * sizes) * U
    _close(grad_table, size[:, None] * want[None], size[:, None] * bound[None], what="grad_table")
