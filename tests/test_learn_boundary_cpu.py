"""Refusals of the learning operators' entry points: argument errors are reported before any GPU work, so this runs without a GPU."""
import ctypes

import pytest

import paper_1910_10892_amd as mrf

FAKE = ctypes.c_void_p(0x1000)      # never dereferenced by the host checks
INF, NAN = float("inf"), float("nan")


def test_layer_norm_refusals():
    lib = mrf.load_library()

    def forward(N=4, C=8, x=FAKE, xt=0, eps=1e-5, y=FAKE, yt=0):
        return lib.mrf_layer_norm_forward(N, C, x, xt, None, None, eps, y, yt, None, None, None)

    assert forward(N=-1) == -2 and forward(C=0) == -2 and forward(N=1 << 31) == -2 and forward(C=-3) == -2
    assert forward(C=0x7fff0001) == -2 and mrf.mrf_layer_norm_workspace_bytes(1, 0x7fff0001) == 0 < mrf.mrf_layer_norm_workspace_bytes(1, 0x7fff0000)
    assert forward(xt=3) == -12 and forward(xt=-1) == -12 and forward(yt=1) == -12 and forward(xt=1, yt=2) == -12 and forward(yt=9) == -12
    for eps in (0.0, -1e-5, INF, NAN):
        assert forward(eps=eps) == -12
    assert forward(x=None) == -1 and forward(y=None) == -1
    assert forward(N=0, x=None, y=None) == 0

    need = mrf.mrf_layer_norm_workspace_bytes(4, 8)
    assert need > 0 and mrf.mrf_layer_norm_workspace_bytes(0, 8) > 0
    assert mrf.mrf_layer_norm_workspace_bytes(-1, 8) == 0 and mrf.mrf_layer_norm_workspace_bytes(4, 0) == 0

    def backward(N=4, C=8, dy=FAKE, yt=0, x=FAKE, xt=0, mean=FAKE, rstd=FAKE, gg=FAKE, gb=FAKE, ws=FAKE, size=need):
        return lib.mrf_layer_norm_backward(N, C, dy, yt, x, xt, None, mean, rstd, FAKE, gg, gb, ws, size, None)

    assert backward(dy=None) == -1 and backward(x=None) == -1 and backward(mean=None) == -1 and backward(rstd=None) == -1
    assert backward(ws=None) == -1 and backward(size=need - 1) == -6
    assert backward(N=-1) == -2 and backward(C=0) == -2 and backward(xt=2, yt=1) == -12 and backward(xt=0, yt=1) == -12


def test_bucket_pairwise_refusals():
    lib = mrf.load_library()

    def forward(G=2, Q=3, K=5, NB=4, table=FAKE, m=FAKE, first=-2, n=7, offset=0, out=FAKE, t=0):
        return lib.mrf_bucket_pairwise_forward(G, Q, K, NB, table, 0, m, first, n, offset, out, t, None)

    assert forward(G=-1) == -2 and forward(Q=-1) == -2 and forward(K=-1) == -2 and forward(NB=0) == -2 and forward(NB=65537) == -2
    assert forward(G=1 << 31) == -2 and forward(G=(1 << 31) - 1, Q=1 << 20, K=1 << 20) == -2 and forward(Q=1 << 30, K=1 << 30) == -2
    assert forward(Q=1, K=0x7fff0000) == -2 and forward(Q=0x7fff0000, K=1) == -2
    assert forward(t=3) == -12
    assert forward(table=None) == -1 and forward(m=None) == -1 and forward(out=None) == -1
    # the map holds the offsets -2..4: one less at either side, or moved queries, and it does not
    assert forward(first=-1) == -12 and forward(n=6) == -12 and forward(offset=1) == -12 and forward(offset=-1) == -12
    assert forward(offset=1 << 62) == -12 and forward(first=-(1 << 62), n=1 << 62) == -12 and forward(n=-1) == -12
    assert forward(G=0, table=None, m=None, out=None) == 0 and forward(Q=0, out=None) == 0 and forward(K=0, out=None) == 0

    assert mrf.mrf_bucket_pairwise_workspace_bytes(2, 3, 5, 4) > 0 and mrf.mrf_bucket_pairwise_workspace_bytes(2, 3, 5, 0) == 0
    need = mrf.mrf_bucket_pairwise_workspace_bytes(2, 300, 500, 4)

    def backward(G=2, Q=300, K=500, NB=4, dout=FAKE, t=0, m=FAKE, first=-299, n=799, offset=0, grad=FAKE, ws=FAKE, size=need):
        return lib.mrf_bucket_pairwise_backward(G, Q, K, NB, dout, t, 0, m, first, n, offset, grad, ws, size, None)

    assert backward(dout=None) == -1 and backward(m=None) == -1 and backward(grad=None) == -1 and backward(ws=None) == -1
    assert backward(size=need - 1) == -6 and backward(t=-1) == -12 and backward(n=798) == -12 and backward(offset=3) == -12
    assert backward(NB=0) == -2 and backward(G=0, dout=None, grad=None) == 0


def test_distance_bucket_refusals():
    lib = mrf.load_library()
    f = lib.mrf_distance_buckets
    assert f(0, 8, 1, 0, 4, FAKE) == -12 and f(4, 0, 1, 0, 4, FAKE) == -12 and f(4, 8, 1, 0, -1, FAKE) == -12 and f(65537, 8, 1, 0, 4, FAKE) == -12
    assert f(4, 8, 1, 0, 4, None) == -1 and f(4, 8, 1, 0, 0, None) == 0
    with pytest.raises(mrf.MrfError):
        mrf.mrf_distance_buckets(0, 8, 0, 4)


def test_policy_refusals():
    lib = mrf.load_library()

    def logp(N=4, L=8, c=FAKE, t=0, a=FAKE, lb=1, out=FAKE):
        return lib.mrf_softmin_logp(N, L, c, t, a, lb, out, None)

    assert logp(N=-1) == -2 and logp(N=1 << 31) == -2 and logp(L=0) == -3 and logp(L=257) == -3 and logp(L=0, lb=4) == -3
    assert logp(L=0x7fff0001, lb=4) == -3
    assert logp(lb=2) == -12 and logp(lb=8) == -12 and logp(t=3) == -12
    assert logp(c=None) == -1 and logp(a=None) == -1 and logp(out=None) == -1 and logp(N=0, c=None, a=None, out=None) == 0

    need = mrf.mrf_softmin_policy_workspace_bytes()

    def policy(N=4, L=8, c=FAKE, a=FAKE, A=FAKE, per=1, ref=FAKE, low=0.2, high=0.2, kl=0.0, scale=1.0, loss=FAKE, ws=FAKE, size=need, lb=1, t=0):
        return lib.mrf_softmin_policy(N, L, c, t, a, lb, A, per, None, ref, None, low, high, kl, scale, loss, None, None, ws, size, None)

    assert policy(N=-1) == -2 and policy(L=300) == -3 and policy(lb=3) == -12 and policy(t=7) == -12 and policy(per=0) == -12
    for bad in (-0.1, 1.0, NAN, INF):
        assert policy(low=bad) == -12
    for bad in (-0.1, NAN, INF):
        assert policy(high=bad) == -12 and policy(kl=bad) == -12
    for bad in (NAN, INF, -INF):
        assert policy(scale=bad) == -12
    assert policy(kl=0.1, ref=None) == -1
    assert policy(c=None) == -1 and policy(a=None) == -1 and policy(A=None) == -1 and policy(loss=None) == -1 and policy(ws=None) == -1
    assert policy(size=need - 1) == -6
    assert "learning operator" in mrf.mrf_strerror(-12)


def test_binding_refuses_sizes_beyond_32_bits():
    """The library's row lengths are 32-bit arguments: a longer one is refused, not cut off."""
    import torch

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    n = (1 << 32) + 8
    with pytest.raises(ValueError, match="at most"):
        mrf.mrf_layer_norm_forward(empty(1, n), None, None, 1e-5, empty(1, n), None, None)
    with pytest.raises(ValueError, match="at most"):
        mrf.mrf_layer_norm_backward(empty(1, n), empty(1, n), None, empty(1), empty(1), empty(1, n), None, None, None)
    with pytest.raises(ValueError, match="at most"):
        mrf.mrf_bucket_pairwise_forward(empty(1, 4), empty(8, dtype=torch.int32), 0, empty(1, n, 2))
    with pytest.raises(ValueError, match="at most"):
        mrf.mrf_bucket_pairwise_backward(empty(1, 2, n), empty(8, dtype=torch.int32), 0, empty(1, 4), None)
    with pytest.raises(ValueError, match="at most"):
        mrf.mrf_softmin_logp(empty(1, n), empty(1, dtype=torch.int32), empty(1))
    with pytest.raises(ValueError, match="at most"):
        mrf.mrf_softmin_policy(empty(1, n), empty(1, dtype=torch.int32), empty(1), None, None, None, 0.2, 0.2, 0.0, empty(3), None, None, None)


def test_policy_backward_refusals():
    lib = mrf.load_library()
    need = mrf.mrf_softmin_policy_workspace_bytes()

    def backward(N=4, L=8, c=FAKE, a=FAKE, A=FAKE, per=1, ref=FAKE, low=0.2, high=0.2, kl=0.0, up=FAKE, grad=FAKE, ws=FAKE, size=need, lb=1, t=0):
        return lib.mrf_softmin_policy_backward(N, L, c, t, a, lb, A, per, None, ref, None, low, high, kl, up, grad, ws, size, None)

    assert backward(N=-1) == -2 and backward(N=1 << 31) == -2 and backward(L=300) == -3 and backward(L=0, lb=4) == -3
    assert backward(lb=3) == -12 and backward(t=7) == -12 and backward(per=0) == -12
    for bad in (-0.1, 1.0, NAN, INF):
        assert backward(low=bad) == -12
    for bad in (-0.1, NAN, INF):
        assert backward(high=bad) == -12 and backward(kl=bad) == -12
    assert backward(kl=0.1, ref=None) == -1
    assert backward(c=None) == -1 and backward(a=None) == -1 and backward(A=None) == -1 and backward(up=None) == -1 and backward(grad=None) == -1
    assert backward(ws=None) == -1 and backward(size=need - 1) == -6
    assert backward(N=0, c=None, a=None, A=None, grad=None) == 0


def test_distance_buckets_of_offsets_at_the_end_of_64_bits():
    """Offsets that the sums of 64 bits would wrap around, or whose distance has no 64 bits, are refused like those of the calls that read the map."""
    lib = mrf.load_library()
    out = (ctypes.c_int32 * 8)()
    f = lib.mrf_distance_buckets
    far, last = 1 << 40, (1 << 63) - 1
    assert f(8, 16, 1, last - 3, 8, out) == -12 and f(8, 16, 1, -last - 1, 1, out) == -12 and f(8, 16, 1, 1 << 62, 1, out) == -12
    assert f(8, 16, 1, far + 1, 1, out) == -12 and f(8, 16, 1, -far - 1, 1, out) == -12 and f(8, 16, 1, 0, far + 1, None) == -12
    assert f(8, 16, 1, far, 1, out) == 0 and out[0] == 7 and f(8, 16, 1, -far, 1, out) == 0 and out[0] == 3


def test_version_is_that_of_the_learning_operators():
    """0.3.10 had none of them, and no MRF_ERR_BAD_ARGUMENT."""
    assert tuple(int(v) for v in mrf.mrf_version().split(".")) >= (0, 3, 11)
    for name in ("mrf_layer_norm_forward", "mrf_bucket_pairwise_forward", "mrf_softmin_logp", "mrf_softmin_policy", "mrf_softmin_policy_backward"):
        assert hasattr(mrf.load_library(), name)
