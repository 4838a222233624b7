"""Long sums of the sequence operators: many terms of one sign and size, whose roundings all fall the same way, so that a single chain of n of them is off by up to a
quarter of n units in the last place.  Held to the same SUM u as every other sum (see test_gpu_sequence.py, whose bounds these are)."""
import numpy as np
import pytest

from test_gpu_sequence import TYPES, _attention_bounds, _close, _np

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
