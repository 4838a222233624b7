"""The sequence operators at sizes that large calls have their own layouts for: several heads a workgroup, several pieces of a table's gradient, several heads and tokens a
group of lanes, two channels a lane, several turns of a workgroup along the steps.  Definitions and bounds are those of test_gpu_sequence.py."""
import numpy as np
import pytest

from test_gpu_sequence import TYPES, _check_attention, _check_rotation, _check_scan

pytestmark = pytest.mark.gpu


def _lengths(B, n, seed):
    """Lengths up to n, an empty sequence and a whole one among them."""
    m = np.random.default_rng(seed).integers(0, n + 1, B)
    m[0], m[B // 2], m[B - 1] = n, 0, n
    return m.tolist()


@pytest.mark.parametrize("dtype", ["float32", "float16"])      # (bfloat16 is as float16 but for the range; it has the next test)
@pytest.mark.parametrize("B,Q,K,Hq,Hk,D,NB", [(128, 90, 140, 6, 2, 16, 0), (128, 90, 250, 6, 2, 16, 7), (64, 70, 140, 8, 2, 64, 7), (64, 70, 140, 8, 2, 128, 0), (64, 70, 140, 8, 2, 128, 7),
                                              (260, 33, 140, 4, 1, 24, 0)])
def test_attention_backward_with_several_heads_in_a_workgroup(B, Q, K, Hq, Hk, D, NB, dtype):
    """512 blocks of keys or more (or that many with a part of the heads each): 3, 2 and 4 heads that share keys in one workgroup, and two tiles of queries in 16 bits.  The second has
    two pieces of the table's gradient a workgroup."""
    offsets = [-(b % 17) for b in range(B)]
    _check_attention(B, Q, K, Hq, Hk, D, dtype, last=0, offset=K - Q, ragged=(_lengths(B, Q, 1), _lengths(B, K, 2), offsets), NB=NB)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_attention_backward_of_whole_and_banded_sequences_with_several_heads_in_a_workgroup(dtype):
    _check_attention(128, 70, 140, 4, 2, 32, dtype, NB=4, heads_last=True, how="fused")
    _check_attention(128, 75, 140, 4, 2, 32, dtype, first=-40, last=9, NB=3)
    _check_attention(64, 80, 140, 8, 2, 96, dtype, first=-20, last=60)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,Hq,Hk,D,more", [(1, 20011, 5, 3, 32, {}), (2, 70001, 3, 2, 8, dict(axes=2)), (3, 3001, 9, 4, 64, dict(offset=77)), (1, 3001, 7, 2, 96, dict(rotary=32)),
                                              (5, 8000, 6, 5, 16, dict(interleaved=True)), (1, 131073, 2, 1, 2, {}), (1, 10007, 11, 0, 33, dict(gammas=False))])
def test_head_rotation_of_many_tokens(B, T, Hq, Hk, D, more, dtype):
    """Two to four heads a group of lanes, some groups with fewer, and more groups of tokens than workgroups take at once in the backward pass."""
    _check_rotation(B, T, Hq, Hk, D, dtype, **more)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("outer,T,inner", [(4, 1, 8192), (5, 1, 8001), (4, 70, 8192), (3, 40, 11000), (8, 40, 32768), (2, 140, 65536), (8, 35, 65536), (8, 70, 16384), (2, 4500, 4000)])
def test_gated_scan_of_many_channels(outer, T, inner, dtype):
    """One, two, four and eight wavefronts a workgroup, one turn and several, two channels a lane in 16 bits where rows are even; the last divided into chunks of several turns."""
    lengths = ([T, 0, max(T - 1, 1), 1, 17, T // 2, 33, T] * 2)[:outer]
    _check_scan(outer, T, inner, dtype, reverse=bool(T % 2), lengths=lengths)
    if T < 1000:
        _check_scan(outer, T, inner, dtype, reverse=not T % 2, complement=False, carried=False, how="fused" if T > 1 else "dense")
