"""Plain fp64 definitions of the sequence operators -- TEST INFRASTRUCTURE ONLY (the product never imports it).  numpy, no blocking,
no shortcuts.

attention() / attention_grad()      a sequence at a time, queries x keys written down
head_rotation() / head_rotation_grad()
gated_scan() / gated_scan_grad()    step by step
"""
from __future__ import annotations

import numpy as np


def attention_pairs(Q, K, first=None, last=None, offset=0, q_length=None, k_length=None):
    """[Q][K]: whether a key counts for a query; and the offsets key - query - offset."""
    d = np.arange(K)[None, :] - np.arange(Q)[:, None] - offset
    ok = np.ones((Q, K), bool)
    if first is not None:
        ok &= d >= first
    if last is not None:
        ok &= d <= last
    if q_length is not None:
        ok &= (np.arange(Q) < q_length)[:, None]
    if k_length is not None:
        ok &= (np.arange(K) < k_length)[None, :]
    return ok, d


def attention_bias(d, table, bucket_of, map_offset):
    """Values [Hq][..] of a table [Hq][n_buckets] at the offsets d, the map's ends beyond them; -infinity from -2^20 down."""
    which = np.clip(np.asarray(bucket_of)[np.clip(d - map_offset, 0, len(bucket_of) - 1)], 0, table.shape[1] - 1)
    table = np.asarray(table, np.float64)
    return np.where(table <= -2.0 ** 20, -np.inf, table)[:, which], which


def attention(q, k, v, scale, ok, bias=None):
    """out [Q][Hq][D], lse [Hq][Q], P [Hq][Q][K] of one sequence: q [Q][Hq][D], k, v [K][Hk][D], ok [Q][K], bias [Hq][Q][K].  Keys and queries
    that count nowhere may hold anything."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    G = q.shape[1] // k.shape[1]
    q, k, v = np.where(ok.any(1)[:, None, None], q, 0.0), np.where(ok.any(0)[:, None, None], k, 0.0), np.where(ok.any(0)[:, None, None], v, 0.0)
    s = scale * np.einsum("ihd,jhd->hij", q, np.repeat(k, G, 1))
    if bias is not None:
        s = s + bias
    s = np.where(ok[None], s, -np.inf)
    top = np.where(ok.any(1)[None], s.max(2, initial=-np.inf), 0.0)
    e = np.exp(s - top[:, :, None])
    total = e.sum(2)
    with np.errstate(divide="ignore"):
        lse = np.where(total > 0, top + np.log(total), -np.inf)
    p = e / np.where(total > 0, total, 1.0)[:, :, None]
    return np.einsum("hij,jhd->ihd", p, np.repeat(v, G, 1)), lse, p


def attention_grad(grad_out, q, k, v, scale, ok, bias=None):
    """grad_q, grad_k, grad_v, dS [Hq][Q][K], dP."""
    q, k, v, g = (np.asarray(t, np.float64) for t in (q, k, v, grad_out))
    Hk, G = k.shape[1], q.shape[1] // k.shape[1]
    _, _, p = attention(q, k, v, scale, ok, bias)
    q, g = (np.where(ok.any(1)[:, None, None], t, 0.0) for t in (q, g))
    k, v = (np.where(ok.any(0)[:, None, None], t, 0.0) for t in (k, v))
    dp = np.einsum("ihd,jhd->hij", g, np.repeat(v, G, 1))
    # P_j depends on s_m through [j = m] P_j - P_j P_m
    ds = p * dp - p * np.einsum("hij,hij->hi", p, dp)[:, :, None]
    shared = lambda t: t.reshape(t.shape[0], Hk, G, -1).sum(2)  # noqa: E731
    grad_q = scale * np.einsum("hij,jhd->ihd", ds, np.repeat(k, G, 1))
    grad_k = shared(scale * np.einsum("hij,ihd->jhd", ds, q))
    grad_v = shared(np.einsum("hij,ihd->jhd", p, g))
    return grad_q, grad_k, grad_v, ds, dp


def table_grad(ds, which, n_buckets):
    """[Hq][n_buckets] sums of dS [Hq][Q][K] over the pairs of each bucket."""
    return np.stack([(ds * (which == n)[None]).sum((1, 2)) for n in range(n_buckets)], 1)


def _angles(T, inv_freq, positions, offset):
    """[T][pairs]; positions [T][axes] or None."""
    inv_freq = np.asarray(inv_freq, np.float64)
    if positions is None:
        positions = np.arange(T)[:, None]
    positions = np.asarray(positions, np.float64) + offset
    axis = np.arange(len(inv_freq)) * positions.shape[1] // max(len(inv_freq), 1)
    return positions[:, axis] * inv_freq


def _pair(rotary, interleaved):
    n = np.arange(rotary // 2)
    return (2 * n, 2 * n + 1) if interleaved else (n, n + rotary // 2)


def _turn(x, angle, interleaved):
    """x [T][H][D] turned by angle [T][pairs]."""
    a, b = _pair(2 * angle.shape[1], interleaved)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def head_rotation(x, gamma, eps, inv_freq, positions=None, offset=0, interleaved=False):
    """x [T][H][D], gamma [D]."""
    x = np.asarray(x, np.float64)
    h = x / np.sqrt((x * x).mean(2, keepdims=True) + eps)
    return _turn(h * np.asarray(gamma, np.float64), _angles(x.shape[0], inv_freq, positions, offset), interleaved)


def head_rotation_grad(grad_out, x, gamma, eps, inv_freq, positions=None, offset=0, interleaved=False):
    """grad_x, grad_gamma."""
    x, gamma = np.asarray(x, np.float64), np.asarray(gamma, np.float64)
    D = x.shape[2]
    u = _turn(np.asarray(grad_out, np.float64), -_angles(x.shape[0], inv_freq, positions, offset), interleaved)
    n = np.sqrt((x * x).mean(2, keepdims=True) + eps)
    h, a = x / n, u * gamma
    return (a - h * (a * h).sum(2, keepdims=True) / D) / n, (u * h).sum((0, 1))


def _gate(z):
    e = np.exp(-np.abs(z))
    return np.where(z < 0, e, 1.0) / (1.0 + e), np.where(z < 0, 1.0, e) / (1.0 + e)


def gated_scan(x, z, initial=None, complement=True, reverse=False, length=None):
    """y [T][C], state behind the last step, of one row x, z [T][C]."""
    T = x.shape[0] if length is None else min(max(int(length), 0), x.shape[0])
    h = np.zeros(x.shape[1]) if initial is None else np.asarray(initial, np.float64).copy()
    y = np.zeros(x.shape)
    for t in (range(T - 1, -1, -1) if reverse else range(T)):
        a, rest = _gate(np.asarray(z[t], np.float64))
        h = a * h + (rest if complement else 1.0) * np.asarray(x[t], np.float64)
        y[t] = h
    return y, h


def gated_scan_grad(grad_y, x, z, initial=None, grad_final=None, complement=True, reverse=False, length=None):
    """grad_x, grad_z [T][C], grad_initial [C]."""
    T = x.shape[0] if length is None else min(max(int(length), 0), x.shape[0])
    order = list(range(T - 1, -1, -1) if reverse else range(T))
    first = np.zeros(x.shape[1]) if initial is None else np.asarray(initial, np.float64)
    y, _ = gated_scan(x, z, initial, complement, reverse, length)
    c = np.zeros(x.shape[1]) if grad_final is None else np.asarray(grad_final, np.float64).copy()
    gx, gz = np.zeros(x.shape), np.zeros(x.shape)
    for n in range(T - 1, -1, -1):
        t = order[n]
        before = y[order[n - 1]] if n else first
        a, rest = _gate(np.asarray(z[t], np.float64))
        g = grad_y[t] + c
        xt = np.asarray(x[t], np.float64)
        gx[t] = (rest if complement else 1.0) * g
        gz[t] = a * rest * g * (before - xt if complement else before)
        c = a * g
    return gx, gz, c
