"""Plain fp64 definitions of the learning operators around the message passing -- TEST INFRASTRUCTURE ONLY
(the product never imports it).  numpy, no blocking, no shortcuts.

layer_norm() / layer_norm_grad()          normalisation over the last index, its gradients by the chain rule
distance_bucket()                         the bucket of one offset, by comparing integers
bucket_pairwise() / bucket_pairwise_grad()
softmin_logp()                            log-probabilities of labels (Appendix, Eq. supp-isgmr-confidence)
policy()                                  clipped policy loss with a KL term, its gradient with respect to the costs
"""
from __future__ import annotations

import numpy as np


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    """y, mean, rstd in float64; x [N][C]."""
    x = np.asarray(x, np.float64)
    mu = x.mean(-1)
    v = ((x - mu[:, None]) ** 2).mean(-1)
    rstd = 1.0 / np.sqrt(v + eps)
    y = (x - mu[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mu, rstd


def layer_norm_grad(grad_y, x, gamma=None, eps=1e-5):
    """grad_x, grad_gamma, grad_beta."""
    x, dy = np.asarray(x, np.float64), np.asarray(grad_y, np.float64)
    C = x.shape[-1]
    h, _, rstd = layer_norm(x, eps=eps)
    a = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    # y_c depends on x_j through h: d h_c / d x_j = s ([c = j] - 1 / C - h_c h_j / C)
    grad_x = rstd[:, None] * (a - a.sum(-1, keepdims=True) / C - h * (a * h).sum(-1, keepdims=True) / C)
    return grad_x, (dy * h).sum(0), dy.sum(0)


def distance_bucket(d, n_buckets, far, two_sided=True):
    """Bucket of offset d, with integers only: distances n >= m (the ones with a bucket of their own) get m + j for the
    largest j with (n / m)^(side - m) >= (far / m)^j."""
    d = int(d)
    side = n_buckets // 2 if two_sided and n_buckets > 1 else n_buckets
    m = max(side // 2, 1)
    n = abs(d) if (two_sided or d < 0) else 0
    far = max(int(far), m + 1)
    if n < m:
        b = n
    else:
        j, w = 0, side - m
        while j < w and n ** w * m ** (j + 1) >= far ** (j + 1) * m ** w:
            j += 1
        b = m + j
    b = min(b, side - 1)
    return b + (n_buckets - side if two_sided and n_buckets > 1 and d > 0 else 0)


def bucket_index(Q, K, bucket_of, first_offset, n_buckets, query_offset=0):
    """[Q][K] bucket of every entry (clamped)."""
    at = np.arange(K)[None, :] - np.arange(Q)[:, None] - query_offset - first_offset
    return np.clip(np.asarray(bucket_of)[at], 0, n_buckets - 1)


def bucket_pairwise(table, Q, K, bucket_of, first_offset, query_offset=0):
    """[G][Q][K] from table [G][NB]."""
    table = np.asarray(table, np.float64)
    return table[:, bucket_index(Q, K, bucket_of, first_offset, table.shape[1], query_offset)]


def bucket_pairwise_grad(grad_out, n_buckets, bucket_of, first_offset, query_offset=0):
    """[G][NB], and the sums of the absolute values (for tolerances)."""
    g = np.asarray(grad_out, np.float64)
    index = bucket_index(g.shape[1], g.shape[2], bucket_of, first_offset, n_buckets, query_offset)
    grad, size = np.zeros((g.shape[0], n_buckets)), np.zeros((g.shape[0], n_buckets))
    for b in range(n_buckets):
        grad[:, b] = g[:, index == b].sum(-1)
        size[:, b] = np.abs(g[:, index == b]).sum(-1)
    return grad, size


def softmin_logp(cost, labels):
    """[N]; costs of +infinity are labels that are not allowed, rows of nothing else get -infinity."""
    z = -np.asarray(cost, np.float64)
    a = np.clip(np.asarray(labels).astype(np.int64), 0, z.shape[1] - 1)
    top = z.max(-1)
    out = np.full(z.shape[0], -np.inf)
    ok = top != -np.inf
    # (differences from the largest first: costs of 1e30 would swallow the logarithm)
    out[ok] = (z[ok, a[ok]] - top[ok]) - np.log(np.exp(z[ok] - top[ok, None]).sum(-1))
    return out


def policy(cost, labels, advantage, old_logp=None, ref_logp=None, mask=None, clip_low=0.2, clip_high=0.2, kl_weight=0.0, per=1):
    """loss [3], logp [N], grad_cost [N][L]."""
    cost = np.asarray(cost, np.float64)
    N, L = cost.shape
    counts = np.ones(N, bool) if mask is None else np.asarray(mask) != 0
    n = max(int(counts.sum()), 1)
    logp, grad = np.zeros(N), np.zeros((N, L))
    gain = divergence = 0.0
    for i in np.flatnonzero(counts):
        lp = softmin_logp(cost[i:i + 1], labels[i:i + 1])[0]
        logp[i] = lp
        if np.all(cost[i] == np.inf):
            continue
        a = min(max(int(labels[i]), 0), L - 1)
        A = float(advantage[i // per])
        r = 1.0 if old_logp is None else np.exp(lp - float(old_logp[i]))
        held = min(max(r, 1.0 - clip_low), 1.0 + clip_high) * A
        gain += min(r * A, held)
        g = -r * A if r * A <= held else 0.0
        if ref_logp is not None:
            d = float(ref_logp[i]) - lp
            divergence += np.expm1(d) - d if d < np.inf else np.inf
            if kl_weight > 0:
                g += kl_weight * (1.0 - np.exp(d))
        # lp = -c_a - log sum exp(-c):  d lp / d c_l = f_l - [l = a]
        z = cost[i].min() - cost[i]
        f = np.exp(z) / np.exp(z).sum()
        grad[i] = g / n * f
        grad[i, a] -= g / n
    total = -gain / n + (kl_weight * divergence / n if kl_weight > 0 else 0.0)
    return np.array([total, -gain / n, divergence / n]), logp, grad
