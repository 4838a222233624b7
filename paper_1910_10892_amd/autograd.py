"""torch.autograd wrapper around the C-ABI entry points, for end-to-end learning as in Sec. 5.2
of the paper: the final costs c of ISGMR / TRWP as a differentiable function of the unary
potentials, the edge weights and the pairwise function.

layer_norm, bucket_pairwise and policy_loss wrap the learning operators around it in the same way:
scores to unaries, a few values to a pairwise function, rewards to a gradient of the costs.

Marshalling only: the forward call is mrf_isgmr_forward / mrf_trwp_forward (which store the
argmin indices p, q, Alg. 1 / 2), the backward call is mrf_isgmr_backward /
mrf_trwp_backward (Alg. 3 / 4).  No arithmetic of the method happens here.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import mrfmp as _m


class _MessagePassing(torch.autograd.Function):
    @staticmethod
    def forward(ctx, unary, pairwise, edge_weight, cfg):
        algo, dirs, K, rho, kind, trunc, scale, w_scalar = cfg
        unary = unary.contiguous()
        pairwise = pairwise.contiguous()
        edge_weight = None if edge_weight is None else edge_weight.contiguous()
        B, H, W, L = unary.shape
        prob = _m.MrfProblem(unary, pairwise, dirs, K, edge_weight, w_scalar, rho, kind, trunc, scale)
        R = prob.R
        dev = unary.device
        cost = torch.empty_like(unary)
        labels = torch.empty((B, H, W), dtype=torch.uint8, device=dev)
        p = torch.empty((K, R, B, H, W, L), dtype=torch.uint8, device=dev)
        q = torch.empty((K, R, B, H, W), dtype=torch.uint8, device=dev)
        code = _m.MRF_ISGMR if algo == "isgmr" else _m.MRF_TRWP
        ws = torch.empty(max(_m.mrf_workspace_bytes(prob, code, False), _m.mrf_workspace_bytes(prob, code, True)),
                         dtype=torch.uint8, device=dev)
        (_m.mrf_isgmr_forward if code == _m.MRF_ISGMR else _m.mrf_trwp_forward)(prob, cost, labels, p, q, None, ws)
        ctx.prob, ctx.code, ctx.ws = prob, code, ws
        ctx.save_for_backward(p, q)
        ctx.has_w = edge_weight is not None
        ctx.mark_non_differentiable(labels)
        return cost, labels

    @staticmethod
    def backward(ctx, grad_cost, _grad_labels):
        p, q = ctx.saved_tensors
        prob = ctx.prob
        B, H, W, L = prob.shape
        dev = grad_cost.device
        need_u, need_v, need_w = ctx.needs_input_grad[0], ctx.needs_input_grad[1], ctx.needs_input_grad[2]
        g_unary = torch.empty((B, H, W, L), dtype=torch.float32, device=dev)
        g_w = torch.empty((prob.R, B, H, W), dtype=torch.float32, device=dev) if (need_w and ctx.has_w) else None
        g_v = torch.empty((L, L), dtype=torch.float32, device=dev) if need_v else None
        fn = _m.mrf_isgmr_backward if ctx.code == _m.MRF_ISGMR else _m.mrf_trwp_backward
        fn(prob, grad_cost.contiguous().float(), p, q, g_unary, g_w, g_v, ctx.ws)
        return (g_unary if need_u else None), g_v, g_w, None


class _MessagePassingEdgeTables(torch.autograd.Function):
    @staticmethod
    def forward(ctx, unary, pairwise_edge, cfg):
        algo, dirs, K, rho, rho_edge = cfg
        unary = unary.contiguous()
        pairwise_edge = pairwise_edge.contiguous()
        B, H, W, L = unary.shape
        prob = _m.MrfProblem(unary, None, dirs, K, rho=rho, rho_edge=rho_edge, pairwise_edge=pairwise_edge)
        R = prob.R
        dev = unary.device
        cost = torch.empty_like(unary)
        labels = torch.empty((B, H, W), dtype=torch.uint8, device=dev)
        p = torch.empty((K, R, B, H, W, L), dtype=torch.uint8, device=dev)
        q = torch.empty((K, R, B, H, W), dtype=torch.uint8, device=dev)
        code = _m.MRF_ISGMR if algo == "isgmr" else _m.MRF_TRWP
        ws = torch.empty(max(_m.mrf_workspace_bytes(prob, code, False), _m.mrf_workspace_bytes(prob, code, True)),
                         dtype=torch.uint8, device=dev)
        (_m.mrf_isgmr_forward if code == _m.MRF_ISGMR else _m.mrf_trwp_forward)(prob, cost, labels, p, q, None, ws)
        ctx.prob, ctx.code, ctx.ws = prob, code, ws
        ctx.save_for_backward(p, q)
        ctx.mark_non_differentiable(labels)
        return cost, labels

    @staticmethod
    def backward(ctx, grad_cost, _grad_labels):
        p, q = ctx.saved_tensors
        prob = ctx.prob
        B, H, W, L = prob.shape
        dev = grad_cost.device
        need_u, need_t = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        g_unary = torch.empty((B, H, W, L), dtype=torch.float32, device=dev)
        g_t = torch.empty((prob.R, B, H, W, L, L), dtype=torch.float32, device=dev) if need_t else None
        fn = _m.mrf_isgmr_backward if ctx.code == _m.MRF_ISGMR else _m.mrf_trwp_backward
        fn(prob, grad_cost.contiguous().float(), p, q, g_unary, None, g_t, ctx.ws)
        return (g_unary if need_u else None), g_t, None


def message_passing_edge_tables(unary, pairwise_edge, *, algo="isgmr", dirs=((0, 1), (0, -1), (1, 0), (-1, 0)),
                                K=5, rho=None, rho_edge=None):
    """As message_passing, for pairwise potentials given per edge: pairwise_edge [R,B,H,W,L,L],
    entry (r,i,mu,lambda) = theta_{i-r,i}(mu,lambda) stored at the node the edge arrives at
    (L <= 64).  Gradients flow to unary and pairwise_edge (Eq. supp-gradient-pairwise).  rho_edge
    [R,B,H,W]: TRW coefficients per edge (TRWP), in place of rho."""
    if algo not in ("isgmr", "trwp"):
        raise ValueError("algo must be 'isgmr' or 'trwp'")
    if algo == "trwp" and rho is None and rho_edge is None:
        raise ValueError("TRWP needs rho (one value per direction) or rho_edge")
    return _MessagePassingEdgeTables.apply(unary, pairwise_edge, (algo, dirs, int(K), rho, rho_edge))


def message_passing(unary, pairwise, edge_weight=None, *, algo="isgmr", dirs=((0, 1), (0, -1), (1, 0), (-1, 0)),
                    K=5, rho=None, pairwise_kind=0, trunc=0.0, scale=1.0, edge_weight_scalar=1.0):
    """Final costs c [B,H,W,L] (differentiable) and labels x* [B,H,W] (uint8) of K iterations of
    ISGMR or TRWP.  unary [B,H,W,L], pairwise [L,L] (V[mu at i-r][lambda at i]) and edge_weight
    [R,B,H,W] (stored at the destination node of each edge; None = edge_weight_scalar everywhere)
    are float32 CUDA tensors.  Gradients flow to all three (Alg. 3 / 4)."""
    if algo not in ("isgmr", "trwp"):
        raise ValueError("algo must be 'isgmr' or 'trwp'")
    if algo == "trwp" and rho is None:
        raise ValueError("TRWP needs rho (one value per direction)")
    cfg = (algo, dirs, int(K), rho, int(pairwise_kind), float(trunc), float(scale), float(edge_weight_scalar))
    return _MessagePassing.apply(unary, pairwise, edge_weight, cfg)


# ---- learning operators around the message passing


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, dtype):
        x = x.contiguous()
        weight = None if weight is None else weight.contiguous()
        bias = None if bias is None else bias.contiguous()
        y = torch.empty(x.shape, dtype=dtype, device=x.device)
        mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
        _m.mrf_layer_norm_forward(x, weight, bias, eps, y, mean, rstd)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.has_bias, ctx.dtype = bias is not None, dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_y):
        x, weight, mean, rstd = ctx.saved_tensors
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        C, dev = x.shape[-1], x.device
        grad_x = torch.empty_like(x) if need_x else None
        grad_w = torch.empty((C,), dtype=torch.float32, device=dev) if need_w and weight is not None else None
        grad_b = torch.empty((C,), dtype=torch.float32, device=dev) if need_b and ctx.has_bias else None
        ws = None
        if grad_w is not None or grad_b is not None:
            ws = torch.empty(_m.mrf_layer_norm_workspace_bytes(mean.numel(), C), dtype=torch.uint8, device=dev)
        _m.mrf_layer_norm_backward(grad_y.contiguous().to(ctx.dtype), x, weight, mean, rstd, grad_x, grad_w, grad_b, ws)
        return grad_x, grad_w, grad_b, None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5, dtype=None):
    """Layer norm over the last index of x (float32, float16 or bfloat16; weight and bias [C] float32 or
    None), in x's type or, with dtype=torch.float32, in the type that message_passing takes as unaries.
    Gradients flow to all three."""
    return _LayerNorm.apply(x, weight, bias, float(eps), x.dtype if dtype is None else dtype)


class _BucketPairwise(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, bucket_of, cfg):
        first_offset, Q, K, query_offset, heads_last, dtype = cfg
        table = table.contiguous()
        groups = tuple(table.shape[1:] if heads_last else table.shape[:-1])
        out = torch.empty((*groups, Q, K), dtype=dtype, device=table.device)
        _m.mrf_bucket_pairwise_forward(table, bucket_of, first_offset, out, query_offset, heads_last)
        ctx.save_for_backward(bucket_of)
        ctx.cfg, ctx.table_shape = cfg, table.shape
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        (bucket_of,) = ctx.saved_tensors
        first_offset, Q, K, query_offset, heads_last, dtype = ctx.cfg
        grad = torch.empty(ctx.table_shape, dtype=torch.float32, device=grad_out.device)
        NB = grad.shape[0] if heads_last else grad.shape[-1]
        ws = torch.empty(_m.mrf_bucket_pairwise_workspace_bytes(grad.numel() // NB, Q, K, NB), dtype=torch.uint8, device=grad_out.device)
        _m.mrf_bucket_pairwise_backward(grad_out.contiguous().to(dtype), bucket_of, first_offset, grad, ws, query_offset, heads_last)
        return grad, None, None


def bucket_pairwise(table, bucket_of, first_offset, Q, K, *, query_offset=0, heads_last=False, dtype=torch.float32):
    """[..., Q, K] with entry (q, k) = table[..., bucket_of[k - q - query_offset - first_offset]], from a
    learned table [..., n_buckets] float32 (heads_last: [n_buckets, ...]); bucket_of is an int32 CUDA tensor
    (mrf_distance_buckets makes the usual one).  A table [n_buckets] with Q = K = L and first_offset =
    -(L - 1) gives the pairwise function of message_passing, one [R,B,H,W,n_buckets] the tables of
    message_passing_edge_tables.  Gradients flow to the table."""
    return _BucketPairwise.apply(table, bucket_of.contiguous(), (int(first_offset), int(Q), int(K), int(query_offset), bool(heads_last), dtype))


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, cost, labels, advantage, old_logp, ref_logp, mask, cfg):
        clip_low, clip_high, kl_weight, per, scale = cfg
        cost = cost.contiguous()
        dev = cost.device
        loss = torch.empty((3,), dtype=torch.float32, device=dev)
        logp = torch.empty(cost.shape[:-1], dtype=torch.float32, device=dev)
        ws = torch.empty(_m.mrf_softmin_policy_workspace_bytes(), dtype=torch.uint8, device=dev)
        _m.mrf_softmin_policy(cost, labels, advantage, old_logp, ref_logp, mask, clip_low, clip_high, kl_weight, loss, logp, None, ws,
                              pixels_per_advantage=per, grad_scale=scale)
        ctx.save_for_backward(cost, labels, advantage, old_logp, ref_logp, mask)
        ctx.given = labels.numel(), cost.shape[-1], per, _m._type_of(cost, "cost"), _m._label_bytes(labels), clip_low, clip_high, kl_weight
        ctx.ws = ws
        total, terms = loss[0].clone(), loss[1:]
        ctx.mark_non_differentiable(terms, logp)
        return total, terms, logp

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_total, _grad_terms, _grad_logp):
        # (the gradient is not made with the loss: what comes from above is multiplied in before its entries are rounded to 16 bits)
        cost, labels, advantage, old_logp, ref_logp, mask = ctx.saved_tensors
        grad = torch.empty_like(cost)
        # (the forward call has checked all but the gradients; checks here cost more than the launch)
        _m._policy_backward(ctx.given, cost, labels, advantage, old_logp, ref_logp, mask, grad_total.float(), grad, ctx.ws)
        return grad, None, None, None, None, None, None


def policy_loss(cost, labels, advantage, old_logp=None, ref_logp=None, mask=None, *, clip_low=0.2, clip_high=0.2, kl_weight=0.0,
                pixels_per_advantage=1, grad_scale=1.0):
    """Clipped policy loss of labels [...] (uint8 or int32) under the SoftMin of cost [..., L], as
    mrf_softmin_policy states it: (loss, terms, logp) with terms = [first term, mean k] and logp [...]
    the labels' log-probabilities.  The gradient flows from loss to cost: it is formed in 32 bits, times what comes
    from above, and rounded once to cost's type (a loss scaler keeps float16 gradients in range).  grad_scale is the
    library's factor on the gradient of a call that knows no other; it changes nothing here.  advantage, old_logp and
    ref_logp are given numbers: one that asks for a gradient of its own is refused."""
    if torch.is_grad_enabled():
        for name, t in (("advantage", advantage), ("old_logp", old_logp), ("ref_logp", ref_logp)):
            if t is not None and t.requires_grad:
                raise ValueError("policy_loss has no gradient with respect to %s: detach it" % name)
    labels, advantage, old_logp, ref_logp, mask = (None if t is None else t.contiguous() for t in (labels, advantage, old_logp, ref_logp, mask))
    return _PolicyLoss.apply(cost, labels, advantage, old_logp, ref_logp, mask,
                             (float(clip_low), float(clip_high), float(kl_weight), int(pixels_per_advantage), float(grad_scale)))


def softmin_logp(cost, labels):
    """Log-probabilities [...] float32 of labels under the SoftMin of cost [..., L] (what policy_loss takes as
    old_logp and ref_logp); no gradient."""
    cost = cost.detach().contiguous()
    logp = torch.empty(cost.shape[:-1], dtype=torch.float32, device=cost.device)
    _m.mrf_softmin_logp(cost, labels.contiguous(), logp)
    return logp
