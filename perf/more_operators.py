"""Operators that carry information along scanlines and sequences, in front of the unaries, as cases that can be timed: attention of heads
with a bias by bucketed distance, the norm of queries and keys per head with the rotation by position, and the gated linear
recurrence, each forward and backward.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes the inputs and the buffers that
a program keeps, `run()` is one pass (elementary torch operations in 32 bits, or with `own` the library's entry
points), `exact()` the same from the definitions in 64 bits, `work()` what a pass cannot do without.

Fields of a case
  op      "attention" | "rotate" | "scan"
  step    True: forward and backward pass (training); False: forward pass alone (inference)
  x       type of the tensors ("f32", "f16", "bf16")
  attention  B sequences of Q queries and K keys, Hq query heads on H key heads of D entries; first, last: a key counts where
             first <= key - query - offset <= last (None: no bound); offset: position of query 0 among the keys; ragged: keys (and queries, where
             there are as many) behind a sequence's own length do not count and hold anything, NaN too, the offset of single queries is their
             length's; NB, far: bias from NB buckets of distances (0: none); heads_last: its table lies as an embedding does
  rotate     B x T tokens, Hq query heads and H key heads of D entries, of which the first `rot` turn; axes: 1 (positions in a sequence
             from `offset` on) or 2 (rows and columns of an image); fused: q, k (and v) are parts of one projection
  scan       outer x T x inner, along T; reverse; complement: h = a h + (1 - a) x, else a h + x; ragged: lengths of their own; carried: state comes
             in and goes out; fused: x and z are halves of one projection
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
LARGEST = 1.2e9       # bytes of a drawn case at most


def _attention(name, B, Q, K, Hq, H, D, x="bf16", step=True, first=None, last=None, offset=0, ragged=False, NB=0, far=128, heads_last=False):
    return {"name": name, "op": "attention", "step": step, "x": x, "B": B, "Q": Q, "K": K, "Hq": Hq, "H": H, "D": D, "first": first, "last": last,
            "offset": offset, "ragged": ragged, "NB": NB, "far": far, "heads_last": heads_last}


def _rotate(name, B, T, Hq, H, D, x="bf16", step=True, rot=None, axes=1, offset=0, fused=False, interleaved=False):
    return {"name": name, "op": "rotate", "step": step, "x": x, "B": B, "T": T, "Hq": Hq, "H": H, "D": D, "rot": D if rot is None else rot,
            "axes": axes, "offset": offset, "fused": fused, "interleaved": interleaved}


def _scan(name, outer, T, inner, x="bf16", step=True, reverse=False, complement=True, ragged=False, carried=False, fused=False):
    return {"name": name, "op": "scan", "step": step, "x": x, "outer": outer, "T": T, "inner": inner, "reverse": reverse, "complement": complement,
            "ragged": ragged, "carried": carried, "fused": fused}


def listed():
    return [
        # a learning step on the rows of a thumbnail of the smallest configuration: launches and latency
        _attention("attention_thumbnail", 32, 48, 48, 2, 2, 16, "f32", NB=16, far=32),
        # the rows of a driving frame at half resolution, each pixel against those at up to 96 disparities, bias by disparity
        _attention("attention_disparities", 192, 624, 624, 4, 4, 32, first=-96, last=0, NB=32, far=96),
        # sequences of their own length, bias of sixteen heads by relative position from an embedding
        _attention("attention_bias", 4, 2048, 2048, 16, 16, 64, "f16", ragged=True, NB=32, far=128, heads_last=True),
        # a training step on long sequences, four query heads to a key head: the largest case
        _attention("attention_causal", 2, 4096, 4096, 16, 4, 128, last=0),
        # single queries against a long cache, each of its own length: the form for single tokens
        _attention("attention_row", 16, 1, 16411, 16, 4, 128, step=False, last=0, offset=16410, ragged=True),
        # queries and keys of an image's pixels, positions by row and column
        _rotate("rotate_thumbnail", 1, 32 * 48, 2, 2, 16, "f32", axes=2),
        # a training step on long sequences, out of one projection
        _rotate("rotate_sequence", 2, 4096, 16, 4, 128, fused=True),
        # the tokens of 16 requests far along
        _rotate("rotate_row", 16, 1, 16, 4, 128, step=False, offset=100003, fused=True),
        # the rows of a thumbnail, right to left
        _scan("scan_thumbnail", 32, 48, 16, "f32", reverse=True),
        # the columns of a segmentation batch's features: a state for each pixel of a row and channel
        _scan("scan_columns", 4, 512, 512 * 32),
        # one long sequence, few channels: split over its length
        _scan("scan_long", 1, 65537, 256, "f32", complement=False),
        # one step of 64 requests, state in and out
        _scan("scan_step", 64, 1, 2048, step=False, carried=True, fused=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """One more case: single tokens to long sequences, each type, direction and layout."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["attention", "attention", "rotate", "scan"])
        x = rng.choice(["bf16", "bf16", "f16", "f32"])
        step = rng.random() < 0.7
        H = rng.choice([1, 2, 4, 5, 8])
        Hq = H * rng.choice([1, 1, 2, 4, 7])
        D = rng.choice([_log_int(rng, 8, 128), 16 * rng.randint(1, 8), 32, 64, 64, 128])
        if op == "attention":
            kind = rng.choice(["self", "self", "band", "cross", "row"])
            B = _log_int(rng, 1, 64)
            Q = K = _log_int(rng, 16, 5000)
            NB = rng.choice([0, 16, 32])
            first, last, offset = None, rng.choice([None, 0]), 0
            if kind == "band":
                first, last = -_log_int(rng, 1, K), rng.choice([0, 0, _log_int(rng, 1, K)])
            if kind == "cross":
                Q, last = _log_int(rng, 1, 2000), None
            if kind == "row":
                Q, K, step, last = rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 1, 40000), False, 0
                offset = max(K - Q, 0)
            c = _attention("", B, Q, K, Hq, H, D, x, step, first, last, offset, rng.random() < 0.5, NB, rng.choice([64, 128]), rng.random() < 0.5)
            if B * Hq * Q * K > 6.0e8:      # scores that the plain form writes down
                continue
        elif op == "rotate":
            D += D % 2
            axes = rng.choice([1, 1, 2])
            rot = 2 * axes * rng.randint(0, D // (2 * axes)) if rng.random() < 0.3 else D - D % (2 * axes)
            c = _rotate("", _log_int(rng, 1, 16), _log_int(rng, 1, 9000), Hq, H, D, x, step, rot, axes,
                        rng.choice([0, _log_int(rng, 10, 500000)]), rng.random() < 0.5, rng.random() < 0.3)
        else:
            inner, T = _log_int(rng, 8, 9000), _log_int(rng, 1, 70000)
            outer = _log_int(rng, 1, max(1.5, 3.0e7 / (inner * T)))
            c = _scan("", outer, T, inner, x, step, rng.random() < 0.4, rng.random() < 0.6, rng.random() < 0.3, rng.random() < 0.4, rng.random() < 0.4)
        del c["name"]
        if _cost(c) <= most and work(c)["bytes"] <= LARGEST:
            return c


def _buckets(NB, far, first, count):
    """Buckets of the offsets first, first + 1, ..: half of them for either sign; the shorter half of the distances one by one,
    the others by their logarithm up to `far`, beyond which all share the last."""
    half = max(NB // 2, 1)
    single = max(half // 2, 1)
    d = np.arange(first, first + count, dtype=np.int64)
    n = np.abs(d)
    spread = np.log(np.maximum(n, 1) / single) / math.log(max(far, single + 1) / single) * (half - single)
    b = np.where(n < single, n, np.minimum(single + np.floor(spread + 1e-9).astype(np.int64), half - 1))
    return (np.minimum(b, half - 1) + np.where((d > 0) & (NB > 1), NB - half, 0)).astype(np.int32)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    dtype = TYPES[case["x"]]
    randn = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
    lengths = lambda n, most: torch.randint(max(1, most // 4), most + 1, (n,), generator=gen, device=dev, dtype=torch.int32)  # noqa: E731
    s = {"case": case}
    if case["op"] == "attention":
        B, Q, K, Hq, H, D, NB = (case[k] for k in ("B", "Q", "K", "Hq", "H", "D", "NB"))
        # normed queries and keys of some contrast, values of heads with a level of their own
        q, k = (1.3 * randn(B, Q, Hq, D)).to(dtype), (1.3 * randn(B, K, H, D)).to(dtype)
        v = (randn(B, K, H, D) + 0.5 * randn(H, D)).to(dtype)
        s.update(q=q, k=k, v=v, scale=1.0 / math.sqrt(D), k_lengths=None, q_lengths=None, query_offsets=None, table=None, bucket_of=None, first=0)
        if case["ragged"]:
            n = lengths(B, K)
            s["k_lengths"] = n
            behind = torch.arange(K, device=dev)[None, :] >= n[:, None]
            k[behind], v[behind] = float("nan"), float("nan")
            if Q == K and case["offset"] == 0:
                s["q_lengths"] = n
                q[behind] = float("nan")
            elif case["last"] is not None and Q < K:
                s["query_offsets"] = (n - K).to(torch.int32)      # added to the offset K - Q: the last queries of a sequence
        if NB:
            s["first"] = -(Q - 1) - case["offset"]
            s.update(table=randn(*((NB, Hq) if case["heads_last"] else (Hq, NB))), bucket_of=torch.from_numpy(_buckets(NB, case["far"], s["first"], Q + K - 1)).to(dev))
        s.update(out=empty(B, Q, Hq, D, dtype=dtype), lse=empty(B, Hq, Q))
        if case["step"]:
            s.update(grad_out=randn(B, Q, Hq, D).to(dtype), grad_q=torch.empty_like(q), grad_k=torch.empty_like(k), grad_v=torch.empty_like(v),
                     grad_table=None if s["table"] is None else torch.empty_like(s["table"]))
            if s["q_lengths"] is not None:
                s["grad_out"][behind] = float("nan")
        return s
    if case["op"] == "rotate":
        B, T, Hq, H, D = (case[k] for k in ("B", "T", "Hq", "H", "D"))
        if case["fused"]:
            parts = randn(B, T, Hq + 2 * H, D).mul_(1.5).to(dtype)
            q, k = parts[:, :, :Hq], parts[:, :, Hq:Hq + H]
        else:
            q, k = randn(B, T, Hq, D).mul_(1.5).to(dtype), randn(B, T, H, D).mul_(1.5).to(dtype)
        pairs = case["rot"] // (2 * case["axes"])      # of an axis
        freq = 10000.0 ** (-np.arange(pairs) / max(pairs, 1))
        s.update(q=q, k=k, gamma_q=1.0 + 0.2 * randn(D), gamma_k=1.0 + 0.2 * randn(D),
                 inv_freq=torch.from_numpy(np.tile(freq, case["axes"]).astype(np.float32)).to(dev) if pairs else None, positions=None,
                 out_q=empty(B, T, Hq, D, dtype=dtype), out_k=empty(B, T, H, D, dtype=dtype))
        if case["axes"] == 2:
            wide = max(1, int(math.sqrt(1.5 * T)))
            t = torch.arange(T, device=dev)
            s["positions"] = torch.stack([t // wide, t % wide], 1).to(torch.int32).expand(B, T, 2).contiguous() + case["offset"]
        if case["step"]:
            s.update(grad_out_q=randn(B, T, Hq, D).to(dtype), grad_out_k=randn(B, T, H, D).to(dtype), grad_q=empty(B, T, Hq, D, dtype=dtype),
                     grad_k=empty(B, T, H, D, dtype=dtype), grad_gamma_q=empty(D), grad_gamma_k=empty(D))
        return s
    outer, T, inner = (case[k] for k in ("outer", "T", "inner"))
    x, z = randn(outer, T, inner), randn(outer, T, inner).mul_(1.5).add_(2.0)      # gates that remember some ten steps
    if case["fused"]:
        both = torch.cat([x, z], 2).to(dtype)
        x, z = both[:, :, :inner], both[:, :, inner:]
    else:
        x, z = x.to(dtype), z.to(dtype)
    s.update(x=x, z=z, initial=None, final=None, lengths=None, y=empty(outer, T, inner, dtype=dtype), states=None)
    if case["carried"]:
        s.update(initial=randn(outer, inner), final=empty(outer, inner))
    if case["ragged"]:
        s["lengths"] = lengths(outer, T)
        behind = torch.arange(T, device=dev)[None, :] >= s["lengths"][:, None]
        x[behind], z[behind] = float("nan"), float("nan")
    if case["step"]:
        s.update(grad_y=randn(outer, T, inner).to(dtype), grad_x=empty(outer, T, inner, dtype=dtype), grad_z=empty(outer, T, inner, dtype=dtype),
                 grad_initial=None, grad_final=None)
        if case["carried"]:
            s.update(grad_initial=empty(outer, inner), grad_final=randn(outer, inner))
        if case["ragged"]:
            s["grad_y"][behind] = float("nan")
    return s


# ---- the plain forms

def _allowed(s):
    """[B, Q, K]: which keys count for which queries; and the offsets key - query - (offset of the sequence)."""
    case = s["case"]
    B, Q, K = case["B"], case["Q"], case["K"]
    dev = s["q"].device
    i, j = torch.arange(Q, device=dev)[:, None], torch.arange(K, device=dev)[None, :]
    rel = (j - i - case["offset"])[None]
    if s["query_offsets"] is not None:
        rel = rel - s["query_offsets"].long()[:, None, None]
    ok = torch.ones((B, Q, K), dtype=torch.bool, device=dev)
    if case["first"] is not None:
        ok = ok & (rel >= case["first"])
    if case["last"] is not None:
        ok = ok & (rel <= case["last"])
    if s["k_lengths"] is not None:
        ok = ok & (j[None] < s["k_lengths"][:, None, None])
    if s["q_lengths"] is not None:
        ok = ok & (i[None] < s["q_lengths"][:, None, None])
    return ok, rel


def _heads_first(t, behind=None, repeat=1):
    """[B, heads, T, D] in 32 bits, zeros behind the lengths."""
    t = t.float()
    if behind is not None:
        t = torch.where((torch.arange(t.shape[1], device=t.device)[None, :] < behind[:, None])[:, :, None, None], t, torch.zeros((), device=t.device))
    return t.transpose(1, 2).repeat_interleave(repeat, 1).contiguous()


def _plain_attention(s):
    case = s["case"]
    B, Q, K, Hq, H, D, NB = (case[k] for k in ("B", "Q", "K", "Hq", "H", "D", "NB"))
    dtype, rep = TYPES[case["x"]], case["Hq"] // case["H"]
    ok, rel = _allowed(s)
    q, k, v = _heads_first(s["q"], s["q_lengths"]), _heads_first(s["k"], s["k_lengths"], rep), _heads_first(s["v"], s["k_lengths"], rep)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    if NB:
        table = s["table"].t() if case["heads_last"] else s["table"]
        where = s["bucket_of"].long()[(rel - s["first"]).clamp(0, Q + K - 2)]
        scores = scores + table[:, where.reshape(-1)].view(Hq, *where.shape).transpose(0, 1)
    scores = torch.where(ok[:, None], scores, torch.full((), -math.inf, device=q.device))
    top = scores.amax(3, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - top)
    total = p.sum(3, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    p = p / total.clamp(min=1e-30)
    out = {"out": torch.matmul(p, v).transpose(1, 2).contiguous().to(dtype), "lse": torch.where(total[..., 0] > 0, lse, torch.full_like(lse, -math.inf))}
    if not case["step"]:
        return out
    g = _heads_first(s["grad_out"], s["q_lengths"])
    dp = torch.matmul(g, v.transpose(2, 3).contiguous())
    ds = p * (dp - (p * dp).sum(3, keepdim=True))
    shared = lambda t: t.view(B, H, rep, K, D).sum(2).transpose(1, 2).contiguous().to(dtype)  # noqa: E731
    out.update(grad_q=(torch.matmul(ds, k) * s["scale"]).transpose(1, 2).contiguous().to(dtype),
               grad_k=shared(torch.matmul(ds.transpose(2, 3).contiguous(), q) * s["scale"]), grad_v=shared(torch.matmul(p.transpose(2, 3).contiguous(), g)))
    if NB:
        # rows of Q + K - 1 values, read as rows that are one longer: a column is a diagonal
        d = torch.nn.functional.pad(ds.sum(0), (Q - 1, 0)).view(Hq, -1)
        d = torch.nn.functional.pad(d, (0, Q)).view(Hq, Q, Q + K).sum(1)[:, :Q + K - 1]
        grad = d @ (s["bucket_of"].long()[:, None] == torch.arange(NB, device=d.device)[None, :]).float()
        out["grad_table"] = grad.t().contiguous() if case["heads_last"] else grad
    return out


def _turns(s, double=False):
    """cos and sin [B, T, 1, pairs] of the angles, which are formed in 64 bits."""
    case = s["case"]
    if case["axes"] == 2:
        at = s["positions"].double().repeat_interleave(case["rot"] // 4, 2)
    else:
        at = (torch.arange(case["T"], device=s["q"].device) + case["offset"]).double()[None, :, None]
    angle = (at * s["inv_freq"].double()).expand(case["B"], -1, -1)[:, :, None]
    c, n = torch.cos(angle), torch.sin(angle)
    return (c, n) if double else (c.float(), n.float())


def _turned(x, turns, case, back=False):
    """The first `rot` entries of x turned pair by pair."""
    rot = case["rot"]
    if not rot:
        return x
    c, n = turns
    n = -n if back else n
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    ya, yb = a * c - b * n, a * n + b * c
    y = torch.stack([ya, yb], 4).flatten(3) if case["interleaved"] else torch.cat([ya, yb], 3)
    return torch.cat([y, x[..., rot:]], 3)


def _plain_rotate(s):
    case, out = s["case"], {}
    dtype = TYPES[case["x"]]
    turns = _turns(s) if case["rot"] else None
    for name in ("q", "k"):
        x, gamma = s[name].float(), s["gamma_" + name]
        r = torch.rsqrt((x * x).mean(3, keepdim=True) + EPS)
        h = x * r
        out["out_" + name] = _turned(h * gamma, turns, case).to(dtype)
        if case["step"]:
            u = _turned(s["grad_out_" + name].float(), turns, case, back=True)
            a = u * gamma
            out["grad_" + name] = (r * (a - h * (a * h).mean(3, keepdim=True))).to(dtype)
            out["grad_gamma_" + name] = (u * h).sum((0, 1, 2))
    return out


def _steps_in_order(s):
    """[outer, T] places of the steps in the order of the recurrence, and which of them there are."""
    case = s["case"]
    dev = s["x"].device
    n = torch.full((case["outer"],), case["T"], device=dev) if s["lengths"] is None else s["lengths"].long()
    u = torch.arange(case["T"], device=dev)[None, :].expand(case["outer"], -1)
    there = u < n[:, None]
    return torch.where(there, n[:, None] - 1 - u, u) if case["reverse"] else u, there, n


def _carry(a, b):
    """h_t = a_t h_(t-1) + b_t from h = 0, by doubling the number of steps that a value stands for."""
    a, b, d = a.clone(), b.clone(), 1
    while d < a.shape[1]:
        b[:, d:] = b[:, d:] + a[:, d:] * b[:, :-d]
        a[:, d:] = a[:, d:] * a[:, :-d]
        d *= 2
    return b


def _plain_scan(s):
    case = s["case"]
    dtype, zero = TYPES[case["x"]], torch.zeros((), device=s["x"].device)
    at, there, n = _steps_in_order(s)
    ordered = case["reverse"] or case["ragged"]
    places, there = at[:, :, None].expand(-1, -1, case["inner"]), there[:, :, None]
    take = lambda t: torch.where(there, t.float().gather(1, places), zero) if ordered else t.float()  # noqa: E731
    give = lambda t: torch.zeros_like(t).scatter_(1, places, torch.where(there, t, zero)).to(dtype) if ordered else t.to(dtype)  # noqa: E731
    x, z = take(s["x"]), take(s["z"])
    a, rest = torch.sigmoid(z), torch.sigmoid(-z)
    b = rest * x if case["complement"] else x
    first = zero.expand(case["outer"], case["inner"]) if s["initial"] is None else s["initial"]
    b = torch.cat([(a[:, :1] * first[:, None] + b[:, :1]), b[:, 1:]], 1)
    h = _carry(a, b)
    out = {"y": give(h)}
    last = (n - 1).clamp(min=0)[:, None, None].expand(-1, 1, case["inner"])
    if case["carried"]:
        out["final"] = h.gather(1, last)[:, 0]
    if not case["step"]:
        return out
    g = take(s["grad_y"])
    if case["carried"]:
        g = g.scatter_add(1, last, s["grad_final"][:, None])
    # the same recurrence from the last step to the first, with the next step's gate
    follows = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    g = _carry(follows.flip(1), g.flip(1)).flip(1)
    before = torch.cat([first[:, None].expand(-1, 1, -1), h[:, :-1]], 1)
    da = g * (before - x) if case["complement"] else g * before
    out.update(grad_x=give(rest * g if case["complement"] else g), grad_z=give(da * a * rest))
    if case["carried"]:
        out["grad_initial"] = a[:, 0] * g[:, 0]
    return out


# ---- the library's entry points

def _workspace(s, nbytes):
    """The scratch that a program keeps beside its buffers: allocated once."""
    if "workspace" not in s:
        s["workspace"] = torch.empty((nbytes(),), dtype=torch.uint8, device="cuda:0")
    return s["workspace"]


def _own(s):
    import paper_1910_10892_amd as mrf
    case = s["case"]
    if case["op"] == "attention":
        att = mrf.MrfAttention(s["q"], s["k"], s["v"], s["scale"], first_offset=case["first"], last_offset=case["last"], query_offset=case["offset"],
                               query_offsets=s["query_offsets"], q_lengths=s["q_lengths"], k_lengths=s["k_lengths"], table=s["table"],
                               bucket_of=s["bucket_of"], map_offset=s["first"], heads_last=case["heads_last"])
        ws = _workspace(s, lambda: max(mrf.mrf_attention_workspace_bytes(att, False), mrf.mrf_attention_workspace_bytes(att, True) if case["step"] else 0))
        mrf.mrf_attention_forward(att, s["out"], s["lse"], ws)
        if not case["step"]:
            return {"out": s["out"], "lse": s["lse"]}
        mrf.mrf_attention_backward(att, s["grad_out"], s["out"], s["lse"], s["grad_q"], s["grad_k"], s["grad_v"], s["grad_table"], ws)
        names = ("out", "lse", "grad_q", "grad_k", "grad_v") + (("grad_table",) if case["NB"] else ())
        return {n: s[n] for n in names}
    if case["op"] == "rotate":
        how = {"positions": s["positions"], "position_offset": 0 if case["axes"] == 2 else case["offset"], "interleaved": case["interleaved"]}
        mrf.mrf_head_rotation_forward(s["q"], s["k"], s["gamma_q"], s["gamma_k"], EPS, s["inv_freq"], s["out_q"], s["out_k"], **how)
        if not case["step"]:
            return {"out_q": s["out_q"], "out_k": s["out_k"]}
        ws = _workspace(s, lambda: mrf.mrf_head_rotation_workspace_bytes(case["B"] * case["T"], case["Hq"], case["H"], case["D"]))
        mrf.mrf_head_rotation_backward(s["grad_out_q"], s["grad_out_k"], s["q"], s["k"], s["gamma_q"], s["gamma_k"], EPS, s["inv_freq"], s["grad_q"],
                                       s["grad_k"], s["grad_gamma_q"], s["grad_gamma_k"], ws, **how)
        return {n: s[n] for n in ("out_q", "grad_q", "grad_gamma_q", "out_k", "grad_k", "grad_gamma_k")}
    how = {"complement": case["complement"], "reverse": case["reverse"]}
    sizes = case["outer"], case["T"], case["inner"]
    ws = _workspace(s, lambda: mrf.mrf_gated_scan_workspace_bytes(*sizes))
    if case["step"] and s["states"] is None:
        s["states"] = torch.empty((case["outer"], mrf.mrf_gated_scan_states(case["T"]), case["inner"]), device="cuda:0")
    mrf.mrf_gated_scan_forward(s["x"], s["z"], s["initial"], s["lengths"], s["y"], s["final"], s["states"], ws, **how)
    out = {"y": s["y"]}
    if case["carried"]:
        out["final"] = s["final"]
    if not case["step"]:
        return out
    mrf.mrf_gated_scan_backward(s["grad_y"], s["grad_final"], s["x"], s["z"], s["lengths"], s["states"], s["grad_x"], s["grad_z"], s["grad_initial"], ws, **how)
    out.update(grad_x=s["grad_x"], grad_z=s["grad_z"])
    if case["carried"]:
        out["grad_initial"] = s["grad_initial"]
    return out


def run(s):
    if own:
        return _own(s)
    return {"attention": _plain_attention, "rotate": _plain_rotate, "scan": _plain_scan}[s["case"]["op"]](s)


# ---- the definitions in 64 bits

def _exact_attention(s):
    case = s["case"]
    B, Q, K, Hq, H, D, NB = (case[k] for k in ("B", "Q", "K", "Hq", "H", "D", "NB"))
    dev, zeros = s["q"].device, lambda *shape: torch.zeros(shape, dtype=torch.float64, device=s["q"].device)  # noqa: E731
    nk = [K] * B if s["k_lengths"] is None else s["k_lengths"].tolist()
    nq = [Q] * B if s["q_lengths"] is None else s["q_lengths"].tolist()
    off = [case["offset"] + (0 if s["query_offsets"] is None else int(s["query_offsets"][b])) for b in range(B)]
    out, lse = zeros(B, Q, Hq, D), torch.full((B, Hq, Q), -math.inf, dtype=torch.float64, device=dev)
    gq, gk, gv, gt = zeros(B, Q, Hq, D), zeros(B, K, H, D), zeros(B, K, H, D), zeros(Hq, NB)
    table = None if not NB else (s["table"].t() if case["heads_last"] else s["table"]).double()
    rows = max(1, int(3.0e8 / (Hq * K)))
    for b in range(B):
        k, v = s["k"][b, :nk[b]].double().transpose(0, 1), s["v"][b, :nk[b]].double().transpose(0, 1)      # [H, keys, D]
        for a in range(0, nq[b], rows):
            i = torch.arange(a, min(a + rows, nq[b]), device=dev)
            rel = torch.arange(nk[b], device=dev)[None, :] - i[:, None] - off[b]
            barred = torch.zeros_like(rel, dtype=torch.bool)
            if case["first"] is not None:
                barred |= rel < case["first"]
            if case["last"] is not None:
                barred |= rel > case["last"]
            q = s["q"][b, i].double().view(len(i), H, Hq // H, D).permute(1, 2, 0, 3)      # [H, group, queries, D]
            z = torch.matmul(q.reshape(H, -1, D), k.transpose(1, 2)).view(Hq, len(i), nk[b]) * s["scale"]
            if NB:
                which = s["bucket_of"].long()[(rel - s["first"]).clamp(0, Q + K - 2)]
                for h in range(Hq):
                    z[h] += table[h][which]
            z.masked_fill_(barred, -math.inf)
            ls = torch.logsumexp(z, 2)
            lse[b][:, i] = ls
            p = torch.exp(z - torch.where(torch.isfinite(ls), ls, torch.zeros_like(ls))[..., None])
            grouped = lambda t: t.view(H, -1, nk[b])  # noqa: E731
            o = torch.matmul(grouped(p), v).view(Hq, len(i), D)
            out[b, i] = o.transpose(0, 1)
            if not case["step"]:
                continue
            g = s["grad_out"][b, i].double().transpose(0, 1).contiguous()      # [Hq, queries, D]
            gg = g.view(H, -1, D)
            ds = p * (torch.matmul(gg, v.transpose(1, 2)).view(Hq, len(i), nk[b]) - (g * o).sum(2)[..., None])
            gq[b, i] = (torch.matmul(grouped(ds), k) * s["scale"]).view(Hq, len(i), D).transpose(0, 1)
            gk[b, :nk[b]] += (torch.matmul(grouped(ds).transpose(1, 2), q.reshape(H, -1, D)) * s["scale"]).transpose(0, 1)
            gv[b, :nk[b]] += torch.matmul(grouped(p).transpose(1, 2), gg).transpose(0, 1)
            for n in range(NB):
                gt[:, n] += ds[:, which == n].sum(1)
    result = {"out": out, "lse": lse}
    if case["step"]:
        result.update(grad_q=gq, grad_k=gk, grad_v=gv)
        if NB:
            result["grad_table"] = gt.t().contiguous() if case["heads_last"] else gt
    return result


def _exact_rotate(s):
    case, out = s["case"], {}
    D, rot = case["D"], case["rot"]
    # the rotation as complex numbers: entry pairs times exp(i angle)
    pairs = torch.arange(rot // 2, device=s["q"].device)
    ia, ib = (2 * pairs, 2 * pairs + 1) if case["interleaved"] else (pairs, pairs + rot // 2)
    turn = torch.complex(*_turns(s, double=True)) if rot else None

    def turned(x, factor):
        y = x.clone()
        if rot:
            w = torch.complex(x[..., ia], x[..., ib]) * factor
            y[..., ia], y[..., ib] = w.real, w.imag
        return y

    for name in ("q", "k"):
        x, gamma = s[name].double(), s["gamma_" + name].double()
        n = torch.sqrt((x * x).sum(3, keepdim=True) / D + EPS)
        out["out_" + name] = turned(x / n * gamma, turn)
        if case["step"]:
            u = turned(s["grad_out_" + name].double(), None if turn is None else turn.conj())
            out["grad_gamma_" + name] = (u * x / n).sum((0, 1, 2))
            # through the norm: d n / d x = x / (D n)
            out["grad_" + name] = u * gamma / n - (u * gamma * x).sum(3, keepdim=True) / (n * n) * x / (D * n)
    return out


def _exact_scan(s):
    case = s["case"]
    outer, T, inner = (case[k] for k in ("outer", "T", "inner"))
    at, there, n = _steps_in_order(s)
    row = torch.arange(outer, device=at.device)
    pieces = 1 if T < 2048 else 256
    length = -(-T // pieces)
    pad = pieces * length - T
    # behind the last step nothing changes: gate 1, nothing added
    there = torch.nn.functional.pad(there, (0, pad))
    at = torch.nn.functional.pad(at, (0, pad))
    ordered = lambda t: torch.where(there[..., None], t[row[:, None], at].double(), torch.zeros((), dtype=torch.float64, device=at.device))  # noqa: E731
    z, x = ordered(s["z"]), ordered(s["x"])
    a = torch.where(there[..., None], 1.0 / (1.0 + torch.exp(-z)), torch.ones_like(z))
    rest = torch.where(there[..., None], 1.0 / (1.0 + torch.exp(z)), torch.zeros_like(z))
    del z

    def along(gate, add, start):
        """Step by step, all pieces side by side; then from piece to piece; then step by step again."""
        gate, add = (t.view(outer, pieces, length, inner) for t in (gate, add))
        h, f = torch.zeros_like(gate[:, :, 0]), torch.ones_like(gate[:, :, 0])
        for t in range(length if pieces > 1 else 0):
            h, f = gate[:, :, t] * h + add[:, :, t], gate[:, :, t] * f
        carry, state = [], start
        for p in range(pieces):
            carry.append(state)
            state = f[:, p] * state + h[:, p]
        h, y = torch.stack(carry, 1), torch.empty_like(gate)
        for t in range(length):
            h = gate[:, :, t] * h + add[:, :, t]
            y[:, :, t] = h
        return y.view(outer, -1, inner)

    first = torch.zeros((outer, inner), dtype=torch.float64, device=at.device) if s["initial"] is None else s["initial"].double()
    h = along(a, rest * x if case["complement"] else x, first)
    placed = lambda t: torch.zeros((outer, T, inner), dtype=torch.float64, device=at.device).index_put_(  # noqa: E731
        (row[:, None].expand_as(at)[there], at[there]), t[there])
    out = {"y": placed(h)}
    if case["carried"]:
        out["final"] = h[:, -1].clone()
    if not case["step"]:
        return out
    # what reaches step t: its own, and the next step's through that step's gate
    g = ordered(s["grad_y"])
    end = torch.zeros_like(first) if s["grad_final"] is None else s["grad_final"].double()
    g = along(torch.cat([torch.ones_like(a[:, :1]), a[:, 1:].flip(1)], 1), g.flip(1), end).flip(1)
    before = torch.cat([first[:, None], h[:, :-1]], 1)
    out.update(grad_x=placed(rest * g if case["complement"] else g), grad_z=placed(g * (before - x if case["complement"] else before) * a * rest))
    if case["carried"]:
        out["grad_initial"] = a[:, 0] * g[:, 0]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "rotate": _exact_rotate, "scan": _exact_scan}[case["op"]](s)


def _pairs(case):
    """Pairs of a query and a key that count, in a sequence of full length."""
    i = np.arange(case["Q"], dtype=np.int64) + case["offset"]
    lo = np.zeros_like(i) if case["first"] is None else np.maximum(i + case["first"], 0)
    hi = np.full_like(i, case["K"] - 1) if case["last"] is None else np.minimum(i + case["last"], case["K"] - 1)
    return int(np.maximum(hi - lo + 1, 0).sum())


def work(case):
    """Inputs read once, outputs written once.  Operations: attention 4 D a pair forward and 10 D backward (five products), norm and rotation 8 an
    element forward and 16 backward, recurrence 6 forward and 14 backward.  Ragged sequences are 5/8 of the longest on average."""
    e, step = BYTES[case["x"]], case["step"]
    if case["op"] == "attention":
        B, Q, K, Hq, H, D = (case[k] for k in ("B", "Q", "K", "Hq", "H", "D"))
        fill = 0.625 if case["ragged"] else 1.0
        both = fill * fill if case["ragged"] and Q == K else fill
        rows, keys = B * Q * Hq * D * e, B * K * H * D * e * fill
        small = 4 * B * Hq * Q + 4 * case["NB"] * Hq
        pairs = B * Hq * _pairs(case) * both
        if not step:
            return {"bytes": int(2 * rows + 2 * keys + small), "flops": int(4 * pairs * D)}
        return {"bytes": int(6 * rows + 6 * keys + 2 * small), "flops": int(14 * pairs * D)}
    if case["op"] == "rotate":
        n = case["B"] * case["T"] * (case["Hq"] + case["H"]) * case["D"]
        return {"bytes": (5 if step else 2) * n * e + (4 if step else 2) * 4 * case["D"], "flops": (24 if step else 8) * n}
    n = int(case["outer"] * case["T"] * case["inner"] * (0.625 if case["ragged"] else 1.0))
    ends = 4 * case["outer"] * case["inner"] * (2 if case["carried"] else 0)
    return {"bytes": (8 if step else 3) * n * e + ends * (2 if step else 1), "flops": (20 if step else 6) * n}
