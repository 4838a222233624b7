"""The learning operators around the message passing, as cases that can be timed: the layer norm that turns a
network's scores into unaries, the pairwise function from a table of label distances in buckets, and the clipped
policy loss on the SoftMin probabilities of the final costs (with the log-probabilities it is fed).

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes the inputs and the buffers that
a program keeps, `run()` is one pass (elementary torch operations in 32 bits, or with `own` the library's entry
points), `exact()` the same from the definitions in 64 bits, `work()` what a pass cannot do without.

Fields of a case
  op       "norm" | "bucket" | "policy" | "logp"
  step     True: forward and backward pass (training); False: forward pass alone (inference)
  norm     N rows of C values; x and y: types of the input and the output ("f32", "f16", "bf16"); affine: with weight and bias
  bucket   G groups (heads, or edges) of a Q x K matrix from NB buckets; far: distance from which all share a bucket;
           offset: position of the first query; heads_last: the table lies as [NB][G], as an embedding does; x: type of the matrix
  policy   N pixels of L labels; per: pixels that share an advantage; mask: pixels without ground truth do not count (and hold
           anything, NaN too); barred: labels that are not allowed have infinite cost; on_policy: no old log-probabilities;
           kl: weight of the KL term (0: no reference); x: type of the costs; scale: factor on the gradient (loss scaling for f16)
  logp     N pixels of L labels, x: type of the costs
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
CLIP_LOW, CLIP_HIGH = 0.2, 0.28
LARGEST = 9.0e8       # bytes of a drawn case at most


def _norm(name, N, C, x="f32", y="f32", step=True, affine=True):
    return {"name": name, "op": "norm", "step": step, "N": N, "C": C, "x": x, "y": y, "affine": affine}


def _bucket(name, G, Q, K, NB, far, x="f32", step=True, offset=0, heads_last=False):
    return {"name": name, "op": "bucket", "step": step, "G": G, "Q": Q, "K": K, "NB": NB, "far": far, "x": x, "offset": offset,
            "heads_last": heads_last}


def _policy(name, N, L, x="f32", per=1, mask=False, barred=False, on_policy=False, kl=0.04):
    return {"name": name, "op": "policy", "step": True, "N": N, "L": L, "x": x, "per": per, "mask": mask, "barred": barred,
            "on_policy": on_policy, "kl": kl, "scale": float(2 ** int(math.log2(N))) if x == "f16" else 1.0}


def _logp(name, N, L, x="f32"):
    return {"name": name, "op": "logp", "step": False, "N": N, "L": L, "x": x}


def listed():
    return [
        # a learning step on a thumbnail of the smallest configuration: launches and latency
        _norm("norm_thumbnail", 32 * 48, 16),
        # a segmentation network's scores in 16 bits, a batch of four images, to unaries in 32 bits
        _norm("norm_segment", 4 * 512 * 512, 21, "bf16", "f32"),
        # inference on a driving frame: the largest single image, 192 disparities
        _norm("norm_driving", 384 * 1248, 192, step=False),
        # the features in front of the scores: few rows, long ones, all in 16 bits
        _norm("norm_features", 4096, 2048, "bf16", "bf16"),
        # the one learned table of a denoising problem, 256 grey levels
        _bucket("bucket_table", 1, 256, 256, 32, 128),
        # a table for each edge of a 256 x 256 image in four directions, from sixteen values that a network predicts
        _bucket("bucket_edges", 4 * 256 * 256, 21, 21, 16, 16),
        # the bias of sixteen heads over long sequences
        _bucket("bucket_heads", 16, 2048, 2048, 32, 128, "bf16", heads_last=True),
        # one query against all keys before it: the form for single tokens
        _bucket("bucket_row", 16, 1, 4099, 32, 128, step=False, offset=4098, heads_last=True),
        # a crop of a segmentation problem, one reward for each pixel
        _policy("policy_crop", 37 * 53, 21),
        # a batch of four segmented images, one reward for each image, void pixels, barred classes
        _policy("policy_segment", 4 * 512 * 512, 21, per=512 * 512, mask=True, barred=True),
        # tokens over a vocabulary, costs in 16 bits
        _policy("policy_vocabulary", 2047, 32000, "bf16", kl=0.02),
        # log-probabilities of the labels of a ragged stereo image
        _logp("logp_stereo", 283 * 411, 70),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: single rows to frames, few columns to vocabularies, each type and direction."""
    while True:
        op = rng.choice(["norm", "norm", "bucket", "bucket", "policy", "policy", "logp"])
        x = rng.choice(["f32", "f32", "bf16", "f16"])
        if op == "norm":
            C = rng.choice([_log_int(rng, 5, 256), _log_int(rng, 5, 256), _log_int(rng, 200, 9000)])
            c = _norm("", _log_int(rng, 1, 1.2e8 / C), C, x, rng.choice([x, "f32"]), rng.random() < 0.7, rng.random() < 0.8)
        elif op == "bucket":
            kind = rng.choice(["table", "edges", "edges", "heads", "row"])
            if kind == "table":
                L = _log_int(rng, 16, 256)
                c = _bucket("", 1, L, L, rng.randint(4, 64), max(8, L // 2))
            elif kind == "edges":
                L = rng.randint(5, 64)
                c = _bucket("", _log_int(rng, 100, 1.0e8 / (L * L)), L, L, rng.randint(4, 40), max(4, L - 1), rng.choice(["f32", "f32", x]))
            else:
                K = _log_int(rng, 64, 5000)
                Q = 1 if kind == "row" else _log_int(rng, 16, 3000)
                c = _bucket("", rng.randint(1, 32), Q, K, rng.choice([16, 32, 64]), rng.choice([64, 128, 300]), x, kind == "heads",
                            max(K - Q, 0), rng.random() < 0.5)
        else:
            L = rng.choice([_log_int(rng, 5, 256), _log_int(rng, 5, 256), _log_int(rng, 300, 50000)])
            N = _log_int(rng, 1, 1.0e8 / L)
            if op == "logp":
                c = _logp("", N, L, x)
            else:
                c = _policy("", N, L, x, rng.choice([1, 1, max(1, N // 4)]), rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.2,
                            rng.choice([0.0, 0.01, 0.04]))
        del c["name"]
        if work(c)["bytes"] <= LARGEST:
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
    randn = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    rand = lambda *shape: torch.rand(shape, generator=gen, device=dev)  # noqa: E731
    empty = lambda shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
    s = {"case": case}
    if case["op"] == "norm":
        N, C = case["N"], case["C"]
        # scores: classes have a level of their own, pixels a contrast
        x = (randn(N, C).mul_(2.0).add_(randn(C))).mul_(0.5 + rand(N, 1)).to(TYPES[case["x"]])
        s.update(x=x, gamma=1.0 + 0.2 * randn(C) if case["affine"] else None, beta=0.2 * randn(C) if case["affine"] else None,
                 y=empty((N, C), TYPES[case["y"]]))
        if case["step"]:
            s.update(grad_y=randn(N, C).to(TYPES[case["y"]]), mean=empty((N,)), rstd=empty((N,)), grad_x=torch.empty_like(x),
                     grad_gamma=empty((C,)) if case["affine"] else None, grad_beta=empty((C,)) if case["affine"] else None)
        return s
    if case["op"] == "bucket":
        G, Q, K, NB = (case[k] for k in ("G", "Q", "K", "NB"))
        shape = (NB, G) if case["heads_last"] else (G, NB)
        first = -(Q - 1) - case["offset"]
        s.update(table=randn(*shape), first=first, out=empty((G, Q, K), TYPES[case["x"]]),
                 bucket_of=torch.from_numpy(_buckets(NB, case["far"], first, Q + K - 1)).to(dev))
        if case["step"]:
            s.update(grad_out=randn(G, Q, K).to(TYPES[case["x"]]), grad_table=empty(shape))
        return s
    N, L = case["N"], case["L"]
    cost = randn(N, L).mul_(2.0).to(TYPES[case["x"]])
    # the labels are drawn from the distribution (Gumbel's maximum)
    labels = (-cost.float() - torch.log(-torch.log(rand(N, L).clamp_(1e-7, 1.0 - 1e-6)))).argmax(1)
    s.update(labels=labels.to(torch.uint8 if L <= 256 else torch.int32), logp=empty((N,)), cost=cost)
    if case["op"] == "logp":
        return s
    if case["barred"]:
        barred = rand(N, L) < 0.05
        barred[torch.arange(N, device=dev), labels] = False
        cost.masked_fill_(barred, float("inf"))
        del barred
    lp = _logp64(cost, labels)
    # the parameters have moved since the labels were drawn: log ratios of a few tenths.  None lies so near a bound of the clipping (where
    # the gradient jumps) that single precision could not tell its side
    delta = 0.2 * randn(N).double()
    for edge in (math.log(1.0 - CLIP_LOW), math.log(1.0 + CLIP_HIGH)):
        delta = torch.where((delta - edge).abs() < 1e-3, delta + 4e-3, delta)
    s.update(old_logp=None if case["on_policy"] else (lp - delta).float(), ref_logp=(lp + 0.3 * randn(N)).float() if case["kl"] > 0 else None,
             # rewards above a baseline that lags behind
             advantage=randn(-(-N // case["per"])) + 0.5, mask=None, loss=empty((3,)), grad_cost=torch.empty_like(cost))
    if case["mask"]:
        s["mask"] = (rand(N) < 0.9).to(torch.uint8)
        cost[(s["mask"] == 0) & (rand(N) < 0.5)] = float("nan")
    return s


def _logp64(cost, labels):
    """Log-probabilities of the labels in 64 bits, a few million costs at a time."""
    rows = max(1, (1 << 24) // cost.shape[1])
    out = []
    for a in range(0, cost.shape[0], rows):
        z = -cost[a:a + rows].double()
        out.append(z.gather(1, labels[a:a + rows].long()[:, None])[:, 0] - torch.logsumexp(z, 1))
    return torch.cat(out)


# ---- the plain forms

def _plain_norm(s):
    case = s["case"]
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    h = xc * rstd
    y = h * s["gamma"] + s["beta"] if case["affine"] else h
    out = {"y": y.to(TYPES[case["y"]])}
    if case["step"]:
        dy = s["grad_y"].float()
        a = dy * s["gamma"] if case["affine"] else dy
        dx = rstd * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
        out["grad_x"] = dx.to(TYPES[case["x"]])
        if case["affine"]:
            out.update(grad_gamma=(dy * h).sum(0), grad_beta=dy.sum(0))
    return out


def _plain_bucket(s):
    case = s["case"]
    G, Q, K, NB = (case[k] for k in ("G", "Q", "K", "NB"))
    dev = s["table"].device
    bucket = s["bucket_of"].long()
    where = bucket[torch.arange(K, device=dev)[None, :] - torch.arange(Q, device=dev)[:, None] - case["offset"] - s["first"]]
    table = s["table"].t() if case["heads_last"] else s["table"]
    out = {"out": table.to(TYPES[case["x"]])[:, where.reshape(-1)].view(G, Q, K)}
    if case["step"]:
        # rows of Q + K - 1 values, read as rows that are one longer: a column is a diagonal
        g = torch.nn.functional.pad(s["grad_out"].float(), (Q - 1, 0)).view(G, -1)
        g = torch.nn.functional.pad(g, (0, Q)).view(G, Q, Q + K)
        diagonals = g.sum(1)[:, :Q + K - 1]
        select = (bucket[:, None] == torch.arange(NB, device=dev)[None, :]).float()
        grad = diagonals @ select
        out["grad_table"] = grad.t().contiguous() if case["heads_last"] else grad
    return out


def _plain_policy(s):
    case = s["case"]
    z = -s["cost"].float()
    counts = torch.ones(case["N"], dtype=torch.bool, device=z.device) if s["mask"] is None else s["mask"] != 0
    z = torch.where(counts[:, None], z, torch.zeros((), device=z.device))
    at = s["labels"].long()[:, None]
    e = z - z.amax(1, keepdim=True)
    w = torch.exp(e)
    total = w.sum(1, keepdim=True)
    lp = (e.gather(1, at) - torch.log(total))[:, 0]
    A = s["advantage"].repeat_interleave(case["per"])[:case["N"]]
    ratio = torch.ones_like(lp) if s["old_logp"] is None else torch.exp(lp - s["old_logp"])
    free, clipped = ratio * A, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * A
    gain = torch.minimum(free, clipped)
    slope = -torch.where(free <= clipped, free, torch.zeros_like(free))
    kl = torch.zeros_like(lp)
    if s["ref_logp"] is not None:
        d = s["ref_logp"] - lp
        kl = torch.expm1(d) - d
        slope = slope - case["kl"] * torch.expm1(d)
    n = counts.sum().clamp(min=1).float()
    zero = torch.zeros_like(lp)
    gain, kl, slope = torch.where(counts, gain, zero), torch.where(counts, kl, zero), torch.where(counts, slope, zero)
    surrogate, divergence = -gain.sum() / n, kl.sum() / n
    grad = w / total
    grad.scatter_add_(1, at, torch.full_like(lp, -1.0)[:, None])
    grad = grad * (slope / n * case["scale"])[:, None]
    return {"loss": torch.stack([surrogate + case["kl"] * divergence, surrogate, divergence]), "logp": torch.where(counts, lp, zero),
            "grad_cost": grad.to(s["cost"].dtype)}


def _plain_logp(s):
    z = -s["cost"].float()
    e = z - z.amax(1, keepdim=True)
    return {"logp": (e.gather(1, s["labels"].long()[:, None]) - torch.log(torch.exp(e).sum(1, keepdim=True)))[:, 0]}


# ---- the library's entry points

def _workspace(s, nbytes):
    """The scratch that a program keeps beside its buffers: allocated once."""
    if "workspace" not in s:
        s["workspace"] = torch.empty((nbytes(),), dtype=torch.uint8, device="cuda:0")
    return s["workspace"]


def _own(s):
    import paper_1910_10892_amd as mrf
    case = s["case"]
    if case["op"] == "norm":
        if not case["step"]:
            mrf.mrf_layer_norm_forward(s["x"], s["gamma"], s["beta"], EPS, s["y"], None, None)
            return {"y": s["y"]}
        ws = _workspace(s, lambda: mrf.mrf_layer_norm_workspace_bytes(case["N"], case["C"]))
        mrf.mrf_layer_norm_forward(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
        mrf.mrf_layer_norm_backward(s["grad_y"], s["x"], s["gamma"], s["mean"], s["rstd"], s["grad_x"], s["grad_gamma"], s["grad_beta"], ws)
        out = {"y": s["y"], "grad_x": s["grad_x"]}
        if case["affine"]:
            out.update(grad_gamma=s["grad_gamma"], grad_beta=s["grad_beta"])
        return out
    if case["op"] == "bucket":
        mrf.mrf_bucket_pairwise_forward(s["table"], s["bucket_of"], s["first"], s["out"], query_offset=case["offset"],
                                        heads_last=case["heads_last"])
        if not case["step"]:
            return {"out": s["out"]}
        ws = _workspace(s, lambda: mrf.mrf_bucket_pairwise_workspace_bytes(case["G"], case["Q"], case["K"], case["NB"]))
        mrf.mrf_bucket_pairwise_backward(s["grad_out"], s["bucket_of"], s["first"], s["grad_table"], ws, query_offset=case["offset"],
                                         heads_last=case["heads_last"])
        return {"out": s["out"], "grad_table": s["grad_table"]}
    if case["op"] == "logp":
        mrf.mrf_softmin_logp(s["cost"], s["labels"], s["logp"])
        return {"logp": s["logp"]}
    ws = _workspace(s, mrf.mrf_softmin_policy_workspace_bytes)
    mrf.mrf_softmin_policy(s["cost"], s["labels"], s["advantage"], s["old_logp"], s["ref_logp"], s["mask"], CLIP_LOW, CLIP_HIGH, case["kl"],
                           s["loss"], s["logp"], s["grad_cost"], ws, pixels_per_advantage=case["per"], grad_scale=case["scale"])
    return {"loss": s["loss"], "logp": s["logp"], "grad_cost": s["grad_cost"]}


def run(s):
    if own:
        return _own(s)
    return {"norm": _plain_norm, "bucket": _plain_bucket, "policy": _plain_policy, "logp": _plain_logp}[s["case"]["op"]](s)


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        N, C = case["N"], case["C"]
        rows, y, dx = max(1, (1 << 24) // C), [], []
        gamma = s["gamma"].double() if case["affine"] else torch.ones(C, dtype=torch.float64, device=s["x"].device)
        beta = s["beta"].double() if case["affine"] else torch.zeros_like(gamma)
        dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(gamma)
        for a in range(0, N, rows):
            x = s["x"][a:a + rows].double()
            mu = x.sum(1) / C
            sd = torch.sqrt(((x - mu[:, None]) ** 2).sum(1) / C + EPS)
            h = (x - mu[:, None]) / sd[:, None]
            y.append(torch.addcmul(beta, h, gamma))
            if case["step"]:
                dy = s["grad_y"][a:a + rows].double()
                dh = dy * gamma
                # through the standard deviation and the mean, one after the other
                dsd = -(dh * h).sum(1) / sd
                dxc = dh / sd[:, None] + (dsd / (C * sd))[:, None] * (x - mu[:, None])
                dx.append(dxc - dxc.sum(1, keepdim=True) / C)
                dgamma += (dy * h).sum(0)
                dbeta += dy.sum(0)
        out = {"y": torch.cat(y)}
        if case["step"]:
            out["grad_x"] = torch.cat(dx)
            if case["affine"]:
                out.update(grad_gamma=dgamma, grad_beta=dbeta)
        return out
    if case["op"] == "bucket":
        G, Q, K, NB = (case[k] for k in ("G", "Q", "K", "NB"))
        table = (s["table"].t() if case["heads_last"] else s["table"]).double()
        # entry (q, k) has the offset k - q - offset
        at = (np.arange(K)[None, :] - np.arange(Q)[:, None] - case["offset"]) - s["first"]
        which = s["bucket_of"].cpu().numpy()[at]
        out = torch.empty((G, Q, K), dtype=torch.float64, device=table.device)
        grad = torch.zeros((G, NB), dtype=torch.float64, device=table.device)
        rows = max(1, (1 << 25) // (Q * K))
        for b in range(NB):
            mine = torch.from_numpy(np.flatnonzero(which == b)).to(table.device)
            if mine.numel() == 0:
                continue
            out.view(G, Q * K)[:, mine] = table[:, b:b + 1]
            for a in range(0, G, rows) if case["step"] else ():
                grad[a:a + rows, b] = s["grad_out"][a:a + rows].view(-1, Q * K)[:, mine].double().sum(1)
        if not case["step"]:
            return {"out": out}
        return {"out": out, "grad_table": grad.t().contiguous() if case["heads_last"] else grad}
    if case["op"] == "logp":
        return {"logp": _logp64(s["cost"], s["labels"])}
    N, L = case["N"], case["L"]
    dev = s["cost"].device
    counted = torch.arange(N, device=dev) if s["mask"] is None else torch.nonzero(s["mask"])[:, 0]
    n = max(int(counted.numel()), 1)
    logp = torch.zeros(N, dtype=torch.float64, device=dev)
    grad = torch.zeros((N, L), dtype=torch.float64, device=dev)
    gains = divergence = 0.0
    rows = max(1, (1 << 24) // L)
    for a in range(0, counted.numel(), rows):
        i = counted[a:a + rows]
        lab = s["labels"][i].long()
        lp_all = torch.log_softmax(-s["cost"][i].double(), 1)
        lp = lp_all[torch.arange(i.numel(), device=dev), lab]
        A = s["advantage"][i // case["per"]].double()
        ratio = torch.ones_like(lp) if s["old_logp"] is None else torch.exp(lp - s["old_logp"][i].double())
        # the clipped side holds where it is the smaller one: a rise beyond the upper bound, a fall below the lower one
        held = ((A > 0) & (ratio > 1.0 + CLIP_HIGH)) | ((A < 0) & (ratio < 1.0 - CLIP_LOW))
        bound = torch.where(A > 0, torch.full_like(A, 1.0 + CLIP_HIGH), torch.full_like(A, 1.0 - CLIP_LOW))
        gains += float((torch.where(held, bound, ratio) * A).sum())
        slope = torch.where(held, torch.zeros_like(A), -ratio * A)
        if s["ref_logp"] is not None:
            d = s["ref_logp"][i].double() - lp
            divergence += float((torch.expm1(d) - d).sum())
            slope = slope + case["kl"] * (1.0 - torch.exp(d))
        # d lp / d c = f - [label]
        slope = slope * case["scale"] / n
        row = torch.exp(lp_all) * slope[:, None]
        row[torch.arange(i.numel(), device=dev), lab] -= slope
        grad[i] = row
        logp[i] = lp
    return {"loss": torch.tensor([-gains / n + case["kl"] * divergence / n, -gains / n, divergence / n], dtype=torch.float64), "logp": logp,
            "grad_cost": grad}


def work(case):
    """Inputs read once, outputs written once; operations of an element: norm 8 forward and 14 backward, bucket one addition backward,
    SoftMin 6 (minimum, difference, exponential, sum) and 3 for the gradient."""
    if case["op"] == "norm":
        n, x, y = case["N"] * case["C"], BYTES[case["x"]], BYTES[case["y"]]
        params = 8 * case["C"] if case["affine"] else 0
        if not case["step"]:
            return {"bytes": n * (x + y) + params, "flops": 8 * n}
        return {"bytes": n * (2 * x + 2 * y) + 2 * params, "flops": 22 * n}
    if case["op"] == "bucket":
        n, table = case["G"] * case["Q"] * case["K"], 4 * case["G"] * case["NB"]
        once = n * BYTES[case["x"]] + table
        return {"bytes": once * (2 if case["step"] else 1) + 4 * (case["Q"] + case["K"] - 1), "flops": n if case["step"] else 0}
    n, label = case["N"] * case["L"], 1 if case["L"] <= 256 else 4
    if case["op"] == "logp":
        return {"bytes": n * BYTES[case["x"]] + case["N"] * (label + 4), "flops": 6 * n}
    extra = label + 4 + (0 if case["on_policy"] else 4) + (4 if case["kl"] > 0 else 0) + (1 if case["mask"] else 0)
    return {"bytes": 2 * n * BYTES[case["x"]] + case["N"] * extra + 4 * -(-case["N"] // case["per"]) + 12, "flops": 9 * n}
