"""The operators on rows of class scores: what a classifier answers with, and what a student of
its answers is trained on.

  votes    a forest's answers in full: how many of its trees vote for each class
  top      the k best classes of each row of scores, with the row's log-sum-exp
  sample   a class drawn from each row by temperature, top-k, top-p and min-p
  distill  the loss of a student against a teacher's top scores, and the student's gradient

Scores are float32, float16 or bfloat16, or uint8 votes, whose score is ln(votes).  A score
of NaN is taken as -inf by `top` and `sample`; a row in which no score is above -inf is empty.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "u8": torch.uint8}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "u8": 1}
INF = float("inf")


def _votes(n, features, classes, trees, depth, **more):
    return {"op": "votes", "n": n, "features": features, "classes": classes, "trees": trees,
            "depth": depth, **more}


def _top(n, classes, k, type, **more):
    return {"op": "top", "n": n, "classes": classes, "k": k, "type": type, **more}


def _sample(n, classes, type, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, per_row=False, **more):
    return {"op": "sample", "n": n, "classes": classes, "type": type, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "per_row": per_row, **more}


def _distill(n, classes, k, type, temperature, fused, **more):
    return {"op": "distill", "n": n, "classes": classes, "k": k, "type": type,
            "temperature": temperature, "fused": fused, **more}


def listed():
    return [
        # One 256 x 256 image of 19 attributes: the answers of a small forest, a call of a few
        # microseconds.
        _votes(65_536, 19, 7, 32, 6, name="votes_image"),
        # The forest of the framework's benchmark: 32 trees of depth 10 over 4 million records.
        _votes(4_194_304, 32, 8, 32, 10, name="votes_batch"),
        # The votes of a forest for a million records, cut to the four strongest classes.
        _top(1_000_003, 32, 4, "u8", name="top_votes"),
        # One row of an odd number of classes, as for the alternatives to a single answer: latency.
        _top(1, 50_001, 128, "f32", name="top_row"),
        # A teacher's answers written down for training: a batch of rows over a large vocabulary.
        _top(2_048, 131_072, 64, "bf16", name="top_teacher"),
        # A class drawn by each record's votes, the stray ones cut off.
        _sample(1_000_003, 32, "u8", 1.0, 0, 0.9, 0.0, name="sample_votes"),
        # A single token: latency.
        _sample(1, 131_072, "bf16", 0.8, 50, 0.95, 0.0, name="sample_token"),
        # A batch of requests, each with settings of its own.
        _sample(64, 32_768, "f16", 0.9, 40, 0.9, 0.02, True, name="sample_requests"),
        # A wide batch whose nucleus can be most of the vocabulary.
        _sample(256, 131_072, "bf16", 1.0, 0, 0.9, 0.0, name="sample_nucleus"),
        # A small student of a forest's answers: many records, few classes, a loss with autograd.
        _distill(262_144, 32, 4, "f32", 1.0, False, name="distill_votes"),
        # Odd rows in half precision, loss and gradient in one call.
        _distill(1_000, 50_001, 100, "f16", 2.0, True, name="distill_odd"),
        # A training batch over a large vocabulary: the loss, then the backward pass.
        _distill(4_096, 65_536, 64, "bf16", 2.0, False, name="distill_batch"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["votes", "top", "top", "sample", "sample", "sample", "distill", "distill"])
    if op == "votes":
        return _votes(_log(rng, 1, 1_000_000), rng.randint(1, 64), rng.randint(2, 64),
                      rng.randint(1, 64), rng.randint(1, 9))
    classes = rng.choice([_log(rng, 2, 64), _log(rng, 65, 2_048), _log(rng, 2_049, 200_000)])
    if op == "top":
        n = _log(rng, 1, min(1_000_000, (1 << 26) // classes))
        return _top(n, classes, _log(rng, 1, min(classes, 256)),
                    rng.choice(["f32", "f16", "bf16", "u8"]))
    if op == "sample":
        n = _log(rng, 1, min(1_000_000, (1 << 24) // classes))
        return _sample(n, classes, rng.choice(["f32", "f16", "bf16", "u8"]),
                       rng.choice([0.0, 1.0, round(rng.uniform(0.3, 1.5), 3)]),
                       rng.choice([0, _log(rng, 1, min(classes, 256)), _log(rng, 1, classes)]),
                       rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                       rng.choice([0.0, round(rng.uniform(0.005, 0.3), 4)]), rng.random() < 0.3)
    n = _log(rng, 1, min(500_000, (1 << 26) // classes))
    return _distill(n, classes, _log(rng, 1, min(classes, 256)),
                    rng.choice(["f32", "f16", "bf16"]), rng.choice([1.0, round(rng.uniform(0.5, 4.0), 3)]),
                    rng.random() < 0.5)


def work(case):
    n = case["n"]
    if case["op"] == "votes":
        tables = case["trees"] * 8 * (2 << case["depth"])
        return {"bytes": n * (4 * case["features"] + case["classes"]) + tables,
                "flops": n * case["trees"] * case["depth"]}
    scores, k = n * case["classes"], case.get("k", 0)
    if case["op"] == "top":      # scores in; value and index of each kept class and a sum out
        return {"bytes": scores * BYTES[case["type"]] + n * (8 * k + 4), "flops": 3 * scores}
    if case["op"] == "sample":   # scores and a random number in, a label out
        more = 16 if case["per_row"] else 0
        return {"bytes": scores * BYTES[case["type"]] + n * (8 + more), "flops": 3 * scores}
    # the student's scores in and their gradient out; teacher, row's weight and row's loss
    return {"bytes": 2 * scores * BYTES[case["type"]] + n * (8 * k + 8), "flops": 6 * scores}


# ---- inputs -----------------------------------------------------------------------------


def _scores(case, g):
    """Rows from sure to undecided; in one row of eight a third of the classes is masked."""
    n, classes = case["n"], case["classes"]
    if case["type"] == "u8":     # 32 voters, most classes without a vote
        r = torch.rand(n, classes, generator=g, device="cuda")
        return (r.pow_(6).mul_(33)).to(torch.uint8)
    x = torch.randn(n, classes, generator=g, device="cuda")
    x *= 2 + 3 * torch.rand(n, 1, generator=g, device="cuda")
    some = torch.arange(n, device="cuda")[3::8]
    if len(some):
        x[some] = x[some].masked_fill(
            torch.rand(len(some), classes, generator=g, device="cuda") < 0.3, -INF)
    return x.to(TYPES[case["type"]])


def _trees(case, seed):
    """Complete trees of one depth in level order: features, thresholds, and the leaves' classes."""
    r = np.random.RandomState(seed % (1 << 31))
    inner, leaves, t = (1 << case["depth"]) - 1, 1 << case["depth"], case["trees"]
    feature = r.randint(0, case["features"], (t, inner)).astype(np.int32)
    threshold = r.rand(t, inner).astype(np.float32)
    cls = (case["classes"] * r.rand(t, leaves) ** 2).astype(np.int32)
    return feature, threshold, cls


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    n = case["n"]
    state = {"case": case}
    if case["op"] == "votes":
        feature, threshold, cls = _trees(case, seed)
        state["x"] = torch.rand(n, case["features"], generator=g, device="cuda")
        if own:
            from paper_1111_1373_amd import dtree
            t, inner = feature.shape
            size = 2 * inner + 1
            nodes = np.zeros((t, size), dtype=dtree.NODE_DTYPE)
            nodes["feature"][:, :inner], nodes["threshold"][:, :inner] = feature, threshold
            nodes["left"][:, :inner] = 2 * np.arange(inner) + 1
            nodes["cls"][:, :inner], nodes["cls"][:, inner:] = -1, cls
            state["forest"] = dtree.Forest(nodes.reshape(-1), np.arange(t + 1) * size,
                                           case["features"], case["classes"])
        else:
            state["feature"] = torch.from_numpy(feature).long().cuda()
            state["threshold"] = torch.from_numpy(threshold).cuda()
            state["cls"] = torch.from_numpy(cls).long().cuda()
        return state
    state["x"] = x = _scores(case, g)
    if case["op"] == "sample":
        state["u"] = torch.rand(n, generator=g, device="cuda")
        for name, t in (("temperature", torch.float32), ("top_k", torch.int32),
                        ("top_p", torch.float32), ("min_p", torch.float32)):
            v = case[name]
            if case["per_row"]:      # half of the requests differ from the common setting
                r = torch.rand(n, generator=g, device="cuda")
                v = torch.where(r < 0.5, torch.full_like(r, v), r * v).to(t)
            state[name] = v
    if case["op"] == "distill":
        k = case["k"]
        teacher = x.float()
        teacher += torch.randn(teacher.shape, generator=g, device="cuda")
        values, index = torch.topk(teacher, k, dim=1)
        index = index.to(torch.int32)
        index[5::16] = -1            # padding: rows without an answer
        state["values"], state["index"] = values.contiguous(), index.contiguous()
        # the rows' weights in a mean; in half precision under a loss scale, as it is trained with
        scale = 64.0 if case["type"] == "f16" else 1.0 / n
        state["weight"] = torch.rand(n, generator=g, device="cuda") * scale
        if own and not case["fused"]:
            x.requires_grad_(True)
    return state


# ---- one pass ---------------------------------------------------------------------------


def run(state):
    case = state["case"]
    if own:
        return _own(case, state)
    return {"votes": _plain_votes, "top": _plain_top, "sample": _plain_sample,
            "distill": _plain_distill}[case["op"]](case, state)


def _own(case, s):
    from paper_1111_1373_amd import scores
    if case["op"] == "votes":
        return {"votes": s["forest"].classify(s["x"], out_kind="votes_u8")}
    if case["op"] == "top":
        values, index, lse = scores.top_scores(s["x"], case["k"])
        return {"values": values, "index": index, "lse": lse}
    if case["op"] == "sample":
        return {"labels": scores.sample(s["x"], s["u"], s["temperature"], s["top_k"], s["top_p"],
                                        s["min_p"])}
    if case["fused"]:
        loss, grad = scores.distill_grad(s["x"], s["values"], s["index"], s["weight"],
                                         case["temperature"])
    else:
        loss = scores.distill_loss(s["x"], s["values"], s["index"], case["temperature"])
        grad, = torch.autograd.grad(loss, s["x"], s["weight"])
    return {"loss": loss.detach(), "grad": grad}


def _plain_votes(case, s):
    x, feature, threshold = s["x"], s["feature"], s["threshold"]
    tree = torch.arange(case["trees"], device=x.device)
    at = torch.zeros(case["n"], case["trees"], dtype=torch.long, device=x.device)
    for _ in range(case["depth"]):
        left = torch.gather(x, 1, feature[tree, at]) < threshold[tree, at]
        at = 2 * at + 2 - left.long()
    cls = s["cls"][tree, at - ((1 << case["depth"]) - 1)]
    votes = torch.zeros(case["n"], case["classes"], dtype=torch.int32, device=x.device)
    votes.scatter_add_(1, cls, torch.ones_like(cls, dtype=torch.int32))
    return {"votes": votes.to(torch.uint8)}


def _plain_top(case, s):
    x, k = s["x"], case["k"]
    x = x.float().log() if x.dtype == torch.uint8 else x.float()
    x = torch.where(torch.isnan(x), -INF, x)
    values, index = torch.sort(x, dim=1, descending=True, stable=True)
    m = values[:, :1]
    e = torch.where(x == m, 1.0, torch.exp(x - m))
    lse = torch.where(m[:, 0] == -INF, -INF, m[:, 0] + e.sum(1).log())
    values, index = values[:, :k].contiguous(), index[:, :k].to(torch.int32)
    return {"values": values, "index": torch.where(values == -INF, -1, index), "lse": lse}


def _column(v, n, device):
    """A setting for each row: float32 as it is given, in 64 bits."""
    if isinstance(v, torch.Tensor):
        return v.double()[:, None]
    return torch.full((n, 1), v, dtype=torch.float32, device=device).double()


def _plain_sample(case, s):
    # 64 bits: the weights' sums decide between neighbours at the borders of top-p and of `u`
    x, n, classes = s["x"], case["n"], case["classes"]
    temperature, top_k, top_p, min_p = (_column(s[name], n, x.device) for name in
                                        ("temperature", "top_k", "top_p", "min_p"))
    top_k = torch.where(top_k < 1, classes, top_k)
    top_k = torch.where(temperature <= 0, 1, top_k)      # temperature 0: the best class
    v = x.double()
    score = v.log() if x.dtype == torch.uint8 else torch.where(torch.isnan(v), -INF, v)
    best, order = torch.sort(score, dim=1, descending=True, stable=True)
    m = best[:, :1]
    w = torch.where(best == m, 0.0, (best - m) / temperature).exp()
    if x.dtype == torch.uint8:                           # votes at temperature 1: whole numbers
        w = torch.where(temperature == 1, torch.gather(v, 1, order), w)
    first = w[:, :1].clone()
    rank = torch.arange(classes, device=x.device)
    w = torch.where(rank < top_k, w, 0.0)
    upto = torch.cumsum(w, 1)
    before = torch.cat([torch.zeros_like(m), upto[:, :-1]], 1)
    kept = ((before < top_p * upto[:, -1:]) | (top_p >= 1) | (rank == 0)) & (w >= min_p * first)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, 0.0))
    upto = torch.cumsum(w, 1)                            # in the classes' order
    label = (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1)
    return {"labels": torch.where(m[:, 0] == -INF, -1, label).to(torch.int32)}


def _plain_distill(case, s):
    x, index, t = s["x"], s["index"].long(), case["temperature"]
    there = (index >= 0) & (index < case["classes"])
    index = torch.where(there, index, 0)
    z = x.float() / t
    m = z.amax(1, keepdim=True)
    q = torch.exp(z - torch.where(m == -INF, 0.0, m))
    total = q.sum(1, keepdim=True)
    lse = m + total.log()
    v = torch.where(there, s["values"] / t, -INF)
    top = v.amax(1, keepdim=True)
    empty = (top == -INF) | (m == -INF)
    v = torch.where(empty, 0.0, v - top)
    logp = v - v.exp().sum(1, keepdim=True).log()
    p = torch.where(empty | ~there, 0.0, logp.exp())
    logq = torch.gather(z, 1, index) - lse
    loss = t * t * torch.where(p > 0, p * (logp - logq), 0.0).sum(1)
    grad = (q / total).scatter_add_(1, index, -p)
    grad = grad * torch.where(empty, 0.0, t * s["weight"][:, None])
    return {"loss": torch.where(empty[:, 0], 0.0, loss),
            "grad": torch.where(empty, 0.0, grad).to(x.dtype)}


# ---- the definitions in 64 bits -----------------------------------------------------------


def exact(case, seed):
    """From the definitions, on the host; None for what is whole numbers, and for cases that would
    take long."""
    if case["op"] in ("votes", "sample") or case["n"] * case["classes"] > 70_000_000:
        return None
    if case["op"] == "distill" and case["n"] * case["k"] > 3_000_000:
        return None
    s = prepare(case, seed)
    x = s["x"].detach().float().cpu().numpy().astype(np.float64)
    n, classes = x.shape
    if case["op"] == "top":
        if case["type"] == "u8":
            with np.errstate(divide="ignore"):
                x = np.log(x)
        k = case["k"]
        values = -np.sort(np.partition(-x, k - 1, axis=1)[:, :k] if k < classes else -x, axis=1)
        with np.errstate(divide="ignore", invalid="ignore"):
            lse = np.log(np.exp(x - values[:, :1]).sum(1)) + values[:, 0]
        return {"values": values, "index": None, "lse": np.where(values[:, 0] == -INF, -INF, lse)}
    t = case["temperature"]
    index, values = s["index"].cpu().numpy(), s["values"].cpu().numpy().astype(np.float64)
    weight = s["weight"].cpu().numpy().astype(np.float64)
    x /= t
    loss = np.zeros(n)
    x[x.max(1) == -INF] = 0.0        # an empty row's teacher is empty too
    x -= x.max(1, keepdims=True)
    log_z = np.log(np.exp(x).sum(1))
    grad = np.exp(x - log_z[:, None])
    for i in range(n):
        j = index[i]
        on = (j >= 0) & (values[i] > -INF)
        if not on.any():
            grad[i] = 0
            continue
        a = np.exp((values[i][on] - values[i][on].max()) / t)
        p = a / a.sum()
        p_on = p > 0
        loss[i] = t * t * np.sum(p[p_on] * (np.log(p[p_on]) - (x[i, j[on][p_on]] - log_z[i])))
        np.subtract.at(grad[i], j[on], p)
    grad *= t * weight[:, None]
    return {"loss": loss, "grad": grad}
