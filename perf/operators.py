"""The token operators' workloads: words into vectors, vocabulary logits into answers and losses.

A case is one call of one operator (``op``):

* ``embed``: ``n`` token ids look up rows of a ``vocab`` x ``dim`` table of type ``dtype``, times a scale, as ``out``;
* ``embed_grad``: the table's gradient (type ``out``) from ``n`` output gradients (type ``dtype``);
* ``logprobs``: ``n`` rows of logits: the given token's log probability, the entropy and the ``top`` alternatives;
* ``logprobs_grad``: the logits' gradient from those of the log probabilities and entropies;
* ``distill``: loss and logits' gradient against the ``top`` logits of a teacher.

``mask``: a part of the vocabulary is masked out with -inf row by row, and every eighth row has no token (-1) or weight.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
SCALE = 0.5          # of the embedding
ZIPF_SHIFT = 10.0    # token v is drawn with weight 1 / (v + ZIPF_SHIFT)
LEFT_OUT = 8         # with a mask, one row in so many has no token


def listed():
    return [
        # a tagger over a handful of short sentences, the smallest call of an encoder's input
        {"name": "embed_112", "op": "embed", "n": 112, "vocab": 8192, "dim": 64, "dtype": "f32", "out": "f32"},
        # the leaves of a large mini-batch of trees, 32-bit master table, 16-bit inputs
        {"name": "embed_28629", "op": "embed", "n": 28629, "vocab": 65536, "dim": 512, "dtype": "f32", "out": "bf16"},
        # a training step over a small mini-batch of lattices: odd rows of 100, a 32-bit gradient
        {"name": "embed_grad_1627", "op": "embed_grad", "n": 1627, "vocab": 20011, "dim": 100, "dtype": "f32", "out": "f32"},
        # the same for the largest mini-batch: frequent words have thousands of rows each
        {"name": "embed_grad_262144", "op": "embed_grad", "n": 262144, "vocab": 131072, "dim": 512, "dtype": "bf16",
         "out": "f32"},
        # serving: one new token's answer, with its alternatives
        {"name": "logprobs_1", "op": "logprobs", "n": 1, "vocab": 131072, "dtype": "bf16", "top": 8, "temp": 1.0,
         "mask": False},
        # serving a batch of requests under constrained decoding, a vocabulary of an odd size, sharpened
        {"name": "logprobs_63_mask", "op": "logprobs", "n": 63, "vocab": 32003, "dtype": "bf16", "top": 20, "temp": 0.7,
         "mask": True},
        # scoring long given texts, with a few alternatives each
        {"name": "logprobs_8192", "op": "logprobs", "n": 8192, "vocab": 65536, "dtype": "bf16", "top": 5, "temp": 1.0,
         "mask": False},
        # a small policy step in 32 bits, constrained
        {"name": "logprobs_grad_300_mask", "op": "logprobs_grad", "n": 300, "vocab": 10007, "dtype": "f32", "temp": 1.3,
         "mask": True},
        # the largest policy step
        {"name": "logprobs_grad_8192", "op": "logprobs_grad", "n": 8192, "vocab": 65536, "dtype": "bf16", "temp": 1.0,
         "mask": False},
        # distilling a tagger's small vocabulary in 32 bits
        {"name": "distill_128", "op": "distill", "n": 128, "vocab": 8192, "dtype": "f32", "top": 16, "temp": 2.0,
         "mask": False},
        # a mini-batch of padded texts, vocabulary of an odd size
        {"name": "distill_1000_mask", "op": "distill", "n": 1000, "vocab": 50021, "dtype": "bf16", "top": 32, "temp": 1.0,
         "mask": True},
        # the largest vocabulary
        {"name": "distill_4096", "op": "distill", "n": 4096, "vocab": 131072, "dtype": "bf16", "top": 64, "temp": 2.0,
         "mask": False},
    ]


def draw(rng):
    """Any operator, from one row to the listed cases' largest products, in either type."""
    def between(lo, hi):
        return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))

    op = rng.choice(["embed", "embed_grad", "logprobs", "logprobs_grad", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    vocab = between(1000, 131072)
    if op in ("embed", "embed_grad"):
        dim = between(32, 512)
        return {"op": op, "n": between(1, 262144), "vocab": vocab, "dim": dim if rng.random() < 0.5 else -(-dim // 8) * 8,
                "dtype": dtype, "out": rng.choice(["f32", "bf16"])}
    rows = (1 << 30) // (vocab * BYTES[dtype])      # a gigabyte of logits, as the largest listed cases have
    case = {"op": op, "n": between(1, min(rows, 8192)), "vocab": vocab, "dtype": dtype, "temp": rng.choice([0.7, 1.0, 2.0]),
            "mask": rng.random() < 0.5}
    if op != "logprobs_grad":
        case["top"] = between(4, 128) if op == "distill" else between(1, 64) - 1
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------


def _ids(case, g, dev, n):
    weight = 1.0 / (torch.arange(case["vocab"], device=dev, dtype=torch.float64) + ZIPF_SHIFT)
    edges = weight.cumsum(0)
    u = torch.rand(n, generator=g, device=dev, dtype=torch.float64) * edges[-1]
    return torch.searchsorted(edges, u).clamp_(max=case["vocab"] - 1).to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    op, n, V = case["op"], case["n"], case["vocab"]
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = {"case": dict(case)}
    if op in ("embed", "embed_grad"):
        s["ids"] = _ids(case, g, dev, n)
        rows = V if op == "embed" else n
        s["table" if op == "embed" else "dout"] = normal(rows, case["dim"]).to(dtype)
        return s
    # logits of a trained model: a wide bulk, a few tokens well above it, the given one often among them
    s["ids"] = _ids(case, g, dev, n)
    x = torch.randn((n, V), generator=g, device=dev, dtype=dtype).mul_(2.5)
    high = torch.randint(0, V, (n, 4), generator=g, device=dev)
    high[:, 0] = torch.where(torch.rand(n, generator=g, device=dev) < 0.7, s["ids"].long(), high[:, 0])
    x.scatter_(1, high, (9.0 + 3.0 * normal(n, 4)).to(dtype))
    if case["mask"]:
        x.masked_fill_(torch.rand((n, V), generator=g, device=dev, dtype=dtype) < 0.3, -math.inf)
        s["ids"][LEFT_OUT - 1::LEFT_OUT] = -1
    s["logits"] = x
    if op == "logprobs_grad":
        # what the forward call has left, and the gradients that the loss of its results gives
        s["stats"], s["entropy"] = _row_stats(x, s["ids"], case["temp"])
        s["g_logprob"] = normal(n)
        s["g_entropy"] = 0.01 * normal(n)
    if op == "distill":
        # a teacher's best tokens: distinct ids, falling logits; one list in four is shorter (cut at a probability)
        K = case["top"]
        start = torch.randint(0, V, (n, 1), generator=g, device=dev)
        step = torch.randint(1, V // K + 1, (n, 1), generator=g, device=dev)
        k = torch.arange(K, device=dev)
        ids = (start + k * step) % V
        short = torch.rand((n, 1), generator=g, device=dev) < 0.25
        keep = torch.randint(1, K + 1, (n, 1), generator=g, device=dev)
        s["top_ids"] = torch.where(short & (k >= keep), -1, ids).to(torch.int32)
        # the student is on its way there, and a mask holds for both
        x.scatter_(1, ids, (4.0 + 2.5 * normal(n, K)).to(dtype))
        s["top_logits"] = 12.0 - torch.empty((n, K), device=dev).exponential_(generator=g).mul_(0.5).cumsum(1)
        s["weight"] = (0.5 + torch.rand(n, generator=g, device=dev)) / n
        if case["mask"]:
            s["weight"][LEFT_OUT - 1::LEFT_OUT] = 0.0
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"embed": _embed, "embed_grad": _embed_grad, "logprobs": _logprobs, "logprobs_grad": _logprobs_grad,
            "distill": _distill}[case["op"]](state, case)


def _own(s, case):
    from paper_2302_03851_amd import tokens
    op = case["op"]
    if op == "embed":
        s["out"] = tokens.embed(s["ids"], s["table"], SCALE, dtype=DTYPES[case["out"]], out=s.get("out"))
        return {"out": s["out"]}
    if op == "embed_grad":
        s["out"] = tokens.embed_grad(s["ids"], s["dout"], case["vocab"], SCALE, dtype=DTYPES[case["out"]], out=s.get("out"))
        return {"dtable": s["out"]}
    if op == "logprobs":
        r = s["out"] = tokens.logprobs(s["logits"], s["ids"], case["temp"], case["top"], out=s.get("out"))
        return {"logprob": r.logprob, "entropy": r.entropy, "stats": r.stats, "top_ids": r.top_ids,
                "top_logprobs": r.top_logprobs}
    if op == "logprobs_grad":
        s["out"] = tokens.logprobs_grad(s["logits"], s["ids"], s["stats"], s["entropy"], s["g_logprob"], s["g_entropy"],
                                        case["temp"], out=s.get("out"))
        return {"dlogits": s["out"]}
    r = s["out"] = tokens.distill(s["logits"], s["top_ids"], s["top_logits"], case["temp"], s["weight"], out=s.get("out"))
    return {"loss": r.loss, "dlogits": r.dlogits}


# ---- the plain forms: 32 bits throughout, rounded once at the end ------------------------------------------------


def _embed(s, case):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < case["vocab"])
    rows = s["table"][torch.where(there, ids, 0)].float()
    return {"out": torch.where(there[:, None], rows * SCALE, 0.0).to(DTYPES[case["out"]])}


def _embed_grad(s, case):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < case["vocab"])
    d = torch.zeros((case["vocab"] + 1, case["dim"]), device=ids.device)
    d.index_add_(0, torch.where(there, ids, case["vocab"]), s["dout"].float())
    return {"dtable": (d[:-1] * SCALE).to(DTYPES[case["out"]])}


def _shifted(x, temp):
    """Row maxima (n, 1), (x - max) / temp, its exponentials and their sums."""
    top = x.amax(1, keepdim=True)
    y = (x - torch.where(top == -math.inf, 0.0, top)) / temp
    e = torch.exp(y)
    return top, y, e, e.sum(1, keepdim=True)


def _row_stats(x, ids, temp):
    """What the forward call leaves for the gradient: each row's maximum and ln sum exp((x - max) / temp), and its entropy."""
    top, y, e, total = _shifted(x.float(), temp)
    empty = total == 0
    log_total = torch.where(empty, 0.0, torch.log(total))
    p = e / torch.where(empty, 1.0, total)
    entropy = -torch.where(p > 0, p * (y - log_total), 0.0).sum(1)
    none = (ids < 0) | (ids >= x.shape[1])
    stats = torch.where(none[:, None], 0.0, torch.cat([top, log_total], 1))
    return stats, torch.where(none, 0.0, entropy)


def _logprobs(s, case):
    x, ids, K, V = s["logits"].float(), s["ids"].long(), case["top"], case["vocab"]
    none = (ids < 0) | (ids >= V)
    top, y, e, total = _shifted(x, case["temp"])
    empty = total == 0
    log_total = torch.where(empty, 0.0, torch.log(total))
    p = e / torch.where(empty, 1.0, total)
    lp = torch.where(empty, -math.inf, y - log_total)
    del e
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    del p
    given = lp.gather(1, torch.where(none, 0, ids)[:, None])[:, 0]
    # the largest logits, the lowest index first among equals: order by (value, -index) as whole numbers
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * 2**32 + (2**32 - 1 - torch.arange(V, device=x.device))
    low = -2**63
    key = torch.where((x > -math.inf) & ~none[:, None], key, low)
    key = torch.topk(key, min(K, V), dim=1).values
    at = torch.where(key == low, -1, (2**32 - 1) - (key & (2**32 - 1)))
    best = torch.where(at < 0, -math.inf, lp.gather(1, at.clamp(min=0)))
    return {"logprob": torch.where(none, 0.0, given), "entropy": torch.where(none, 0.0, entropy),
            "stats": torch.where(none[:, None], 0.0, torch.cat([top, log_total], 1)),
            "top_ids": at.to(torch.int32), "top_logprobs": best}


def _logprobs_grad(s, case):
    x, ids = s["logits"].float(), s["ids"].long()
    top, log_total = s["stats"][:, :1], s["stats"][:, 1:]
    out = ((ids < 0) | (ids >= case["vocab"]) | ((s["g_logprob"] == 0) & (s["g_entropy"] == 0)))[:, None] | (top == -math.inf)
    lp = (x - torch.where(out, 0.0, top)) / case["temp"] - log_total
    p = torch.exp(lp)
    d = -p * s["g_logprob"][:, None]
    d -= torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0) * s["g_entropy"][:, None]
    d.scatter_add_(1, torch.where(out[:, 0], 0, ids)[:, None], s["g_logprob"][:, None])
    return {"dlogits": torch.where(out, 0.0, d / case["temp"]).to(s["logits"].dtype)}


def _distill(s, case):
    x, V, temp = s["logits"].float(), case["vocab"], case["temp"]
    ids = s["top_ids"].long()
    there = (ids >= 0) & (ids < V)
    t = torch.where(there, s["top_logits"].float(), -math.inf)
    _, _, te, ttotal = _shifted(t, temp)
    out = (s["weight"][:, None] == 0) | (ttotal == 0)
    q = torch.zeros_like(x).scatter_add_(1, torch.where(there, ids, 0), te / torch.where(ttotal == 0, 1.0, ttotal))
    _, y, e, total = _shifted(x, temp)
    empty = total == 0
    lp = torch.where(empty, -math.inf, y - torch.log(total))
    p = e / torch.where(empty, 1.0, total)
    loss = temp * temp * torch.where(q > 0, q * (torch.log(q) - lp), 0.0).sum(1)
    d = s["weight"][:, None] * temp * (p - q)
    return {"loss": torch.where(out[:, 0], 0.0, loss), "dlogits": torch.where(out | empty, 0.0, d).to(s["logits"].dtype)}


# ---- what a pass cannot do without -------------------------------------------------------------------------------


def _distinct(case):
    """Expected number of different words among n drawn ones."""
    w = 1.0 / (np.arange(case["vocab"]) + ZIPF_SHIFT)
    return float(-np.expm1(case["n"] * np.log1p(-w / w.sum())).sum())


def work(case):
    op, n, V = case["op"], case["n"], case["vocab"]
    if op == "embed":
        row = case["dim"]
        return {"bytes": 4 * n + _distinct(case) * row * BYTES[case["dtype"]] + n * row * BYTES[case["out"]],
                "flops": float(n * row)}
    if op == "embed_grad":
        row = case["dim"]
        return {"bytes": 4 * n + n * row * BYTES[case["dtype"]] + V * row * BYTES[case["out"]], "flops": float(n * row)}
    read = n - (n // LEFT_OUT if case["mask"] else 0)    # rows without a token or a weight need not be read
    logits = V * BYTES[case["dtype"]]
    if op == "logprobs":                                 # difference, factor, exponential and two sums a logit
        return {"bytes": read * logits + n * (4 + 16 + 8 * case["top"]), "flops": 6.0 * read * V}
    if op == "logprobs_grad":
        return {"bytes": (read + n) * logits + n * (4 + 12 + 8), "flops": 8.0 * read * V}
    return {"bytes": (read + n) * logits + n * (8 * case["top"] + 8), "flops": 7.0 * read * V}


# ---- the definitions in 64 bits, a block of rows at a time -------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    op, V = case["op"], case["vocab"]
    ids = s["ids"].long()
    if op == "embed":
        out = torch.zeros((case["n"], case["dim"]), dtype=torch.float64, device=ids.device)
        out[ids >= 0] = s["table"].double().index_select(0, ids[ids >= 0]) * SCALE
        return {"out": out}
    if op == "embed_grad":
        out = torch.zeros((V, case["dim"]), dtype=torch.float64, device=ids.device)
        order = torch.argsort(ids[ids >= 0], stable=True)
        rows = torch.nonzero(ids >= 0)[:, 0][order]
        word, count = torch.unique_consecutive(ids[rows], return_counts=True)
        out[word] = torch.segment_reduce(s["dout"][rows].double(), "sum", lengths=count) * SCALE
        return {"dtable": out}
    block = max(1, (1 << 27) // V)
    parts = [_exact_rows({k: v[a:a + block] if torch.is_tensor(v) else v for k, v in s.items()}, case)
             for a in range(0, case["n"], block)]
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_rows(s, case):
    op, V, T = case["op"], case["vocab"], case["temp"]
    x, ids = s["logits"].double(), s["ids"].long()
    n = x.shape[0]
    row = torch.arange(n, device=x.device)
    lp = torch.log_softmax(x / T, 1)                     # no row of these inputs is masked out whole
    if op == "logprobs":
        live = ids >= 0
        entropy = torch.special.entr(lp.exp()).sum(1) * live
        top = x.amax(1)
        stats = torch.stack([top, torch.logsumexp(x / T, 1) - top / T], 1) * live[:, None]
        best = torch.topk(lp, case["top"], dim=1).values
        best[~live] = -math.inf
        given = lp[row, ids.clamp(min=0)]
        given[~live] = 0.0
        return {"logprob": given, "entropy": entropy, "stats": stats, "top_ids": None, "top_logprobs": best}
    p = lp.exp()
    if op == "logprobs_grad":
        live = ids >= 0
        entropy = torch.special.entr(p).sum(1)
        one = torch.zeros_like(p)
        one[row, ids.clamp(min=0)] = 1.0
        d = s["g_logprob"].double()[:, None] * (one - p)
        d -= s["g_entropy"].double()[:, None] * (p * entropy[:, None] - torch.special.entr(p))
        return {"dlogits": d * live[:, None] / T}
    listed = s["top_ids"].long()
    q = torch.softmax(s["top_logits"].double().masked_fill(listed < 0, -math.inf) / T, 1)
    at = listed.clamp(min=0)
    live = s["weight"] != 0
    # entries with q = 0 are left out; the ids of a row differ
    each = torch.where(q > 0, q * (q.log() - lp.gather(1, at)), 0.0)
    d = p.scatter_add(1, at, -q) * (s["weight"].double()[:, None] * T)
    return {"loss": torch.where(live, T * T * each.sum(1), 0.0), "dlogits": d * live[:, None]}
