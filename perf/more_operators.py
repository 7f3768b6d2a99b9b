"""Workloads of the head on the cells' states and of the losses over log probabilities.

A case is one call of one operator (``op``):

* ``layer_norm``: ``n`` rows of ``dim`` values of type ``dtype``, scaled and shifted, as ``out``, with each row's mean and
  reciprocal deviation;
* ``layer_norm_grad``: the rows', the scale's and the shift's gradients;
* ``linear``: ``n`` rows of ``k`` by a ``k`` x ``m`` weight, with bias, activation ``act`` and, with ``res``, a residual;
  ``keep``: the values before the activation are a result too;
* ``linear_grad``: the rows', the weight's and the bias's gradients;
* ``preference``: the loss of ``s`` pairs of sequences over ``n`` tokens by ``kind``, and the log probabilities' gradient;
* ``policy``: the clipped policy loss of ``s`` sequences over ``n`` tokens with a KL term, and the same gradient.

``turned``: the weight is stored output by output.  ``prompts``: tokens of a sequence's first part have no id.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-5
BETA, SMOOTHING = 0.1, 0.1
LOW, HIGH, KL = 0.2, 0.28, 0.04
ACTS = ["none", "relu", "gelu", "silu", "tanh"]


def listed():
    return [
        # the states of a handful of short sentences, the smallest call
        {"name": "layer_norm_112", "op": "layer_norm", "n": 112, "dim": 64, "dtype": "f32", "out": "f32"},
        # the leaves of a large mini-batch of trees
        {"name": "layer_norm_28629", "op": "layer_norm", "n": 28629, "dim": 512, "dtype": "bf16", "out": "bf16"},
        # a training step over a small mini-batch of lattices: odd rows of 100
        {"name": "layer_norm_grad_1627", "op": "layer_norm_grad", "n": 1627, "dim": 100, "dtype": "f32", "out": "f32"},
        # the largest mini-batch
        {"name": "layer_norm_grad_262144", "op": "layer_norm_grad", "n": 262144, "dim": 512, "dtype": "bf16", "out": "bf16"},
        # serving: one new token's logits
        {"name": "linear_1", "op": "linear", "n": 1, "k": 512, "m": 131072, "dtype": "bf16", "out": "f32", "act": "none",
         "bias": True, "res": False, "keep": False, "turned": False},
        # a hidden layer over the states of a large mini-batch of trees
        {"name": "linear_28629", "op": "linear", "n": 28629, "k": 512, "m": 1536, "dtype": "bf16", "out": "bf16",
         "act": "gelu", "bias": True, "res": True, "keep": False, "turned": True},
        # a training step of a tagger over lattices in 32 bits, rows and vocabulary of odd sizes
        {"name": "linear_grad_1627", "op": "linear_grad", "n": 1627, "k": 100, "m": 20011, "dtype": "f32", "out": "f32",
         "act": "none", "turned": False},
        # the largest vocabulary product and its two gradients
        {"name": "linear_grad_8192", "op": "linear_grad", "n": 8192, "k": 512, "m": 65536, "dtype": "bf16", "out": "bf16",
         "act": "none", "turned": False},
        # a few pairs of short answers
        {"name": "preference_8", "op": "preference", "s": 8, "n": 1627, "kind": "logistic", "mean": False, "prompts": True},
        # a large mini-batch of pairs of long answers, by their mean log ratios
        {"name": "preference_1024", "op": "preference", "s": 1024, "n": 2097152, "kind": "squared", "mean": True,
         "prompts": True},
        # a small group of answers
        {"name": "policy_16", "op": "policy", "s": 16, "n": 4075, "mean": True, "prompts": False},
        # the largest step: thousands of answers, each behind its prompt
        {"name": "policy_4096", "op": "policy", "s": 4096, "n": 4194304, "mean": True, "prompts": True},
    ]


def draw(rng):
    """Any operator, from one row or pair to the listed cases' largest products, in either type."""
    def between(lo, hi):
        return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))

    op = rng.choice(["layer_norm", "layer_norm_grad", "linear", "linear_grad", "preference", "policy"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("layer_norm", "layer_norm_grad"):
        dim = between(16, 8192)
        dim = dim if rng.random() < 0.5 else -(-dim // 16) * 16
        return {"op": op, "n": between(1, min(262144, (1 << 27) // dim)), "dim": dim, "dtype": dtype,
                "out": rng.choice([dtype, "f32"])}
    if op in ("linear", "linear_grad"):
        k, m = between(32, 1024), between(64, 65536)
        if rng.random() < 0.5:
            k, m = -(-k // 32) * 32, -(-m // 64) * 64
        case = {"op": op, "n": between(1, min(65536, (1 << 36) // (k * m), (1 << 29) // m)), "k": k, "m": m, "dtype": dtype,
                "out": rng.choice([dtype, "f32"]), "act": rng.choice(ACTS), "turned": rng.random() < 0.5}
        if op == "linear":
            case["bias"], case["res"] = rng.random() < 0.75, rng.random() < 0.5
            case["keep"] = case["act"] != "none" and rng.random() < 0.5
        return case
    s = between(1, 4096)
    case = {"op": op, "s": s, "n": min(4194304, s * between(4, 2048)), "mean": rng.random() < 0.5,
            "prompts": rng.random() < 0.5}
    if op == "preference":
        case["kind"] = rng.choice(["logistic", "hinge", "squared"])
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    op, n = case["op"], case["n"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = {"case": dict(case)}
    if op in ("layer_norm", "layer_norm_grad"):
        # states of cells: each column with a middle of its own, some rows larger than others
        D, dtype = case["dim"], DTYPES[case["dtype"]]
        s["x"] = ((normal(n, D) + 0.5 * normal(D)) * (0.2 + torch.rand((n, 1), generator=g, device=dev))).to(dtype)
        s["weight"] = 1.0 + 0.1 * normal(D)
        if op == "layer_norm":
            s["bias"] = 0.1 * normal(D)
        else:
            # what the forward call has left, and the gradient that comes back
            x = s["x"].double()
            mean = x.mean(1, keepdim=True)
            var = (x - mean).square().mean(1, keepdim=True)
            s["stats"] = torch.cat([mean, torch.rsqrt(var + EPS)], 1).float()
            s["dout"] = normal(n, D).to(DTYPES[case["out"]])
        return s
    if op in ("linear", "linear_grad"):
        k, m, dtype = case["k"], case["m"], DTYPES[case["dtype"]]
        s["x"] = normal(n, k).to(dtype)
        shape = (m, k) if case["turned"] else (k, m)
        w = torch.randn(shape, generator=g, device=dev).mul_(1.5 / math.sqrt(k)).to(dtype)
        s["w"] = w.t() if case["turned"] else w
        if op == "linear":
            s["bias"] = 0.2 * normal(m) if case["bias"] else None
            s["res"] = torch.randn((n, m), generator=g, device=dev, dtype=DTYPES[case["out"]]) if case["res"] else None
        else:
            s["dout"] = torch.randn((n, m), generator=g, device=dev, dtype=DTYPES[case["out"]])
            # what the forward call has left: the values before the activation
            s["pre"] = None if case["act"] == "none" else torch.randn((n, m), generator=g, device=dev, dtype=dtype).mul_(1.5)
        return s
    # sequences of uneven lengths, some of them empty; log probabilities of likely and unlikely tokens
    seqs = case["s"] * (2 if op == "preference" else 1)
    cuts = torch.randint(0, n + 1, (seqs - 1,), generator=g, device=dev).sort().values
    ends = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), n)])
    s["first"] = ends.to(torch.int32)
    s["logprob"] = -torch.empty(n, device=dev).exponential_(generator=g).mul_(1.5)
    s["reference"] = s["logprob"] + 0.2 * normal(n)
    s["ids"] = None
    if case["prompts"]:
        at = torch.arange(n, device=dev)
        seq = torch.searchsorted(ends, at, right=True) - 1
        share = 0.6 * torch.rand(seqs, generator=g, device=dev)
        prompt = (at - ends[seq]) < share[seq] * (ends[seq + 1] - ends[seq])
        s["ids"] = torch.randint(0, 65536, (n,), generator=g, device=dev).masked_fill_(prompt, -1).to(torch.int32)
        # log probabilities of tokens without an id are 0
        s["logprob"].masked_fill_(prompt, 0.0)
        s["reference"].masked_fill_(prompt, 0.0)
    s["weight"] = torch.full((case["s"],), 1.0 / case["s"], device=dev)
    if op == "policy":
        s["old"] = s["logprob"] + 0.15 * normal(n)
        s["advantage"] = normal(case["s"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"layer_norm": _layer_norm, "layer_norm_grad": _layer_norm_grad, "linear": _linear, "linear_grad": _linear_grad,
            "preference": _preference, "policy": _policy}[case["op"]](state, case)


def _own(s, case):
    from paper_2302_03851_amd import head, tokens
    op = case["op"]
    if op == "layer_norm":
        r = s["out"] = head.layer_norm(s["x"], s["weight"], s["bias"], EPS, dtype=DTYPES[case["out"]], out=s.get("out"))
        return {"out": r.out, "stats": r.stats}
    if op == "layer_norm_grad":
        r = s["out"] = head.layer_norm_grad(s["x"], s["stats"], s["dout"], s["weight"], out=s.get("out"))
        return {"dx": r.dx, "dweight": r.dweight, "dbias": r.dbias}
    if op == "linear":
        r = s["out"] = head.linear(s["x"], s["w"], s["bias"], case["act"], s["res"], dtype=DTYPES[case["out"]],
                                   keep=case["keep"], out=s.get("out"))
        return {"out": r.out, "pre": r.pre} if case["keep"] else {"out": r.out}
    if op == "linear_grad":
        r = s["out"] = head.linear_grad(s["x"], s["w"], s["dout"], case["act"], s["pre"], out=s.get("out"))
        return {"dx": r.dx, "dweight": r.dweight, "dbias": r.dbias}
    if op == "preference":
        r = s["out"] = tokens.preference_loss(s["logprob"], s["reference"], s["first"], case["kind"], BETA,
                                              smoothing=SMOOTHING if case["kind"] == "logistic" else 0.0,
                                              mean=case["mean"], ids=s["ids"], weight=s["weight"], out=s.get("out"))
        return {"loss": r.loss, "reward": r.reward, "g_logprob": r.g_logprob}
    r = s["out"] = tokens.policy_loss(s["logprob"], s["old"], s["first"], s["advantage"], (LOW, HIGH), s["reference"], KL,
                                      mean=case["mean"], ids=s["ids"], weight=s["weight"], out=s.get("out"))
    return {"loss": r.loss, "kl": r.kl, "clipped": r.clipped, "g_logprob": r.g_logprob}


# ---- the plain forms: 32 bits (64 for long sums and next to the clip's borders), rounded once at the end ---------


def _layer_norm(s, case):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    out = d * rstd * s["weight"] + s["bias"]
    return {"out": out.to(DTYPES[case["out"]]), "stats": torch.cat([mean, rstd], 1)}


def _layer_norm_grad(s, case):
    x, dy = s["x"].float(), s["dout"].float()
    mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
    xh = (x - mean) * rstd
    g = dy * s["weight"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xh).sum(0), "dbias": dy.sum(0)}


def _act(v, act):
    if act == "relu":
        return torch.where(v > 0, v, 0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return torch.tanh(v) if act == "tanh" else v


def _slope(v, act):
    if act == "relu":
        return torch.where(v > 0, 1.0, 0.0)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-v))
        return p * (1.0 + v * (1.0 - p))
    t = torch.tanh(v)
    return 1.0 - t * t


def _linear(s, case):
    v = torch.mm(s["x"].float(), s["w"].float())
    if s["bias"] is not None:
        v += s["bias"]
    y = _act(v, case["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    r = {"out": y.to(DTYPES[case["out"]])}
    if case["keep"]:
        r["pre"] = v.to(s["x"].dtype)
    return r


def _linear_grad(s, case):
    g = s["dout"].float()
    if s["pre"] is not None:
        g = g * _slope(s["pre"].float(), case["act"])
    x, w = s["x"].float(), s["w"].float()
    return {"dx": torch.mm(g, w.t()).to(s["x"].dtype), "dweight": torch.mm(x.t(), g).to(s["w"].dtype), "dbias": g.sum(0)}


def _sequences(s, n):
    """Every token's sequence, whether it counts, and how many of a sequence do (at least 1)."""
    ends = s["first"].long()
    at = torch.arange(n, device=ends.device)
    seq = torch.searchsorted(ends, at, right=True) - 1
    live = torch.ones(n, dtype=torch.bool, device=ends.device) if s["ids"] is None else s["ids"] >= 0
    return seq, live, _total(s, live.double()).clamp(min=1.0)


def _total(s, each):
    """Sums over the sequences: differences of the running sum."""
    upto = torch.cat([each.new_zeros(1), each.cumsum(0)])[s["first"].long()]
    return upto[1:] - upto[:-1]


def _preference(s, case):
    seq, live, count = _sequences(s, case["n"])
    d = torch.where(live, s["logprob"].double() - s["reference"].double(), 0.0)
    scale = 1.0 / count if case["mean"] else torch.ones_like(count)
    total = (_total(s, d) * scale).view(-1, 2)
    diff = total[:, 0] - total[:, 1]
    y = BETA * diff
    if case["kind"] == "logistic":
        far, near = torch.clamp(-y, min=0.0), torch.log1p(torch.exp(-y.abs()))
        loss = (1.0 - SMOOTHING) * (far + near) + SMOOTHING * (far + y + near)
        slope = BETA * (SMOOTHING - 1.0 / (1.0 + torch.exp(y)))
    elif case["kind"] == "hinge":
        loss = torch.clamp(1.0 - y, min=0.0)
        slope = torch.where(y < 1.0, -BETA, 0.0).double()
    else:
        off = diff - 0.5 / BETA
        loss, slope = off * off, 2.0 * off
    slope = slope * s["weight"].double()
    each = torch.stack([slope, -slope], 1).view(-1) * scale
    g = torch.where(live, each[seq], 0.0)
    return {"loss": loss.float(), "reward": (BETA * total).float(), "g_logprob": g.float()}


def _policy(s, case):
    seq, live, count = _sequences(s, case["n"])
    lp = s["logprob"].double()
    ratio = torch.exp(lp - s["old"].double())
    a = s["advantage"].double()[seq]
    clipped = live & (((a > 0) & (ratio > 1.0 + HIGH)) | ((a < 0) & (ratio < 1.0 - LOW)))
    q = s["reference"].double() - lp
    grown = torch.expm1(q)
    kl = torch.where(live, grown - q, 0.0)
    gain = torch.where(live, torch.minimum(ratio * a, ratio.clamp(1.0 - LOW, 1.0 + HIGH) * a), 0.0)
    scale = 1.0 / count if case["mean"] else torch.ones_like(count)
    kl_sum = _total(s, kl) * scale
    loss = KL * kl_sum - _total(s, gain) * scale
    slope = -torch.where(clipped, 0.0, a * ratio) - KL * grown
    g = torch.where(live, slope * (scale * s["weight"].double())[seq], 0.0)
    return {"loss": loss.float(), "kl": kl_sum.float(),
            "clipped": _total(s, clipped.double()).to(torch.int32), "g_logprob": g.float()}


# ---- what a pass cannot do without -------------------------------------------------------------------------------


def work(case):
    op, n = case["op"], case["n"]
    if op == "layer_norm":
        D = case["dim"]
        return {"bytes": n * D * (BYTES[case["dtype"]] + BYTES[case["out"]]) + 8 * D + 8 * n, "flops": 8.0 * n * D}
    if op == "layer_norm_grad":
        D = case["dim"]
        return {"bytes": n * D * (2 * BYTES[case["dtype"]] + BYTES[case["out"]]) + 12 * D + 8 * n, "flops": 14.0 * n * D}
    if op in ("linear", "linear_grad"):
        k, m, b, o = case["k"], case["m"], BYTES[case["dtype"]], BYTES[case["out"]]
        if op == "linear":
            out = n * m * (o + o * case["res"] + b * case["keep"])
            return {"bytes": (n * k + k * m) * b + 4 * m * case["bias"] + out, "flops": 2.0 * n * k * m}
        back = n * m * (o + (b if case["act"] != "none" else 0))
        return {"bytes": 2 * (n * k + k * m) * b + 4 * m + back, "flops": 4.0 * n * k * m}
    ids = 4 * n if case["prompts"] else 0
    if op == "preference":
        return {"bytes": 12 * n + ids + 24 * case["s"], "flops": 6.0 * n}
    return {"bytes": 16 * n + ids + 24 * case["s"], "flops": 40.0 * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "layer_norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        rstd = (var + EPS).pow(-0.5)
        return {"out": torch.addcmul(s["bias"].double(), (x - mean) * rstd, s["weight"].double()),
                "stats": torch.cat([mean, rstd], 1)}
    if op == "layer_norm_grad":
        D, parts = case["dim"], []
        dw = torch.zeros(D, dtype=torch.float64, device="cuda")
        db = torch.zeros_like(dw)
        block = max(1, (1 << 26) // D)
        for i in range(0, case["n"], block):
            x, dy = s["x"][i:i + block].double(), s["dout"][i:i + block].double()
            mean, rstd = s["stats"][i:i + block].double().unbind(1)
            xh = (x - mean[:, None]) * rstd[:, None]
            g = dy * s["weight"].double()
            inner = (torch.linalg.vecdot(g, xh)[:, None] * xh + g.sum(1, keepdim=True)) / D
            parts.append((g - inner) * rstd[:, None])
            dw += torch.linalg.vecdot(dy, xh, dim=0)
            db += dy.sum(0)
        return {"dx": torch.cat(parts), "dweight": dw, "dbias": db}
    if op == "linear":
        v = torch.matmul(s["x"].double(), s["w"].double())
        if s["bias"] is not None:
            v = v + s["bias"].double()
        y = v if case["act"] == "none" else getattr(torch.nn.functional, case["act"])(v)
        if s["res"] is not None:
            y = y + s["res"].double()
        return {"out": y, "pre": v} if case["keep"] else {"out": y}
    if op == "linear_grad":
        g = s["dout"].double()
        if s["pre"] is not None:
            v = s["pre"].double().requires_grad_()
            y = getattr(torch.nn.functional, case["act"])(v)
            g, = torch.autograd.grad(y, v, g)
        x, w = s["x"].double(), s["w"].double()
        return {"dx": torch.matmul(g, w.t()), "dweight": torch.matmul(x.t(), g), "dbias": g.sum(0)}
    return _exact_sequences(s, case)


def _exact_sequences(s, case):
    """By the lengths of the sequences and the derivatives of their losses."""
    first = s["first"].long()
    lens = first[1:] - first[:-1]
    live = (s["ids"] >= 0).double() if case["prompts"] else torch.ones(case["n"], dtype=torch.float64, device="cuda")

    def total(v):
        return torch.segment_reduce(v, "sum", lengths=lens, initial=0.0)

    share = total(live).clamp(min=1.0).reciprocal() if case["mean"] else torch.ones(lens.numel(), dtype=torch.float64, device="cuda")
    lp = s["logprob"].double().requires_grad_()
    if case["op"] == "preference":
        ratio = total((lp.detach() - s["reference"].double()) * live) * share
        won, lost = ratio[0::2], ratio[1::2]
        diff = (won - lost).requires_grad_()
        if case["kind"] == "logistic":
            loss = -(1.0 - SMOOTHING) * torch.nn.functional.logsigmoid(BETA * diff)
            loss = loss - SMOOTHING * torch.nn.functional.logsigmoid(-BETA * diff)
        elif case["kind"] == "hinge":
            loss = torch.relu(1.0 - BETA * diff)
        else:
            loss = (diff - 1.0 / (2.0 * BETA)) ** 2
        slope, = torch.autograd.grad((loss * s["weight"].double()).sum(), diff)
        each = torch.stack([slope, -slope], 1).flatten() * share
        return {"loss": loss.detach(), "reward": BETA * ratio.view(-1, 2), "g_logprob": torch.repeat_interleave(each, lens) * live}
    a = torch.repeat_interleave(s["advantage"].double(), lens)
    ratio = (lp - s["old"].double()).exp()
    border = torch.where(a > 0, 1.0 + HIGH, 1.0 - LOW)
    beyond = ((ratio - border) * a > 0).detach()
    q = s["reference"].double() - lp
    kl = q.expm1() - q
    # past the border the surrogate is a constant
    each = KL * kl - a * torch.where(beyond, border, ratio)
    of_token = torch.repeat_interleave(share * s["weight"].double(), lens) * live
    g, = torch.autograd.grad((each * of_token).sum(), lp)
    return {"loss": total(each.detach() * live) * share, "kl": total(kl.detach() * live) * share,
            "clipped": total(beyond.double() * live).round().to(torch.int32), "g_logprob": g}
