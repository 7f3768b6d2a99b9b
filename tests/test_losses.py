"""Preference and policy losses against their definitions in 64 bits, their
gradients also against differences, and their refusals.

Tolerances.  Everything is computed in 64 bits and rounded once: a result is
off by half a unit in its last place (2^-24 of it), and sums besides by 2^-40
of their terms (their number, up to 2^21 here, times 2^-53, with some units
for the exponentials and logarithms).
"""
import ctypes as C
import math

import pytest

from paper_2302_03851_amd import _lib as L

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
U = 2.0 ** -24
F32 = torch.float32
INF = math.inf
NAN = float("nan")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _close(got, ref, terms=0.0):
    got, ref = got.double(), ref.double()
    ref = torch.where(ref.abs() > torch.finfo(F32).max, ref.float().double(), ref)    # past fp32's range
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)])
    assert torch.isfinite(got[fine]).all()
    terms = torch.as_tensor(terms, device=ref.device, dtype=torch.float64).expand_as(ref).nan_to_num(0.0, 0.0, 0.0)
    tol = (1 + 2.0 ** -20) * U * ref.abs() + 2.0 ** -40 * (terms + ref.abs()) + 2.0 ** -149
    off = ((got - ref).abs() - tol)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, float(off.max())


def _offsets(kind, n, s, g):
    """First tokens of s sequences and the last one's end."""
    if kind == "even":
        return torch.arange(s + 1, device="cuda").mul(n).div(s, rounding_mode="floor")
    if kind == "cuts":
        cuts = torch.randint(0, n + 1, (s - 1,), generator=g, device="cuda").sort().values
        return torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), n)])
    if kind == "gaps":       # tokens before the first and behind the last
        return torch.randint(n // 5, n - n // 7 + 1, (s + 1,), generator=g, device="cuda").sort().values
    if kind == "one":        # all tokens in one of them, the others empty
        f = torch.zeros(s + 1, dtype=torch.int64, device="cuda")
        f[s // 2 + 1:] = n
        return f
    if kind == "none":       # all empty, in the middle
        return torch.full((s + 1,), n // 2, device="cuda")
    f = torch.arange(s + 1, device="cuda")     # "short": one token each as far as they go, the rest in the last
    f = f.clamp(max=n)
    f[s] = n
    return f


def _tokens(n, s, kind, ids, seed):
    g = _gen(seed)
    first = _offsets(kind, n, s, g)
    lp = -torch.empty(n, device="cuda").exponential_(generator=g) * 2
    old = lp + 0.2 * torch.randn(n, generator=g, device="cuda")
    ref = lp + 0.3 * torch.randn(n, generator=g, device="cuda")
    i = None
    if ids:
        i = torch.randint(0, 1000, (n,), generator=g, device="cuda").to(torch.int32)
        dead = torch.rand(n, generator=g, device="cuda") < 0.4
        i[dead] = -1
        # what stands there does not count
        for t in (lp, old, ref):
            t[dead & (torch.rand(n, generator=g, device="cuda") < 0.5)] = NAN
    return g, first, lp, old, ref, i


def _spread(first, n, ids):
    """Each token's sequence (the last index: none), and whether it counts."""
    s = first.numel() - 1
    at = torch.arange(n, device="cuda")
    seq = torch.searchsorted(first, at, right=True) - 1
    out = (seq < 0) | (seq >= s) | (at >= first[-1])
    live = ~out if ids is None else ~out & (ids >= 0)
    return torch.where(out, s, seq), live


def _total(v, seq, live, s):
    # on the host: a million additions to one place take minutes on the GPU
    v = torch.where(live, v, 0.0).cpu()
    return torch.zeros(s + 1, dtype=torch.float64).index_add_(0, seq.cpu(), v)[:s].cuda()


def _preference(lp, ref, first, kind, beta, smoothing, mean, ids, weight):
    n, s = lp.numel(), first.numel() - 1
    seq, live = _spread(first, n, ids)
    d = lp.double() - (0.0 if ref is None else ref.double())
    scale = 1 / _total(torch.ones_like(d), seq, live, s).clamp(min=1) if mean else torch.ones(s, dtype=torch.float64, device="cuda")
    total, size = _total(d, seq, live, s) * scale, _total(d.abs(), seq, live, s) * scale
    total, size = total.view(-1, 2), size.view(-1, 2)
    w = torch.ones(s // 2, dtype=torch.float64, device="cuda") if weight is None else weight.double()
    total = torch.where(w[:, None] == 0, 0.0, total)
    diff = total[:, 0] - total[:, 1]
    y = beta * diff
    if kind == "logistic":
        loss = (1 - smoothing) * torch.nn.functional.softplus(-y, threshold=1e9)
        if smoothing:
            loss = loss + smoothing * torch.nn.functional.softplus(y, threshold=1e9)
        slope = beta * (smoothing - torch.sigmoid(-y))
        bend = 1.0
    elif kind == "hinge":
        loss, slope = (1 - y).clamp(min=0), torch.where(torch.isnan(y), y, -beta * (y < 1).double())
        bend = 1.0
    else:
        off = diff - 0.5 / beta
        loss, slope = off * off, 2 * off
        bend = 2 / beta
    out = w == 0
    loss, slope = torch.where(out, 0.0, loss), torch.where(out, 0.0, slope) * w
    each = torch.cat([torch.stack([slope, -slope], 1).view(-1) * scale, slope.new_zeros(1)])
    grad = torch.where(live, each[seq], 0.0)
    terms = size.sum(1)
    return loss, beta * total, grad, terms, bend


def _check_preference(lp, ref, first, kind, beta, smoothing, mean, ids, weight):
    from paper_2302_03851_amd import tokens
    r = tokens.preference_loss(lp, ref, first.to(torch.int32), kind, beta, smoothing, mean, ids, weight)
    loss, reward, grad, terms, bend = _preference(lp, ref, first, kind, beta, smoothing, mean, ids, weight)
    slope = 2 * (loss.abs().sqrt() if kind == "squared" else beta) if kind == "squared" else beta
    _close(r.loss, loss, terms * slope + (1 if kind != "squared" else terms ** 2 + 1 / beta ** 2))
    _close(r.reward, reward, beta * terms[:, None])
    seq, _ = _spread(first, lp.numel(), ids)
    per = torch.cat([torch.stack([terms, terms], 1).view(-1), terms.new_zeros(1)])
    w = 1.0 if weight is None else float(weight.abs().max())
    _close(r.g_logprob, grad, w * (per[seq] * bend + 1 / beta + beta))
    return r


SIZES = [(1, 2), (5, 2), (300, 6), (2047, 40), (2049, 2), (4000, 1000), (32768, 64), (32769, 64), (40960, 2), (40960, 20000),
         (100001, 30), (300007, 4000), (1 << 20, 90000)]


@gpu
@pytest.mark.parametrize("n,s", SIZES)
@pytest.mark.parametrize("layout", ["even", "cuts", "gaps", "one", "none", "short"])
@pytest.mark.parametrize("ids", [False, True])
def test_preference(n, s, layout, ids):
    g, first, lp, _, ref, i = _tokens(n, s, layout, ids, n + s)
    w = torch.randn(s // 2, generator=g, device="cuda")
    w[1::3] = 0.0
    for kind, beta, smoothing, mean, weight, reference in [("logistic", 0.1, 0.0, False, None, ref), ("logistic", 0.5, 0.2, True, w, ref),
                                                           ("hinge", 0.3, 0.0, True, w, None), ("squared", 0.2, 0.0, True, w, ref)]:
        _check_preference(lp, reference, first, kind, beta, smoothing, mean, i, weight)


def _policy(lp, old, ref, first, adv, low, high, coef, per_token, mean, ids, weight):
    n, s = lp.numel(), first.numel() - 1
    seq, live = _spread(first, n, ids)
    w = torch.ones(s, dtype=torch.float64, device="cuda") if weight is None else weight.double()
    w1 = torch.cat([w, w.new_zeros(1)])
    live = live & (w1[seq] != 0)
    a = adv.double() if per_token else torch.cat([adv.double(), adv.new_zeros(1).double()])[seq]
    ratio = torch.exp(lp.double() - old.double())
    beyond = live & (((a > 0) & (ratio > 1 + high)) | ((a < 0) & (ratio < 1 - low)))
    gain = torch.where(beyond, a * torch.where(a > 0, torch.full_like(a, 1 + high), 1 - low), torch.where((a == 0) & ~torch.isnan(ratio), 0.0, a * ratio))
    slope = torch.where(beyond, 0.0, torch.where((a == 0) & ~torch.isnan(ratio), 0.0, -a * ratio))
    kl = torch.zeros_like(gain)
    if ref is not None:
        q = ref.double() - lp.double()
        kl = torch.where(q == INF, INF, torch.expm1(q) - q)
        if coef:
            slope = slope - coef * torch.expm1(q)
    count = _total(torch.ones_like(gain), seq, live, s).clamp(min=1)
    scale = 1 / count if mean else torch.ones_like(count)
    k = _total(kl, seq, live, s) * scale
    loss = -_total(gain, seq, live, s) * scale
    if coef:
        loss = loss + coef * k
    terms = _total(gain.abs() + coef * kl, seq, live, s) * scale
    grad = torch.where(live, slope * torch.cat([scale * w, w.new_zeros(1)])[seq], 0.0)
    return loss, k, _total(beyond.double(), seq, live, s).to(torch.int32), grad, terms


def _check_policy(lp, old, ref, first, adv, low, high, coef, per_token, mean, ids, weight):
    from paper_2302_03851_amd import tokens
    r = tokens.policy_loss(lp, old, first.to(torch.int32), adv, (low, high), ref, coef, per_token, mean, ids, weight)
    loss, kl, clipped, grad, terms = _policy(lp, old, ref, first, adv, low, high, coef, per_token, mean, ids, weight)
    _close(r.loss, loss, terms)
    _close(r.kl, kl)
    assert torch.equal(r.clipped, clipped)
    _close(r.g_logprob, grad, 2 * grad.abs().nan_to_num(0.0, 0.0, 0.0) + (1.0 if weight is None else float(weight.abs().max())))
    return r


@gpu
@pytest.mark.parametrize("n,s", SIZES)
@pytest.mark.parametrize("layout", ["even", "cuts", "gaps", "one", "none", "short"])
@pytest.mark.parametrize("ids", [False, True])
def test_policy(n, s, layout, ids):
    g, first, lp, old, ref, i = _tokens(n, s, layout, ids, n + s + 1)
    w = torch.randn(s, generator=g, device="cuda")
    w[1::3] = 0.0
    adv, each = torch.randn(s, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    each[::7] = 0.0
    for a, per_token, mean, weight, reference, coef in [(adv, False, True, None, ref, 0.04), (each, True, False, w, None, 0.0),
                                                        (adv, False, False, w, ref, 0.0), (each, True, True, w, ref, 0.3)]:
        _check_policy(lp, old, reference, first, a, 0.2, 0.28, coef, per_token, mean, i, weight)


@gpu
def test_long_sums():
    """Sums of a million tokens that nearly cancel."""
    g = _gen(5)
    n = 1 << 21
    lp = -20 * torch.rand(n, generator=g, device="cuda")
    ref = lp + 1e-3 * torch.randn(n, generator=g, device="cuda")
    first = torch.tensor([0, n // 2, n], device="cuda")
    for mean in (False, True):
        _check_preference(lp, ref, first, "logistic", 0.1, 0.0, mean, None, None)
        _check_preference(lp, None, first, "squared", 0.1, 0.0, mean, None, None)
        _check_policy(lp, lp, ref, first, torch.ones(2, device="cuda"), 0.2, 0.2, 0.1, False, mean, None, None)


def _median_us(f, calls=5):
    f()
    times = []
    for _ in range(calls):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return sorted(times)[calls // 2]


def _one_long(n):
    """Log probabilities, old and reference ones, and ids, three of four tokens with one."""
    lp = -torch.rand(n, generator=_gen(n), device="cuda")
    return lp, lp + 0.1, lp - 0.1, (torch.arange(n, device="cuda") % 4 - 1).to(torch.int32)


@gpu
def test_long_sequence_counts():
    """Means over the tokens with an id cost a look at the ids, however long a sequence is (where every chunk added up
    all of its sequence's chunks, 2^26 tokens in one took six times as long as for their sum)."""
    from paper_2302_03851_amd import tokens
    n = 1 << 26
    lp, old, ref, ids = _one_long(n)
    first = torch.tensor([0, 5, n - 3, n], dtype=torch.int32, device="cuda")
    adv = torch.tensor([1.0, 2.0, 3.0], device="cuda")
    r = tokens.policy_loss(lp, old, first, adv, reference=ref, kl=0.1, ids=ids)
    count = (ids[5:n - 3] >= 0).sum().double()
    gain, q = torch.exp(lp.double() - old.double()), ref.double() - lp.double()
    each = torch.where(ids >= 0, 0.1 * (torch.expm1(q) - q) - 2.0 * gain, 0.0)
    _close(r.loss[1], each[5:n - 3].sum() / count, 2.0)
    slope = torch.where(ids >= 0, -2.0 * gain - 0.1 * torch.expm1(q), 0.0)
    _close(r.g_logprob[5:n - 3], slope[5:n - 3] / count, 2.0 / n)

    def run(mean):
        return lambda: tokens.policy_loss(lp, old, first, adv, reference=ref, kl=0.1, mean=mean, ids=ids, out=r)
    assert _median_us(run(True)) <= 3 * _median_us(run(False))


@gpu
def test_long_sequence_time():
    """One sequence of 2^26 tokens costs about what 4096 of 2^14 do (where one thread wrote its 65536 places and one
    wave asked for its sums one by one, six times as much)."""
    from paper_2302_03851_amd import tokens
    n = 1 << 26
    lp, old, ref, ids = _one_long(n)

    def times(first):
        adv = torch.ones(first.numel() - 1, device="cuda")
        q = tokens.preference_loss(lp, ref, first, mean=True, ids=ids)
        r = tokens.policy_loss(lp, old, first, adv, reference=ref, kl=0.1, mean=False, ids=ids)
        return (_median_us(lambda: tokens.preference_loss(lp, ref, first, mean=True, ids=ids, out=q)),
                _median_us(lambda: tokens.policy_loss(lp, old, first, adv, reference=ref, kl=0.1, mean=False, ids=ids, out=r)))
    many = times((torch.arange(4097, device="cuda") << 14).to(torch.int32))
    one = times(torch.tensor([0, n, n], dtype=torch.int32, device="cuda"))
    assert one[0] <= 3 * many[0] and one[1] <= 3 * many[1], (one, many)


@gpu
@pytest.mark.parametrize("layout,s", [("cuts", 300), ("cuts", 20000), ("gaps", 40), ("one", 6), ("short", 3000), ("even", 5000)])
def test_many_chunks(layout, s):
    """Enough tokens for work-groups that count several chunks: sequences that cover some of them, begin, end or lie
    within one."""
    n = 5 * (1 << 20) + 77
    g, first, lp, old, ref, i = _tokens(n, s, layout, True, s)
    _check_policy(lp, old, ref, first, torch.randn(s, generator=g, device="cuda"), 0.2, 0.28, 0.04, False, True, i, None)
    _check_preference(lp, ref, first, "logistic", 0.1, 0.0, True, i, None)


@gpu
def test_empty_sequences_time():
    """A million empty sequences behind the last token, before the first or at one place in the middle cost a look at
    each (where the chunk there went through all of them by itself, 4 ms for the calls that take 0.15 and 0.26)."""
    from paper_2302_03851_amd import tokens
    n, many = 1 << 20, 1 << 20
    lp, old, ref, ids = _one_long(n)
    some = (torch.arange(1025, device="cuda") << 10) - 3
    some[0], some[-1] = 0, n
    for at in (0, 513, 1025):
        first = torch.cat([some[:at], some.new_full((many - 1024,), int(some[min(at, 1024)])), some[at:]])
        assert first.numel() == many + 1
        adv = torch.randn(many, generator=_gen(at), device="cuda")
        _check_policy(lp, old, ref, first, adv, 0.2, 0.28, 0.04, False, True, ids, None)
        _check_preference(lp, ref, first, "logistic", 0.1, 0.0, True, ids, None)
        # the same tokens in as many sequences of one each
        each = torch.arange(many + 1, device="cuda")
        took = []
        for f in (first.to(torch.int32), each.to(torch.int32)):
            q = tokens.preference_loss(lp, ref, f, mean=True, ids=ids)
            r = tokens.policy_loss(lp, old, f, adv, reference=ref, kl=0.1, ids=ids)
            took.append((_median_us(lambda: tokens.preference_loss(lp, ref, f, mean=True, ids=ids, out=q)),
                         _median_us(lambda: tokens.policy_loss(lp, old, f, adv, reference=ref, kl=0.1, ids=ids, out=r))))
        assert took[0][0] <= 3 * took[1][0] and took[0][1] <= 3 * took[1][1], took


@gpu
@pytest.mark.parametrize("n", [400, 70000])
def test_limits(n):
    """Infinite log probabilities, ratios past the range, no advantage, ratios of exactly 1."""
    g = _gen(n)
    s = 40
    first = _offsets("even", n, s, g)
    lp = -torch.rand(n, generator=g, device="cuda")
    ref = lp.clone()
    lp[first[0]], lp[first[3]], ref[first[4]], ref[first[7]] = -INF, -INF, -INF, -INF
    lp[first[8]], lp[first[11]], lp[first[12]] = NAN, INF, -1e38
    ref[first[14]], lp[first[14]] = -INF, -INF
    for mean in (False, True):
        for kind in ("logistic", "hinge", "squared"):
            r = _check_preference(lp, ref, first, kind, 0.1, 0.0, mean, None, None)
        r = _check_preference(lp, ref, first, "logistic", 0.1, 0.0, mean, None, None)
        assert r.loss[0] == INF and r.loss[1] == 0 and r.loss[2] == 0 and r.loss[3] == INF and torch.isnan(r.loss[4])
        assert torch.isfinite(r.g_logprob[:first[8]]).all()
        _check_preference(lp, ref, first, "logistic", 0.1, 0.3, mean, None, None)
    old = -torch.rand(n, generator=g, device="cuda")
    old[first[5]], old[first[6]], old[first[9]] = -1000.0, -INF, -800.0
    adv = torch.randn(s, generator=g, device="cuda")
    adv[5], adv[6], adv[9], adv[10], adv[13] = 1.0, -1.0, 0.0, INF, NAN
    old[first[10] + 1:first[11]] = lp[first[10] + 1:first[11]]
    for mean in (False, True):
        _check_policy(lp, old, ref, first, adv, 0.2, 0.3, 0.05, False, mean, None, None)
        _check_policy(lp, old, None, first, adv, 0.0, 0.0, 0.0, False, mean, None, None)
        _check_policy(lp, old, ref, first, adv, 1.0, 10.0, 0.0, False, mean, None, None)
    same = _check_policy(old, old, old, first, adv, 0.0, 0.0, 1.0, False, True, None, None)
    assert not same.clipped.any()


@gpu
@pytest.mark.parametrize("n", [640, 70000])
@pytest.mark.parametrize("mean", [False, True])
def test_smoothing_of_one(n, mean):
    """All of the weight on the other one: the loss and its gradient of the swapped pair, the limits at infinite
    ratios, and gradients that keep their digits where the loss is next to 0."""
    from paper_2302_03851_amd import tokens
    g = _gen(n)
    s, beta = 32, 0.5
    first = _offsets("even", n, s, g)
    lp = -torch.rand(n, generator=g, device="cuda")
    ref = lp + 0.01 * torch.randn(n, generator=g, device="cuda")
    at = first[:-1] + 1
    lp[at[0]], lp[at[3]], ref[at[4]], ref[at[7]], lp[at[8]] = -INF, -INF, -INF, -INF, NAN
    per = int(first[1] - first[0]) if mean else 1
    for i, margin in ((10, -130.0), (12, 130.0), (14, -60.0), (16, -1400.0), (18, 1400.0)):
        lp[at[i]] += margin * per
    r = tokens.preference_loss(lp, ref, first.to(torch.int32), "logistic", beta, 1.0, mean)
    ratio = _total(lp.double() - ref.double(), *_spread(first, n, None), s)
    live = _total(torch.ones(n, dtype=torch.float64, device="cuda"), *_spread(first, n, None), s)
    scale = 1 / live if mean else torch.ones_like(live)
    y = beta * (ratio * scale).view(-1, 2).diff(dim=1)[:, 0].neg()
    loss = torch.nn.functional.softplus(y, threshold=1e9)
    slope = torch.stack([beta * torch.sigmoid(y), -beta * torch.sigmoid(y)], 1).view(-1) * scale
    # y is off by 2^-40 of its terms, which the exponentials hand on relative to their own size
    terms = beta * (_total((lp.double() - ref.double()).abs(), *_spread(first, n, None), s) * scale).view(-1, 2).sum(1)
    _close(r.loss, loss, terms * torch.sigmoid(y).nan_to_num(0.0))
    seq = _spread(first, n, None)[0]
    _close(r.g_logprob, slope[seq], (slope.abs() * terms.nan_to_num(0.0, 0.0, 0.0).repeat_interleave(2))[seq])
    # -inf: no loss; inf: all of it; NaN stays
    assert r.loss[0] == 0 and r.loss[1] == INF and r.loss[2] == INF and r.loss[3] == 0 and torch.isnan(r.loss[4])
    assert not r.g_logprob[first[0]:first[2]].any() and (r.g_logprob[first[2]:first[3]] > 0).all()
    assert (r.g_logprob[first[10]:first[11]] > 0).all() and (r.g_logprob[first[14]:first[15]] > 0).all()


@gpu
def test_empty_calls():
    from paper_2302_03851_amd import tokens
    none, zero = torch.zeros(0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    lp = torch.full((5,), -1.0, device="cuda")
    r = tokens.preference_loss(lp, lp, zero)
    assert r.loss.shape == (0,) and r.reward.shape == (0, 2) and not r.g_logprob.any()
    r = tokens.preference_loss(none, none, zero.expand(5).contiguous(), "hinge")
    assert r.loss.tolist() == [1.0, 1.0] and not r.reward.any() and r.g_logprob.shape == (0,)
    r = tokens.policy_loss(lp, lp, zero, none)
    assert r.loss.shape == (0,) and not r.g_logprob.any()
    r = tokens.policy_loss(none, none, zero.expand(4).contiguous(), torch.ones(3, device="cuda"))
    assert not r.loss.any() and not r.kl.any() and not r.clipped.any()


@gpu
@pytest.mark.parametrize("n", [300, 50000])
def test_wild_offsets(n):
    """Offsets that fall or leave the tokens: nothing outside the results is touched."""
    from paper_2302_03851_amd import tokens
    g = _gen(n)
    s = 64
    first = torch.randint(-2 ** 31, 2 ** 31 - 1, (s + 1,), generator=g, device="cuda").to(torch.int32)
    first[::3] = torch.randint(0, n, (first[::3].numel(),), generator=g, device="cuda").to(torch.int32)
    lp = -torch.rand(n, generator=g, device="cuda")
    mem = torch.full((n + 64,), 7.0, device="cuda")
    small = torch.full((3 * s + 64,), 7.0, device="cuda")
    for f in (lambda: tokens.preference_loss(lp, lp, first, out=tokens.Preference(small[32:32 + s // 2], small[64:64 + s].view(-1, 2), mem[32:32 + n])),
              lambda: tokens.policy_loss(lp, lp, first, lp[:s], out=tokens.Policy(small[32:32 + s], small[96:96 + s], small[160:160 + s].view(torch.int32), mem[32:32 + n]))):
        f()
        torch.cuda.synchronize()
        assert (mem[:32] == 7).all() and (mem[32 + n:] == 7).all() and (small[:32] == 7).all() and (small[160 + s:] == 7).all()


@gpu
@pytest.mark.parametrize("n,s", [(40000, 9000), (5 * (1 << 20) + 77, 6000)])
def test_wild_offsets_of_many(n, s):
    """The same where tokens look for their sequences by halving, and work-groups count several chunks."""
    from paper_2302_03851_amd import tokens
    g = _gen(n)
    first = torch.randint(-2 ** 31, 2 ** 31 - 1, (s + 1,), generator=g, device="cuda").to(torch.int32)
    first[::3] = torch.randint(0, n, (first[::3].numel(),), generator=g, device="cuda").to(torch.int32)
    sorted_half = first.clone()
    sorted_half[: s // 2] = torch.randint(0, n, (s // 2,), generator=g, device="cuda").sort().values.to(torch.int32)
    same = torch.full_like(first, n // 3)
    same[0], same[s // 2:s // 2 + 2] = 0, torch.tensor([n, n // 2], dtype=torch.int32, device="cuda")
    lp = -torch.rand(n, generator=g, device="cuda")
    ids = (torch.arange(n, device="cuda") % 3 - 1).to(torch.int32)
    adv = torch.randn(s, generator=g, device="cuda")
    for f in (first, sorted_half, same):
        mem = torch.full((n + 64,), 7.0, device="cuda")
        small = torch.full((3 * s + 160,), 7.0, device="cuda")
        tokens.preference_loss(lp, lp, f, mean=True, ids=ids,
                               out=tokens.Preference(small[32:32 + s // 2], small[64 + s:64 + 2 * s].view(-1, 2), mem[32:32 + n]))
        torch.cuda.synchronize()
        assert (mem[:32] == 7).all() and (mem[32 + n:] == 7).all() and (small[:32] == 7).all() and (small[64 + 2 * s:] == 7).all()
        small.fill_(7.0)
        tokens.policy_loss(lp, lp, f, adv, ids=ids, out=tokens.Policy(
            small[32:32 + s], small[64 + s:64 + 2 * s], small[96 + 2 * s:96 + 3 * s].view(torch.int32), mem[32:32 + n]))
        torch.cuda.synchronize()
        assert (mem[:32] == 7).all() and (mem[32 + n:] == 7).all() and (small[:32] == 7).all() and (small[96 + 3 * s:] == 7).all()
        assert (small[32 + s:64 + s] == 7).all() and (small[64 + 2 * s:96 + 2 * s] == 7).all()


@gpu
def test_differences():
    """The gradients against central differences of the losses: steps of 2^-5; the third derivatives stay
    below 40 here, the losses' own roundings give u |loss| / step."""
    from paper_2302_03851_amd import tokens
    g = _gen(8)
    n, step = 40, 2.0 ** -5
    first = torch.tensor([0, 9, 20, 28, 40], dtype=torch.int32, device="cuda")
    lp = -torch.rand(n, generator=g, device="cuda")
    ref = lp + 0.1 * torch.randn(n, generator=g, device="cuda")
    old = lp + 0.02 * torch.randn(n, generator=g, device="cuda")     # no ratio within a step of the clip
    adv = torch.randn(4, generator=g, device="cuda")
    for name, f in [(k, lambda x, k=k: tokens.preference_loss(x, ref, first, k, 0.5, mean=k == "squared")) for k in ("logistic", "squared")] + \
                   [("policy", lambda x: tokens.policy_loss(x, old, first, adv, (0.5, 0.5), ref, 0.3))]:
        r = f(lp)
        noise = U * float(r.loss.abs().sum()) / step
        for t in (0, 8, 9, 27, 39):
            up, down = lp.clone(), lp.clone()
            up[t] += step
            down[t] -= step
            slope = (float(f(up).loss.double().sum()) - float(f(down).loss.double().sum())) / (2 * step)
            assert abs(float(r.g_logprob[t]) - slope) <= step ** 2 / 6 * 40 + 2 * noise


# ---- together ---------------------------------------------------------------------------


def _chain(model, h, ids, loss):
    """The example's loss and gradients by torch's derivatives in 64 bits; loss(lp) gives the mean to descend."""
    leaves = [t.double().requires_grad_() for t in (model.w, model.b, model.W, model.c, model.O)]
    w, b, W, c, O = leaves
    z = torch.nn.functional.layer_norm(h.double(), (h.shape[1],), w, b, 1e-5)
    u = torch.nn.functional.gelu(z @ W + c) + z
    lp = torch.log_softmax(u @ O, 1).gather(1, ids.clamp(min=0).long()[:, None])[:, 0]
    value = loss(lp)
    return value.detach(), torch.autograd.grad(value, leaves)


@gpu
def test_preferred_words_gradients():
    """The head, the log probabilities and both losses as one program, against torch's derivatives in 64 bits.

    Five products of at most 2 n + 16 roundings (n = 64 hidden, up to 400 words or logits) of sums that are up to
    8 times their terms' norm here: 5 * 816 * 8 u = 2^-9, of each gradient's norm."""
    from examples import preferred_words as ex
    h, ids, first = ex.states(8, 400, "cuda:0")
    model = ex.Head(h.shape[1], 400, 3, "cuda:0")
    g = _gen(4)
    model.c = torch.randn(h.shape[1], generator=g, device="cuda")
    model.w = 1 + 0.3 * torch.randn(h.shape[1], generator=g, device="cuda")
    n, s = h.shape[0], first.numel() - 1
    reference = -torch.rand(n, generator=g, device="cuda") * 8
    seq, live = _spread(first.long(), n, ids)

    def close(got, ref):
        for a, b in zip(got, ref):
            assert float((a.double() - b).norm()) <= 2.0 ** -9 * float(b.norm())

    def sums(v):
        return torch.zeros(s + 1, dtype=torch.float64, device="cuda").index_add(0, seq, torch.where(live, v, 0.0))[:s]

    count = sums(torch.ones(n, dtype=torch.float64, device="cuda"))

    def preference(lp):
        r = (sums(lp - reference.double()) / count).view(-1, 2)
        return torch.nn.functional.softplus(-0.5 * (r[:, 0] - r[:, 1])).mean()

    lp, p, gradients = ex.preferred(model, h, ids, first, reference, 0.5)
    value, ref = _chain(model, h, ids, preference)
    assert abs(float(p.loss.double().mean()) - float(value)) <= 2.0 ** -9 * float(value)
    close(gradients, ref)

    old = lp + 0.1 * torch.randn(n, generator=g, device="cuda")
    adv = torch.randn(s, generator=g, device="cuda")
    a = torch.cat([adv, adv.new_zeros(1)]).double()[seq]
    # a ratio within the forward pass's error of a border could fall on either side: none here
    d = (lp.double() - old.double())[live]
    assert min(float((d - math.log(x)).abs().min()) for x in (0.8, 1.28)) > 1e-5

    def policy(lp):
        r = torch.exp(lp - old.double())
        q = reference.double() - lp
        each = -torch.minimum(r * a, r.clamp(0.8, 1.28) * a) + 0.02 * (torch.expm1(q) - q)
        return (sums(each) / count).mean()

    _, p, gradients = ex.tuned(model, h, ids, first, old, reference, adv, 0.02)
    value, ref = _chain(model, h, ids, policy)
    assert abs(float(p.loss.double().mean()) - float(value)) <= 2.0 ** -9 * (abs(float(value)) + 1)
    close(gradients, ref)


@gpu
def test_preferred_words_example():
    from examples import preferred_words
    said = []
    preferences, tunings = preferred_words.run(instances=6, vocab=1003, steps=6, report=said.append)
    assert all(math.isfinite(x) for x in preferences + tunings) and len(preferences) == len(tunings) == 6
    assert abs(preferences[0] - math.log(2)) < 1e-5 and len(said) == 3


# ---- streams and graphs -----------------------------------------------------


def _everything(seed):
    from paper_2302_03851_amd import tokens
    cases = []
    for n, s, layout in [(3000, 20, "cuts"), (90000, 300, "cuts"), (200000, 40000, "cuts"), (40000, 4, "one")]:
        g, first, lp, old, ref, i = _tokens(n, s, layout, True, seed + n)
        cases.append((first.to(torch.int32), lp, old, ref, i, torch.randn(s, generator=g, device="cuda")))

    def go():
        got = []
        for first, lp, old, ref, i, adv in cases:
            got += [*tokens.preference_loss(lp, ref, first, "logistic", 0.1, 0.1, True, i)]
            got += [*tokens.policy_loss(lp, old, first, adv, (0.2, 0.3), ref, 0.1, ids=i)]
        return got

    return go


def _same(a, b):
    return all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(a, b))


@gpu
def test_losses_streams():
    runs = [_everything(s) for s in range(3)]
    ref = [go() for go in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        got = []
        for go, st in zip(runs, streams):
            with torch.cuda.stream(st):
                got.append(go())
        torch.cuda.synchronize()
        assert all(_same(a, b) for a, b in zip(got, ref))


@gpu
def test_losses_captured():
    go = _everything(7)
    ref = go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = go()
    for _ in range(4):
        for t in held:
            t.view(torch.uint8).fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert _same(held, ref)
        assert _same(go(), ref)
        torch.cuda.synchronize()


# ---- refusals ------------------------------------------------------------------------

A = 1 << 30
INVALID, UNSUPPORTED = L.EDB_ERR_INVALID, L.EDB_ERR_UNSUPPORTED


def _pref(**k):
    a = dict(lp=A, ref=2 * A, ids=3 * A, n=100, first=4 * A, pairs=4, kind=0, beta=0.1, smoothing=0.1, mean=1, w=5 * A, loss=6 * A,
             reward=7 * A, g=8 * A, ws=9 * A, wb=1 << 29)
    a.update(k)
    return L.load().edb_preference_loss(*a.values(), None)


def _pol(**k):
    a = dict(lp=A, old=2 * A, ref=3 * A, ids=4 * A, n=100, first=5 * A, s=4, adv=6 * A, each=0, low=0.2, high=0.2, kl=0.1, mean=1, w=7 * A,
             loss=8 * A, div=9 * A, clipped=10 * A, g=11 * A, ws=12 * A, wb=1 << 29)
    a.update(k)
    return L.load().edb_policy_loss(*a.values(), None)


REFUSED = (
    [(_pref, k, e) for k, e in [
        (dict(lp=None), INVALID), (dict(first=None), INVALID), (dict(loss=None), INVALID), (dict(reward=None), INVALID), (dict(g=None), INVALID),
        (dict(n=-1), INVALID), (dict(pairs=-1), INVALID), (dict(pairs=(1 << 24) + 1), UNSUPPORTED), (dict(kind=-1), INVALID), (dict(kind=3), INVALID),
        (dict(beta=0.0), INVALID), (dict(beta=-1.0), INVALID), (dict(beta=INF), INVALID), (dict(beta=NAN), INVALID), (dict(smoothing=-0.1), INVALID),
        (dict(smoothing=1.1), INVALID), (dict(smoothing=NAN), INVALID), (dict(kind=1), INVALID), (dict(kind=2), INVALID),
        (dict(n=50000, wb=0), INVALID), (dict(n=50000, ws=None), INVALID), (dict(n=50000, ws=9 * A + 8), INVALID), (dict(lp=A + 2), INVALID),
        (dict(ids=3 * A + 1), INVALID), (dict(first=4 * A + 2), INVALID), (dict(g=A), INVALID), (dict(g=3 * A + 396), INVALID),
        (dict(loss=4 * A + 32), INVALID), (dict(reward=5 * A + 12), INVALID), (dict(reward=6 * A - 28), INVALID), (dict(g=7 * A + 28), INVALID),
        (dict(n=50000, ws=8 * A + 199984), INVALID)]]
    + [(_pol, k, e) for k, e in [
        (dict(lp=None), INVALID), (dict(old=None), INVALID), (dict(first=None), INVALID), (dict(adv=None), INVALID), (dict(loss=None), INVALID),
        (dict(div=None), INVALID), (dict(clipped=None), INVALID), (dict(g=None), INVALID), (dict(ref=None), INVALID), (dict(n=-1), INVALID),
        (dict(s=-1), INVALID), (dict(s=(1 << 24) + 1), UNSUPPORTED), (dict(low=-0.1), INVALID), (dict(low=1.1), INVALID), (dict(low=NAN), INVALID),
        (dict(high=-0.1), INVALID), (dict(high=INF), INVALID), (dict(high=NAN), INVALID), (dict(kl=-0.1), INVALID), (dict(kl=INF), INVALID),
        (dict(kl=NAN), INVALID), (dict(n=50000, wb=0), INVALID), (dict(n=50000, ws=None), INVALID), (dict(n=50000, ws=12 * A + 4), INVALID),
        (dict(adv=6 * A + 2), INVALID), (dict(g=A + 396), INVALID), (dict(loss=6 * A + 12), INVALID), (dict(g=6 * A + 12), INVALID),
        (dict(g=6 * A + 396, each=1), INVALID), (dict(clipped=9 * A + 12), INVALID), (dict(div=7 * A + 12), INVALID), (dict(loss=5 * A + 16), INVALID),
        (dict(n=50000, ws=11 * A + 199984), INVALID)]])


@pytest.mark.parametrize("call,changed,status", REFUSED, ids=[f"{f.__name__[1:]}-{i}" for i, (f, _, _) in enumerate(REFUSED)])
def test_refusals(call, changed, status):
    """Refused on the host, with a message, before any launch (no GPU needed)."""
    assert call(**changed) == status
    assert L.load().edb_last_error()


def test_nothing_to_do():
    assert _pref(n=0, pairs=0) == L.EDB_OK and _pol(n=0, s=0) == L.EDB_OK


def test_workspace_sizes():
    lib, nb = L.load(), C.c_int64(-1)
    for f in (lib.edb_preference_loss_bytes, lib.edb_policy_loss_bytes):
        assert f(100, 4, C.byref(nb)) == L.EDB_OK and nb.value == 0
        assert f(2 ** 31 - 1, 1 << 24, C.byref(nb)) == L.EDB_OK and nb.value > 0
        assert f(-1, 4, C.byref(nb)) == INVALID and f(1, -4, C.byref(nb)) == INVALID and f(1, 4, None) == INVALID
        assert f(1, (1 << 24) + 1, C.byref(nb)) == UNSUPPORTED


def test_python_checks():
    from paper_2302_03851_amd import tokens
    lp, first = torch.zeros(4), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        tokens.preference_loss(lp, lp, first)
    with pytest.raises(ValueError):
        tokens.policy_loss(lp, lp, first, lp)


@gpu
def test_python_checks_gpu():
    from paper_2302_03851_amd import tokens
    lp, first = torch.zeros(4, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [lambda: tokens.preference_loss(lp, lp[:3], first), lambda: tokens.preference_loss(lp, lp, first[:2]),
           lambda: tokens.preference_loss(lp, lp, first.long()), lambda: tokens.preference_loss(lp, lp, first, "linear"),
           lambda: tokens.preference_loss(lp, lp.double(), first), lambda: tokens.preference_loss(lp, lp, first, ids=lp),
           lambda: tokens.preference_loss(lp, lp, first, weight=lp), lambda: tokens.preference_loss(lp, lp, first[:0]),
           lambda: tokens.policy_loss(lp, lp, first, lp), lambda: tokens.policy_loss(lp, lp, first, lp[:2], per_token=True),
           lambda: tokens.policy_loss(lp, lp.cpu(), first, lp[:2]), lambda: tokens.policy_loss(lp, lp, first[None], lp[:2])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: tokens.preference_loss(lp, lp, first, beta=0.0), lambda: tokens.policy_loss(lp, lp, first, lp[:2], kl=0.1),
              lambda: tokens.policy_loss(lp, lp, first, lp[:2].clone(), clip=(2.0, 0.1))):
        with pytest.raises(L.EdbError):
            f()
