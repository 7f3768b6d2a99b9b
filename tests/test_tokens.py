"""Token operators (embedding and its gradient, log probabilities and theirs,
distillation) against the definitions in 64 bits, and their refusals.

Tolerances.  u = 2^-24 is fp32's rounding unit; a bf16 result adds half a unit
in its last place, at most 2^-8 of the value (8 significant bits).
* An fp32 sum of k terms, in any order, is off by at most k u sum |term|.
* ln sum exp: each exponent (x - m) / T is off by 4 u of itself, the
  exponential by 4 u more, the sum (every thread adds at most V / 64 terms, then a tree) by
  (V / 64 + 16) u, the logarithm by 4 u of its own value.  So l is off by at
  most LSE = (V / 64 + 24 + 4 w) u + 4 u l, w being the p-weighted mean of |x - m| / T;
  a log probability by LSE + 4 u (|x - m| / T + |lp|); the entropy by
  LSE + (V / 64 + 16) u H plus, per term p |y|, 8 u (1 + |y|).
* p is off by LSE + 8 u (1 + |lp|) of itself.
"""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2302_03851_amd import _lib as L

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
INF = math.inf


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _half_ulp(ref, dtype):
    return ref.abs() * (2.0 ** -8 if dtype == BF16 else U)


def _close(got, ref, tol):
    """Equal where not finite, within tol elsewhere."""
    got = got.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    assert torch.equal(torch.isfinite(got), fine)
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)])
    tol = torch.as_tensor(tol, device=ref.device, dtype=torch.float64).nan_to_num(0.0)
    off = (got - ref).abs()[fine] - torch.broadcast_to(tol, ref.shape)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, (float(off.max()), float((got - ref).abs()[fine].max()))


def _view(t, pad, shift):
    """The same matrix as a view with `pad` more elements a row, starting
    `shift` elements into its memory; what lies between is NaN."""
    n, m = t.shape
    mem = torch.full((n * (m + pad) + shift + 16,), float("nan"), dtype=t.dtype, device=t.device)
    v = mem[shift:shift + n * (m + pad)].view(n, m + pad)[:, :m]
    v.copy_(t)
    return v, mem


# ---- embedding ---------------------------------------------------------------

EMBED = [(1, 5, 1), (7, 3, 7), (64, 100, 8), (112, 50, 64), (33, 1000, 100), (1000, 77, 256), (300, 9, 513), (65, 40, 1032)]


def _some_ids(n, V, g, spread):
    """Ids in range, with ones outside on both sides among them."""
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    if spread:
        ids = (ids.double() / V).pow(3).mul(V).to(torch.int32)
        for k, bad in enumerate((-1, V, -2 ** 31, 2 ** 31 - 1)):
            ids[k + 2::11] = bad
    return ids


@gpu
@pytest.mark.parametrize("table,out", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,V,E", EMBED)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_embed(n, V, E, table, out, pad, shift):
    """One fp32 product and one rounding: the same bits as torch's."""
    from paper_2302_03851_amd import tokens
    g = _gen(n + E)
    w, _ = _view(torch.randn((V, E), generator=g, device="cuda").to(table), pad, shift)
    ids = _some_ids(n, V, g, True)
    there = (ids >= 0) & (ids < V)
    ref = torch.where(there[:, None], w[torch.where(there, ids, 0).long()].float() * 1.7, 0.0).to(out)
    dst, mem = _view(torch.zeros((n, E), dtype=out, device="cuda"), pad, shift)
    before = mem.clone()
    got = tokens.embed(ids, w, 1.7, out=dst)
    assert torch.equal(got, ref)
    dst.copy_(before[shift:shift + n * (E + pad)].view(n, E + pad)[:, :E])
    assert torch.equal(mem.view(torch.uint8), before.view(torch.uint8))     # nothing beside the rows


@gpu
@pytest.mark.parametrize("table,out", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("E", [2, 3, 4, 5, 6, 9, 12, 15, 33, 301])
def test_embed_widths(E, table, out):
    """Every way that a row can end, there and in the gradient's few rows."""
    from paper_2302_03851_amd import tokens
    g = _gen(E)
    n, V = 130, 60
    w = torch.randn((V, E), generator=g, device="cuda").to(table)
    ids = _some_ids(n, V, g, False)
    dst, mem = _view(torch.zeros((n, E), dtype=out, device="cuda"), 1, 1)
    before = mem.clone()
    tokens.embed(ids, w, -0.3, out=dst)
    assert torch.equal(dst, (w[ids.long()].float() * -0.3).to(out))
    dst.zero_()
    assert torch.equal(mem.view(torch.uint8), before.view(torch.uint8))
    dout = torch.randn((n, E), generator=g, device="cuda").to(table)
    old = torch.randn((V, E), generator=g, device="cuda").to(out)
    _grad_check(ids, dout, V, 2.0, out, tokens.embed_grad(ids, dout, V, 2.0, out=old.clone(), accumulate=True), old)


@gpu
def test_embed_empty_and_values():
    from paper_2302_03851_amd import tokens
    w = torch.tensor([[1.0, -INF], [float("nan"), 3.0]], device="cuda")
    ids = torch.tensor([1, 0, -1], dtype=torch.int32, device="cuda")
    got = tokens.embed(ids, w, 2.0)
    assert torch.isnan(got[0, 0]) and got[0, 1] == 6 and got[1, 0] == 2 and got[1, 1] == -INF and not got[2].any()
    assert tokens.embed(ids[:0], w).shape == (0, 2)


@gpu
def test_embed_offsets_past_32_bits():
    """Rows beyond 2^31 and 2^32 elements, read, written and summed into."""
    from paper_2302_03851_amd import tokens
    E, far = 8, 1 << 31
    mem = torch.empty(2 * far + E, dtype=BF16, device="cuda")
    w = mem.as_strided((3, E), (far, 1))
    w.copy_(torch.arange(24, device="cuda").view(3, E))
    ids = torch.tensor([2, 0, 1, 2], dtype=torch.int32, device="cuda")
    assert torch.equal(tokens.embed(ids, w), w[ids.long()])
    x = tokens.embed(ids, w, dtype=F32)
    tokens.embed_grad(ids, x, 3, 0.5, out=w)
    ref = torch.stack([x[1] * 0.5, x[2] * 0.5, x[0]]).to(BF16)
    assert torch.equal(w, ref)
    tokens.embed(ids[:3], x[:3].contiguous(), 1.0, out=w)     # three rows of x, far apart
    assert torch.equal(w, x[ids[:3].long().clamp(max=2)].to(BF16))


def _grad_check(ids, dout, V, scale, out_dtype, got, old=None):
    """Any order of the terms, the scale, the addition and the rounding."""
    there = (ids >= 0) & (ids < V)
    at, d = ids[there].long(), dout[there].double()
    k = torch.bincount(at, minlength=V).double()
    often = k.argmax()                                  # its rows by themselves: index_add_ takes very long over them
    rest, own = d[at != often], d[at == often]

    def sums(rows, one):
        return torch.zeros((V, dout.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, at[at != often], rows).index_copy_(
            0, often[None], one.sum(0, keepdim=True))

    ref, mag = sums(rest, own) * scale, sums(rest.abs(), own.abs()) * abs(scale)
    if old is not None:
        ref += old.double()
    _close(got, ref, (k[:, None] + 2) * U * mag + 2 * U * ref.abs() + _half_ulp(ref, out_dtype) * 1.01 + 1e-40)
    return k


GRADS = [(0, 5, 8), (1, 1, 1), (3, 2, 7), (112, 50, 64), (700, 1000, 100), (1627, 300, 128), (4097, 33, 40),
         (9000, 70000, 16), (20000, 513, 33), (33000, 2, 264)]


@gpu
@pytest.mark.parametrize("src,dst", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,V,E", GRADS)
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad(n, V, E, src, dst, accumulate):
    from paper_2302_03851_amd import tokens
    g = _gen(n + V)
    ids = _some_ids(n, V, g, n > 3)
    dout = torch.randn((n, E), generator=g, device="cuda").to(src)
    old = torch.randn((V, E), generator=g, device="cuda").to(dst)
    runs = []
    for _ in range(2):
        out = old.clone() if accumulate else torch.full((V, E), float("nan"), dtype=dst, device="cuda")
        runs.append(tokens.embed_grad(ids, dout, V, -1.3, out=out, accumulate=accumulate))
    assert torch.equal(runs[0].view(torch.uint8), runs[1].view(torch.uint8))
    k = _grad_check(ids, dout, V, -1.3, dst, runs[0], old if accumulate else None)
    if accumulate:
        assert torch.equal(runs[0][k == 0], old[k == 0])


@gpu
@pytest.mark.parametrize("src,dst", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("n", [1024, 1025, 2048, 2049, 4096, 4097, 32768, 32769, 65536, 65537, 131073])
@pytest.mark.parametrize("E", [3, 6, 255, 300])
def test_embed_grad_sizes(n, E, src, dst):
    """At the sizes where the sort and the columns' split change, a third of the ids one word."""
    from paper_2302_03851_amd import tokens
    g = _gen(n + E)
    V = 3001
    ids = _some_ids(n, V, g, True)
    ids[1::3] = 77
    dout = torch.randn((n, E), generator=g, device="cuda").to(src)
    old = torch.randn((V, E), generator=g, device="cuda").to(dst)
    got = [tokens.embed_grad(ids, dout, V, 0.5, out=old.clone(), accumulate=True) for _ in range(2)]
    assert torch.equal(got[0].view(torch.uint8), got[1].view(torch.uint8))
    _grad_check(ids, dout, V, 0.5, dst, got[0], old)
    _grad_check(ids, dout, V, 0.5, dst, tokens.embed_grad(ids, dout, V, 0.5, dtype=dst))


@gpu
@pytest.mark.parametrize("n,src,dst", [(300, F32, BF16), (4096, BF16, F32), (5000, F32, F32), (70000, BF16, BF16)])
@pytest.mark.parametrize("E", [511, 512, 513, 1032, 2049])
def test_embed_grad_wide(n, E, src, dst):
    """Rows of more columns than a wave takes at a time, a third of the ids one word."""
    from paper_2302_03851_amd import tokens
    g = _gen(n + E)
    V = 3001
    ids = _some_ids(n, V, g, True)
    ids[1::3] = 77
    dout = torch.randn((n, E), generator=g, device="cuda").to(src)
    old = torch.randn((V, E), generator=g, device="cuda").to(dst)
    got = [tokens.embed_grad(ids, dout, V, 0.5, out=old.clone(), accumulate=True) for _ in range(2)]
    assert torch.equal(got[0].view(torch.uint8), got[1].view(torch.uint8))
    _grad_check(ids, dout, V, 0.5, dst, got[0], old)
    _grad_check(ids, dout, V, 0.5, dst, tokens.embed_grad(ids, dout, V, 0.5, dtype=dst))


@gpu
@pytest.mark.parametrize("n", [1, 64, 3000, 5000, 70000])
@pytest.mark.parametrize("kind", ["same", "two", "none", "ordered", "falling"])
def test_embed_grad_runs(n, kind):
    """Words with all the rows, with half of them, no words, and one row each."""
    from paper_2302_03851_amd import tokens
    V, E = 70001, 24
    i = torch.arange(n, device="cuda", dtype=torch.int32)
    ids = {"same": i * 0 + 69999, "two": (i % 2) * 70000, "none": i * 0 - 1, "ordered": i, "falling": 70000 - i}[kind]
    dout = torch.randn((n, E), generator=_gen(n), device="cuda")
    got = tokens.embed_grad(ids, dout, V)
    _grad_check(ids, dout, V, 1.0, F32, got)


@gpu
@pytest.mark.parametrize("n,V,E,pad,shift", [(500, 60, 64, 8, 0), (500, 60, 65, 3, 1), (6000, 900, 64, 8, 8), (6000, 900, 7, 1, 1)])
def test_embed_grad_strides(n, V, E, pad, shift):
    """Padded and shifted rows on both sides; NaN between them stays out and stays there."""
    from paper_2302_03851_amd import tokens
    g = _gen(5)
    ids = _some_ids(n, V, g, True)
    dout, _ = _view(torch.randn((n, E), generator=g, device="cuda"), pad, shift)
    out, mem = _view(torch.zeros((V, E), device="cuda"), pad, shift)
    before = mem.clone()
    tokens.embed_grad(ids, dout, V, out=out)
    _grad_check(ids, dout, V, 1.0, F32, out)
    out.copy_(before[shift:shift + V * (E + pad)].view(V, E + pad)[:, :E])
    assert torch.equal(mem.view(torch.uint8), before.view(torch.uint8))


@gpu
def test_embed_grad_differences():
    """sum(dout * embed(W)) is linear in W: its differences are the gradient's products."""
    from paper_2302_03851_amd import tokens
    g = _gen(9)
    V, E, n = 40, 24, 300
    ids = _some_ids(n, V, g, True)
    w = torch.randn((V, E), generator=g, device="cuda")
    dout = torch.randn((n, E), generator=g, device="cuda")
    d = tokens.embed_grad(ids, dout, V, 0.7).double()
    for _ in range(5):
        step = torch.randn((V, E), generator=g, device="cuda")
        f = [(tokens.embed(ids, w + s * step, 0.7).double() * dout.double()).sum() for s in (1, -1)]
        mag = (dout.double().abs() * 4).sum() * 0.7 * 8 * U      # the two lookups' roundings, |w| + |step| below 4 + 4 on the whole
        assert abs(float((f[0] - f[1]) / 2 - (d * step.double()).sum())) <= float(mag) + 1e-5 * float(d.abs().max())


# ---- log probabilities -------------------------------------------------------


def _rows(kind, n, V, dtype, g):
    x = 3 * torch.randn((n, V), generator=g, device="cuda")
    if kind == "masked":
        x[torch.rand((n, V), generator=g, device="cuda") < 0.6] = -INF
        x[0] = -INF                                    # nothing left
        if n > 1:
            x[1] = -INF
            x[1, V // 2] = 1.5                         # one left
        if n > 2:
            x[2, V // 3:] = -INF
    elif kind == "ties":
        x = x.div(3).round()
        x[0] = 0.25
        if n > 1:
            x[1] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0)
    elif kind == "lowest":
        x[:] = torch.finfo(dtype).min
        x[n // 2:, V // 2] = torch.finfo(dtype).max
    elif kind == "rising":
        x = torch.arange(V, device="cuda", dtype=F32).mul(8.0 / V).repeat(n, 1)
    elif kind == "falling":
        x = torch.arange(V, 0, -1, device="cuda", dtype=F32).mul(8.0 / V).repeat(n, 1)
    elif kind == "broken":
        x[0, V // 2] = float("nan")
        if n > 1:
            x[1, V - 1] = INF
        if n > 2:
            x[2] = float("nan")
        if n > 3:
            x[3, ::3] = float("nan")
            x[3, 1::3] = -INF
    return x.to(dtype)


def _reference(x, ids, T):
    """Per row in 64 bits: lp, entropy, m, l and the tolerance of l."""
    x = x.double()
    m = x.amax(1, keepdim=True)
    ref = torch.where(m == -INF, 0.0, m)
    y = (x - ref) / T
    e = torch.exp(y)
    S = e.sum(1, keepdim=True)
    empty = S == 0
    l = torch.where(empty, 0.0, torch.log(S))
    lp = torch.where(empty, -INF, y - l)
    p = torch.exp(lp)
    h = -torch.where(p > 0, p * lp, torch.where(torch.isnan(p), p, 0.0)).sum(1)
    w = torch.where(p > 0, p * y.abs(), 0.0).sum(1, keepdim=True)
    V = x.shape[1]
    tol_l = (V / 64 + 24 + 4 * w) * U + 4 * U * l.abs()
    tol_h = tol_l[:, 0] + (V / 64 + 16) * U * h.abs() + (torch.where(p > 0, p * 8 * U * (1 + y.abs()) * (1 + y.abs()), 0.0)).sum(1)
    return lp, p, y, h, m, l, tol_l, tol_h


def _check_logprobs(x, ids, T, top, r):
    n, V = x.shape
    lp, p, y, h, m, l, tol_l, tol_h = _reference(x, ids, T)
    there = torch.ones(n, dtype=torch.bool, device="cuda") if ids is None else (ids >= 0) & (ids < V)
    broken = torch.isnan(l[:, 0])
    tol_lp = tol_l + 4 * U * (torch.where(torch.isfinite(y), y.abs(), 0.0) + torch.where(torch.isfinite(lp), lp.abs(), 0.0))
    lp = lp.float().double()       # -inf past fp32's range
    if ids is not None:
        at = torch.where(there, ids, 0).long()[:, None]
        _close(r.logprob, torch.where(there, lp.gather(1, at)[:, 0], 0.0), tol_lp.gather(1, at)[:, 0])
    else:
        assert r.logprob is None
    _close(r.entropy, torch.where(there, h, 0.0), tol_h)
    stats = torch.cat([torch.where(broken[:, None], float("nan"), m), l], 1)
    _close(r.stats, torch.where(there[:, None], stats, 0.0), torch.cat([0 * tol_l, tol_l], 1))
    # the list: by value, then by index; no NaN, nothing masked out
    xs = x.float() + 0.0
    key = torch.where(torch.isnan(xs), -INF, xs)
    order = torch.sort(key, dim=1, descending=True, stable=True)
    k = min(top, V)
    want = torch.full((n, top), -1, dtype=torch.int64, device="cuda")
    want[:, :k] = torch.where((order.values[:, :k] > -INF) & there[:, None], order.indices[:, :k], -1)
    assert torch.equal(r.top_ids.long(), want)
    _close(r.top_logprobs, torch.where(want < 0, -INF, lp.gather(1, want.clamp(min=0))), tol_lp.gather(1, want.clamp(min=0)))


def _given(n, V, g):
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    for k, bad in enumerate((-1, V, -2 ** 31, 2 ** 31 - 1)):
        ids[k + 4::9] = bad
    return ids


SIZES = [(1, 1), (3, 2), (5, 7), (4, 64), (9, 65), (6, 513), (30, 1000), (4, 4099), (5, 20000), (3, 70001)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("kind,top,T", [("plain", 0, 1.0), ("plain", 5, 0.7), ("masked", 20, 1.0), ("ties", 64, 2.0),
                                        ("ties", 1, 1.0), ("lowest", 3, 1.0), ("rising", 64, 1.0), ("falling", 33, 1.0),
                                        ("broken", 8, 1.0)])
def test_logprobs(n, V, dtype, kind, top, T):
    from paper_2302_03851_amd import tokens
    g = _gen(V + top)
    x = _rows(kind, n, V, dtype, g)
    ids = _given(n, V, g)
    runs = [tokens.logprobs(x, ids, T, top) for _ in range(2)]
    for a, b in zip(*runs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    _check_logprobs(x, ids, T, top, runs[0])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", [(1, 131072), (2, 131071), (70, 33000), (600, 9001), (1, 300007)])
@pytest.mark.parametrize("top", [0, 50])
def test_logprobs_split_rows(n, V, dtype, top):
    """Few long rows and many, without given tokens, in views with odd strides."""
    from paper_2302_03851_amd import tokens
    x, _ = _view(_rows("plain", n, V, dtype, _gen(V)), 5, 3)
    _check_logprobs(x, None, 1.3, top, tokens.logprobs(x, None, 1.3, top))


@gpu
@pytest.mark.parametrize("n,V,dtype", [(2048, 2049, BF16), (2100, 8191, BF16), (2049, 1025, F32), (511, 16385, BF16),
                                       (300, 20001, F32), (260, 140001, BF16), (255, 65537, BF16), (256, 65537, F32), (40, 65536, F32)])
@pytest.mark.parametrize("kind,top", [("masked", 0), ("masked", 31), ("ties", 32), ("broken", 33), ("plain", 63)])
def test_logprobs_shapes(n, V, dtype, kind, top):
    """Every number of waves to a row, at every length of the list."""
    from paper_2302_03851_amd import tokens
    g = _gen(n + top)
    x = _rows(kind, n, V, dtype, g)
    ids = _given(n, V, g)
    _check_logprobs(x, ids, 1.1, top, tokens.logprobs(x, ids, 1.1, top))


@gpu
@pytest.mark.parametrize("n,V,dtype", [(520, 65536, BF16), (300, 65536, BF16), (520, 131072, BF16), (520, 40000, F32)])
@pytest.mark.parametrize("share", [0.004, 0.006, 0.01, 0.025])
@pytest.mark.parametrize("top", [5, 63])
def test_logprobs_capped(n, V, dtype, share, top):
    """A part of every row's logits at one cap: the first look through the groups fills the list of those that wait
    nearly or just whole, and the next one has more."""
    from paper_2302_03851_amd import tokens
    g = _gen(V + top + int(1000 * share))
    x = _rows("plain", n, V, dtype, g).clamp_(max=9.0)
    x[torch.rand((n, V), generator=g, device="cuda") < share] = 9.0
    _check_logprobs(x, None, 1.0, top, tokens.logprobs(x, None, 1.0, top))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["plain", "masked"])
def test_logprobs_longest(dtype, kind):
    """More parts of one row than a wave has lanes."""
    from paper_2302_03851_amd import tokens
    g = _gen(11)
    V = 10_000_003
    x = _rows(kind, 2, V, dtype, g)[1 if kind == "plain" else 0:][:1]
    ids = torch.tensor([V - 1], dtype=torch.int32, device="cuda")
    r = tokens.logprobs(x, ids, 1.0, 64)
    _check_logprobs(x, ids, 1.0, 64, r)
    one = torch.ones(1, device="cuda")
    ref, tol = _grad_reference(x, ids, 1.0, one, one)
    _close(tokens.logprobs_grad(x, ids, r.stats, r.entropy, one, one), ref, tol + 1.01 * _half_ulp(ref, dtype) + 1e-38)


@gpu
@pytest.mark.parametrize("kind", ["masked", "ties", "rising", "falling", "broken", "lowest"])
def test_logprobs_split_kinds(kind):
    """The odd rows of above where a row is long."""
    from paper_2302_03851_amd import tokens
    g = _gen(3)
    x = _rows(kind, 4, 131072, BF16, g)
    ids = torch.tensor([5, 131071, 0, 70000], dtype=torch.int32, device="cuda")
    _check_logprobs(x, ids, 1.0, 64, tokens.logprobs(x, ids, 1.0, 64))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", [(600, 1), (600, 30), (600, 5001), (600, 20001), (40, 70001)])
@pytest.mark.parametrize("T", [1.0, 0.7, 0.01])
def test_logprobs_peaked(n, V, dtype, T):
    """Rows that one logit decides: entropies and ln sums do not fall below 0, nor log probabilities rise above it."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = _rows("plain", n, V, F32, g)
    at = torch.randint(0, V, (n,), generator=g, device="cuda")
    x[torch.arange(n, device="cuda"), at] = 20 + 40 * torch.rand(n, generator=g, device="cuda")
    x = x.to(dtype)
    ids = at.to(torch.int32)
    r = tokens.logprobs(x, ids, T, 2)
    _check_logprobs(x, ids, T, 2, r)
    assert bool((r.entropy >= 0).all()) and bool((r.stats[:, 1] >= 0).all())
    assert bool((r.logprob <= 0).all()) and bool((r.top_logprobs <= 0).all())


FAR = [(-1e9, 1.0), (-1e9, 0.1), (-1e10, 1.0), (-1e10, 2.0), (-1e15, 1.0), (-1e20, 0.1), (-1e30, 1.0), (-1e30, 2.0), (1e10, 1.0),
       (1e10, 0.1), (-1e6, 1.0), (-6e5, 1.0), (8e5, 1.0), (0.0, 1e-6), (0.0, 1e-9), (0.0, 1e-30)]


def _far(value, n, V, dtype, g):
    """Ordinary logits with a finite number far away in their place: in whole rows, the first or the last part, here
    and there, everywhere but at one place, at one place; 0: none."""
    x = _rows("plain", n, V, F32, g)
    if value:
        x[0::6] = value
        x[1::6, :V // 2] = value
        x[2::6, V // 3:] = value
        x[3::6][torch.rand(x[3::6].shape, generator=g, device="cuda") < 0.6] = value
        one = x[4::6, V // 2].clone()
        x[4::6] = value
        x[4::6, V // 2] = one
        x[5::6, 2 * V // 3] = value
    return x.to(dtype)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", [(6, 1), (12, 7), (30, 1000), (2052, 2049), (516, 16385), (66, 20001), (6, 70001), (6, 131072)])
@pytest.mark.parametrize("value,T", FAR)
def test_logprobs_far(n, V, dtype, value, T):
    """Finite logits of every size have a distribution, at every temperature: forward and gradient."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = _far(value, n, V, dtype, g)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    r = tokens.logprobs(x, ids, T, 9)
    _check_logprobs(x, ids, T, 9, r)
    g1, g2 = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    if T < 1e-20:
        return                                         # the gradients pass fp32's range
    ref, tol = _grad_reference(x, ids, T, g1, g2)
    _close(tokens.logprobs_grad(x, ids, r.stats, r.entropy, g1, g2, T), ref, tol + 1.01 * _half_ulp(ref, dtype) + 1e-38)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logprobs_offsets_past_32_bits(dtype):
    """Rows 2^31 elements apart: forward, gradient and distillation."""
    from paper_2302_03851_amd import tokens
    V, far = 1001, 1 << 31
    x = torch.empty(2 * far + V, dtype=dtype, device="cuda").as_strided((3, V), (far, 1))
    dense = _rows("plain", 3, V, dtype, _gen(1))
    x.copy_(dense)
    ids = torch.tensor([7, 1000, 3], dtype=torch.int32, device="cuda")
    a, b = tokens.logprobs(x, ids, top=4), tokens.logprobs(dense, ids, top=4)
    for s, t in zip(a, b):
        assert torch.equal(s, t)
    one = torch.ones(3, device="cuda")
    q = torch.tensor([[1, 2], [3, -1], [1000, 0]], dtype=torch.int32, device="cuda"), torch.zeros((3, 2), device="cuda")
    ref = tokens.distill(dense, *q)
    got = tokens.distill(x, *q)
    assert torch.equal(got.loss, ref.loss) and torch.equal(got.dlogits, ref.dlogits)
    ref = tokens.logprobs_grad(dense, ids, b.stats, b.entropy, one, one)
    assert tokens.logprobs_grad(x, ids, a.stats, a.entropy, one, one, out=x) is x
    assert torch.equal(x, ref)


def _grad_reference(x, ids, T, g1, g2):
    lp, p, y, h, m, l, tol_l, tol_h = _reference(x, ids, T)
    n, V = x.shape
    there = (ids >= 0) & (ids < V)
    out = ~there | ((g1 == 0) & (g2 == 0)) | (m[:, 0] == -INF)
    one = torch.zeros_like(p).scatter_(1, torch.where(there, ids, 0).long()[:, None], 1.0)
    g1, g2 = g1.double()[:, None], g2.double()[:, None]
    plp = torch.where(p > 0, p * lp, torch.where(torch.isnan(p), p, 0.0))
    d = (g1 * (one - p) - g2 * (plp + p * h[:, None])) / T
    lpa = torch.where(p > 0, lp.abs(), 0.0)
    rel = tol_l + 8 * U * (1 + lpa)
    tol = p * (g1.abs() + g2.abs() * (lpa + h[:, None])) * (rel + 8 * U) + p * g2.abs() * (tol_h[:, None] + tol_l + 8 * U * (1 + lpa)) + 4 * U * g1.abs() * one
    return torch.where(out[:, None], 0.0, d), tol / T


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", SIZES + [(300, 10007), (600, 5003), (520, 8200), (2, 131071)])
@pytest.mark.parametrize("kind,T", [("plain", 0.7), ("masked", 1.0), ("lowest", 1.0), ("broken", 1.0), ("ties", 2.0)])
def test_logprobs_grad(n, V, dtype, kind, T):
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = _rows(kind, n, V, dtype, g)
    ids = _given(n, V, g)
    r = tokens.logprobs(x, ids, T)
    g1 = torch.randn(n, generator=g, device="cuda")
    g2 = torch.randn(n, generator=g, device="cuda")
    g1[2::5] = 0
    g2[2::10] = 0
    zero = torch.zeros_like(g1)
    for a, b in ((g1, g2), (g1, None), (None, g2)):
        ref, tol = _grad_reference(x, ids, T, zero if a is None else a, zero if b is None else b)
        got = tokens.logprobs_grad(x, ids, r.stats, r.entropy, a, b, T)
        _close(got, ref, tol + 1.01 * _half_ulp(ref, dtype) + 1e-38)
    # odd strides on both sides, and in place
    xv, _ = _view(x, 3, 1)
    ov, mem = _view(torch.zeros_like(x), 5, 2)
    before = mem.clone()
    full = tokens.logprobs_grad(x, ids, r.stats, r.entropy, g1, g2, T)
    tokens.logprobs_grad(xv, ids, r.stats, r.entropy, g1, g2, T, out=ov)
    assert torch.equal(ov.contiguous().view(torch.uint8), full.view(torch.uint8))
    ov.zero_()
    before[2:2 + n * (V + 5)].view(n, V + 5)[:, :V] = 0
    assert torch.equal(mem.view(torch.uint8), before.view(torch.uint8))
    tokens.logprobs_grad(x, ids, r.stats, r.entropy, g1, g2, T, out=x)
    assert torch.equal(x.view(torch.uint8), full.view(torch.uint8))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [2001, 9001])
def test_logprobs_grad_small(V, dtype):
    """Probabilities on both sides of the least normal number, whose gradients the temperature lifts above it."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    n, T = 6, 0.1
    x = (-8.6 - 0.8 * torch.rand((n, V), generator=g, device="cuda"))
    x[:, V // 2] = 0.5 * torch.rand(n, generator=g, device="cuda")
    x = x.to(dtype)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    r = tokens.logprobs(x, ids, T)
    g1, g2 = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    ref, tol = _grad_reference(x, ids, T, g1, g2)
    _close(tokens.logprobs_grad(x, ids, r.stats, r.entropy, g1, g2, T), ref, tol + 1.01 * _half_ulp(ref, dtype) + 1e-38)


@gpu
def test_logprobs_grad_differences():
    """Central differences of the 64-bit definition, step 1e-4: their own error
    is below 1e-7, fp32's below 1e-5 of the gradients' scale."""
    from paper_2302_03851_amd import tokens
    g = _gen(2)
    n, V, T = 3, 40, 0.8
    x = _rows("plain", n, V, F32, g)
    ids = torch.tensor([3, 0, 39], dtype=torch.int32, device="cuda")
    g1, g2 = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    r = tokens.logprobs(x, ids, T)
    d = tokens.logprobs_grad(x, ids, r.stats, r.entropy, g1, g2, T).double()

    def f(z):
        lp = torch.log_softmax(z / T, 1)
        given = lp.gather(1, ids.long()[:, None])[:, 0]
        return (g1.double() * given - g2.double() * (lp.exp() * lp).sum(1)).sum()

    for j in range(V):
        step = torch.zeros((n, V), dtype=torch.float64, device="cuda")
        step[:, j] = 1e-4
        for i in range(n):
            one = step.clone()
            one[torch.arange(n) != i] = 0
            diff = (f(x.double() + one) - f(x.double() - one)) / 2e-4
            assert abs(float(diff - d[i, j])) <= 1e-5 * (1 + float(g1.abs().max() + 5 * g2.abs().max())) / T


# ---- distillation ------------------------------------------------------------


def _teacher(n, V, K, g, kind):
    ids = torch.randint(0, V, (n, K), generator=g, device="cuda", dtype=torch.int32)      # equal ids among them
    u = 4 * torch.randn((n, K), generator=g, device="cuda")
    if kind == "distinct":
        ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] if V >= K else
                           torch.arange(K, device="cuda") % V for _ in range(n)]).to(torch.int32)
    if kind == "short":
        ids[:, K // 2:] = -1
        u[:, K // 2:] = float("nan")                   # behind a masked entry
        ids[::5, 0] = V
        u[1::5, 0] = -INF                              # no mass
        ids[2::5] = -1                                 # nothing listed
        u[3::5] = -INF                                 # nothing left
        u[4::5] = torch.finfo(F32).min
    return ids, u


def _distill_reference(x, ids, u, T, w):
    n, V = x.shape
    lp, p, y, h, m, l, tol_l, tol_h = _reference(x, None, T)
    there = (ids >= 0) & (ids < V)
    v = torch.where(there, u.double(), -INF)
    tm = v.amax(1, keepdim=True)
    e = torch.exp((v - torch.where(tm == -INF, 0.0, tm)) / T)
    S = e.sum(1, keepdim=True)
    out = (S[:, 0] == 0) | (w == 0)
    q = torch.zeros_like(p).scatter_add_(1, torch.where(there, ids, 0).long(), e / torch.where(S == 0, 1.0, S))
    lq = torch.where(q > 0, torch.log(torch.where(q > 0, q, 1.0)), 0.0)
    loss = torch.where(out, 0.0, T * T * torch.where(q > 0, q * (lq - lp), torch.where(torch.isnan(q), q, 0.0)).sum(1))
    loss = loss.float().double()   # inf past fp32's range
    empty = m[:, 0] == -INF
    w = w.double()[:, None]
    d = torch.where((out | empty)[:, None], 0.0, w * T * (p - q))
    lpa = torch.where((q > 0) & torch.isfinite(lp), lp.abs(), 0.0)
    ya = torch.where((q > 0) & torch.isfinite(y), y.abs(), 0.0)
    K = ids.shape[1]
    spread = torch.where(torch.isfinite(v), (v - tm).abs() / T, 0.0)
    q_rel = (K + 24) * U + (e / torch.where(S == 0, 1.0, S) * spread).sum(1, keepdim=True) * 8 * U
    dense_spread = torch.zeros_like(p).scatter_reduce_(1, torch.where(there, ids, 0).long(), torch.where(e > 0, spread, 0.0), "amax")
    q_rel = q_rel + 8 * U * dense_spread
    tol_loss = T * T * torch.where(q > 0, q * ((q_rel + 8 * U) * (lq.abs() + lpa + 1) + tol_l + 8 * U * (1 + ya + lpa)), 0.0).sum(1) * 1.01
    lpp = torch.where(p > 0, lp.abs(), 0.0)
    tol_d = w.abs() * T * (p * (tol_l + 8 * U * (2 + lpp)) + q * (q_rel + 8 * U))
    return loss, d, tol_loss + U * K * loss.abs(), tol_d


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", SIZES + [(40, 33000), (6, 131072), (3, 150001), (2, 300007)])
@pytest.mark.parametrize("kind,teacher,K,T", [("plain", "distinct", 16, 2.0), ("masked", "short", 9, 1.0),
                                              ("plain", "equal", 256, 0.7), ("lowest", "equal", 1, 1.0),
                                              ("broken", "distinct", 5, 1.0)])
def test_distill(n, V, dtype, kind, teacher, K, T):
    from paper_2302_03851_amd import tokens
    g = _gen(V + K)
    x = _rows(kind, n, V, dtype, g)
    ids, u = _teacher(n, V, K, g, teacher)
    w = torch.rand(n, generator=g, device="cuda") - 0.3
    w[3::7] = 0
    for weight in (None, w):
        ww = torch.ones_like(w) if weight is None else weight
        loss, d, tol_loss, tol_d = _distill_reference(x, ids, u, T, ww)
        runs = [tokens.distill(x, ids, u, T, weight) for _ in range(2)]
        for a, b in zip(*runs):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        _close(runs[0].loss, loss, tol_loss)
        _close(runs[0].dlogits, d, tol_d + 1.01 * _half_ulp(d, dtype) + 1e-38)
        alone = tokens.distill(x, ids, u, T, weight, grad=False)
        assert alone.dlogits is None and torch.equal(alone.loss.view(torch.uint8), runs[0].loss.view(torch.uint8))
    # odd strides on both sides, and in place
    xv, _ = _view(x, 3, 1)
    ov, mem = _view(torch.zeros_like(x), 5, 2)
    before = mem.clone()
    full = runs[0]
    got = tokens.distill(xv, ids, u, T, w, out=tokens.Distilled(torch.empty_like(loss, dtype=F32), ov))
    assert torch.equal(got.loss.view(torch.uint8), full.loss.view(torch.uint8))
    assert torch.equal(ov.contiguous().view(torch.uint8), full.dlogits.view(torch.uint8))
    ov.zero_()
    before[2:2 + n * (V + 5)].view(n, V + 5)[:, :V] = 0
    assert torch.equal(mem.view(torch.uint8), before.view(torch.uint8))
    tokens.distill(x, ids, u, T, w, out=tokens.Distilled(full.loss, x))
    assert torch.equal(x.view(torch.uint8), full.dlogits.view(torch.uint8))


def _check_distill(x, ids, u, T, weight, got):
    ww = torch.ones(x.shape[0], device="cuda") if weight is None else weight
    loss, d, tol_loss, tol_d = _distill_reference(x, ids, u, T, ww)
    _close(got.loss, loss, tol_loss)
    _close(got.dlogits, d, tol_d + 1.01 * _half_ulp(d, x.dtype) + 1e-38)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vectors", [64, 512, 1024, 2048, 4096, 8192, 16384])
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_distill_row_lengths(dtype, vectors, more):
    """About the lengths (in vectors of 16 bytes) at which a row is held by more threads or in more registers."""
    from paper_2302_03851_amd import tokens
    n, V = 5, vectors * (4 if dtype == F32 else 8) + more
    g = _gen(V)
    x = _rows("masked", n, V, dtype, g)
    ids, u = _teacher(n, V, 7, g, "equal")
    ids[:, 0] = V - 1
    got = tokens.distill(x, ids, u, 1.2)
    _check_distill(x, ids, u, 1.2, None, got)
    tokens.distill(x, ids, u, 1.2, out=tokens.Distilled(got.loss, x))
    assert torch.equal(x.view(torch.uint8), got.dlogits.view(torch.uint8))


@gpu
@pytest.mark.parametrize("n,V,dtype", [(700, 66001, BF16), (600, 33003, F32), (1100, 66001, BF16), (520, 131072, BF16),
                                       (1020, 33003, F32), (1100, 33000, F32), (520, 65536, F32), (200, 65536, BF16),
                                       (300, 40001, BF16), (140, 32767, F32)])
@pytest.mark.parametrize("kind", ["masked", "broken"])
def test_distill_many_long_rows(n, V, dtype, kind):
    """More long rows than work-groups take at a time, rows without weight and without a teacher among them."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = _rows(kind, n, V, dtype, g)
    ids, u = _teacher(n, V, 20, g, "short")
    w = torch.randn(n, generator=g, device="cuda")
    w[torch.rand(n, generator=g, device="cuda") < 0.4] = 0
    w[200:520] = 0
    w[-1] = 0
    full = tokens.distill(x, ids, u, 0.9, w)
    for i in range(0, n, 100):       # the reference a few rows at a time: it is in 64 bits
        part = tokens.Distilled(full.loss[i:i + 100], full.dlogits[i:i + 100])
        _check_distill(x[i:i + 100], ids[i:i + 100], u[i:i + 100], 0.9, w[i:i + 100], part)
    alone = tokens.distill(x, ids, u, 0.9, w, grad=False)
    assert torch.equal(alone.loss.view(torch.uint8), full.loss.view(torch.uint8))
    xv, _ = _view(x, 3, 1)
    got = tokens.distill(xv, ids, u, 0.9, w, out=tokens.Distilled(alone.loss, xv))
    assert torch.equal(got.loss.view(torch.uint8), full.loss.view(torch.uint8))
    assert torch.equal(xv.contiguous().view(torch.uint8), full.dlogits.view(torch.uint8))


@gpu
@pytest.mark.parametrize("n,V,dtype", [(1, 131072, BF16), (9, 65537, BF16), (70, 70001, BF16), (5, 32769, F32), (300, 40001, F32),
                                       (1, 3_000_001, BF16), (3, 2_000_003, F32), (400, 150001, BF16)])
@pytest.mark.parametrize("kind,teacher", [("masked", "short"), ("broken", "equal"), ("lowest", "distinct")])
def test_distill_split_rows(n, V, dtype, kind, teacher):
    """Rows that several work-groups take: the loss alone, strides, and in place, where listed tokens lie in other parts."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = _rows(kind, n, V, dtype, g)
    ids, u = _teacher(n, V, 11, g, teacher)
    ids[:, 1] = V - 1
    w = torch.randn(n, generator=g, device="cuda")
    w[1::6] = 0
    full = tokens.distill(x, ids, u, 1.7, w)
    for i in range(0, n, 100):
        part = tokens.Distilled(full.loss[i:i + 100], full.dlogits[i:i + 100])
        _check_distill(x[i:i + 100], ids[i:i + 100], u[i:i + 100], 1.7, w[i:i + 100], part)
    alone = tokens.distill(x, ids, u, 1.7, w, grad=False)
    assert torch.equal(alone.loss.view(torch.uint8), full.loss.view(torch.uint8))
    xv, mem = _view(x, 3, 1)
    before = mem.clone()
    got = tokens.distill(xv, ids, u, 1.7, w, out=tokens.Distilled(alone.loss, xv))
    assert torch.equal(got.loss.view(torch.uint8), full.loss.view(torch.uint8))
    assert torch.equal(xv.contiguous().view(torch.uint8), full.dlogits.view(torch.uint8))
    xv.copy_(x)
    assert torch.equal(mem.view(torch.uint8), before.view(torch.uint8))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", [(6, 7), (12, 200), (30, 1000), (12, 5001), (12, 12001), (150, 33001), (140, 65000), (1020, 33003), (6, 131072)])
@pytest.mark.parametrize("value,T", [(v, T) for v, T in FAR if T > 1e-20])
def test_distill_far(n, V, dtype, value, T):
    """As test_logprobs_far, in every layout of the rows."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = _far(value, n, V, dtype, g)
    ids, u = _teacher(n, V, 9, g, "equal")
    ids[:, 0] = V // 2
    _check_distill(x, ids, u, T, None, tokens.distill(x, ids, u, T))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", [(9, 1), (9, 200), (9, 9001), (9, 131072)])
@pytest.mark.parametrize("T", [1e-25, 1e-15, 1e18, 1e25])
def test_distill_temperatures(n, V, dtype, T):
    """Temperatures whose square leaves fp32's range, where the loss stays in it (infinite where it does not)."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = _rows("plain", n, V, dtype, g)
    ids, u = _teacher(n, V, 5, g, "equal")
    _check_distill(x, ids, u, T, None, tokens.distill(x, ids, u, T))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,V", [(6, 200), (6, 9001), (6, 131072)])
def test_distill_small(n, V, dtype):
    """Probabilities on both sides of the least normal number, whose gradients the weight lifts above it; listed tokens
    without mass among them."""
    from paper_2302_03851_amd import tokens
    g = _gen(V)
    x = -86 - 8 * torch.rand((n, V), generator=g, device="cuda")
    x[:, V // 2] = 0.5 * torch.rand(n, generator=g, device="cuda")
    x = x.to(dtype)
    ids, u = _teacher(n, V, 5, g, "distinct")
    u[:, 3:] = -INF
    w = torch.rand(n, generator=g, device="cuda") * 65536
    _check_distill(x, ids, u, 1.5, w, tokens.distill(x, ids, u, 1.5, w))
    x = (x.float() * 1.5).to(dtype)
    _check_distill(x, ids, u, 1.5, w, tokens.distill(x, ids, u, 1.5, w))


@gpu
def test_distill_differences():
    """Central differences of the 64-bit loss (as for the log probabilities)."""
    from paper_2302_03851_amd import tokens
    g = _gen(4)
    n, V, T = 2, 30, 1.5
    x = _rows("plain", n, V, F32, g)
    ids, u = _teacher(n, V, 6, g, "equal")
    w = torch.tensor([0.4, -1.1], device="cuda")
    d = tokens.distill(x, ids, u, T, w).dlogits.double()

    def f(z):
        q = torch.zeros((n, V), dtype=torch.float64, device="cuda").scatter_add_(1, ids.long(), torch.softmax(u.double() / T, 1))
        return (w.double() * T * T * (torch.xlogy(q, q) - q * torch.log_softmax(z / T, 1)).sum(1)).sum()

    for i in range(n):
        for j in range(V):
            step = torch.zeros((n, V), dtype=torch.float64, device="cuda")
            step[i, j] = 1e-4
            assert abs(float((f(x.double() + step) - f(x.double() - step)) / 2e-4 - d[i, j])) <= 1e-5


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_millions_of_rows(dtype):
    """More rows than one launch takes: the same bits as the rows by themselves."""
    from paper_2302_03851_amd import tokens
    g = _gen(21)
    n, V = (1 << 22) + 77, 5
    x = torch.randn((n, V), generator=g, device="cuda").to(dtype)
    ids = torch.randint(-1, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    q = torch.randint(-1, V, (n, 2), generator=g, device="cuda", dtype=torch.int32), torch.randn((n, 2), generator=g, device="cuda")
    w = torch.randn(n, generator=g, device="cuda")

    def rows(a, b):
        part = x[a:b].contiguous()
        r = tokens.logprobs(part, ids[a:b], 0.9, 2)
        d = tokens.logprobs_grad(part, ids[a:b], r.stats, r.entropy, w[a:b], w[a:b], 0.9)
        return [*r, d, *tokens.distill(part, q[0][a:b], q[1][a:b], 1.1, w[a:b])]

    whole = rows(0, n)
    for a, b in ((0, 1000), (1398000, 1399000), (2097000, 2098000), (2796000, 2797000), (n - 1000, n)):
        for s, t in zip(whole, rows(a, b)):
            assert torch.equal(s[a:b].contiguous().view(torch.uint8), t.view(torch.uint8))


def _room(gigabytes):
    """Skips where the card has less memory left."""
    import gc
    gc.collect()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 10 ** 9:
        pytest.skip(f"needs {gigabytes} GB of free device memory")


@gpu
def test_most_rows():
    """As many rows as 32 bits count, of one logit each, the same 1024 again and again: log probabilities, and the
    gradient in the logits' place, have the bits of those 1024 by themselves."""
    from paper_2302_03851_amd import tokens
    _room(80)
    n = 2 ** 31 - 1
    few = torch.arange(0x3f00, 0x4300, dtype=torch.int16, device="cuda").view(BF16).view(-1, 1)
    g1 = torch.arange(1024, device="cuda", dtype=F32) % 3
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ref = tokens.logprobs(few, ids[:1024])
    ref_d = tokens.logprobs_grad(few, ids[:1024], ref.stats, g_logprob=g1)

    def again(t):
        return t.repeat(n // 1024 + 1, *[1] * (t.dim() - 1))[:n]

    def check(got, one):
        assert torch.equal(got[:n // 1024 * 1024].view(-1, *one.shape).amax(0), one)
        assert torch.equal(got[:n // 1024 * 1024].view(-1, *one.shape).amin(0), one)
        assert torch.equal(got[n // 1024 * 1024:], one[:n % 1024])

    x = again(few).contiguous()
    r = tokens.logprobs(x, ids)
    check(r.logprob, ref.logprob)
    check(r.entropy, ref.entropy)
    check(r.stats, ref.stats)
    g1 = again(g1).contiguous()
    tokens.logprobs_grad(x, ids, r.stats, g_logprob=g1, out=x)
    check(x, ref_d)
    del x, ids, r, g1
    torch.cuda.empty_cache()


@gpu
def test_embed_grad_most_rows():
    """As many ids as 32 bits count.  Every product is 1; sums of them are exact up to 2^24, and less than 64 additions
    come after that in any tree of threads, chunks and parts: 64 U of the sum."""
    from paper_2302_03851_amd import tokens
    _room(100)
    n = 2 ** 31 - 1
    ids = torch.arange(n, dtype=torch.int32, device="cuda").remainder_(3)
    dout = torch.ones((n, 1), dtype=BF16, device="cuda")
    got = tokens.embed_grad(ids, dout, 4)[:, 0].double()
    ref = torch.tensor([(n + 2) // 3, (n + 1) // 3, n // 3, 0], dtype=torch.float64, device="cuda")
    assert float(((got - ref).abs() - 64 * U * ref).max()) <= 0
    del ids, dout
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("V,E,dtype", [(2 ** 24 + 3, 2050, F32), (2 ** 23 + 5, 4097, BF16)])
def test_embed_grad_largest_table(V, E, dtype):
    """Few ids into a table of more blocks of rows than work-groups that zero them (137 and 69 GB)."""
    from paper_2302_03851_amd import tokens
    _room(145)
    out = torch.empty((V, E), dtype=dtype, device="cuda")
    step = 2 ** 18
    for a in range(0, V, step):
        out[a:a + step].fill_(float("nan"))
    ids = torch.tensor([V - 1, 0, 2 ** 22, 2 ** 22 + 1, -1, V - 1, 2 ** 23 + 1], dtype=torch.int32, device="cuda")
    dout = torch.randint(-8, 8, (7, E), device="cuda", generator=_gen(1)).to(dtype)
    tokens.embed_grad(ids, dout, V, out=out)
    ref = {V - 1: dout[0] + dout[5], 0: dout[1], 2 ** 22: dout[2], 2 ** 22 + 1: dout[3], 2 ** 23 + 1: dout[6]}
    for v, row in ref.items():
        assert torch.equal(out[v], row)
        out[v] = 0
    for a in range(0, V, step):
        assert not out[a:a + step].any()
    del out
    torch.cuda.empty_cache()


# ---- streams and graphs ------------------------------------------------------


def _everything(seed):
    """Inputs of each operator and a function that runs them into fixed outputs."""
    from paper_2302_03851_amd import tokens
    g = _gen(seed)
    n, V, E, K = 700, 9001, 72, 12
    ids = _some_ids(n, V, g, True)
    w = torch.randn((V, E), generator=g, device="cuda")
    x = _rows("masked", n, V, BF16, g)
    q = _teacher(n, V, K, g, "short")
    g1 = torch.randn(n, generator=g, device="cuda")
    # a few long rows, and enough rows for every path of the table's gradient
    long = _rows("plain", 2, 100003, F32, g)
    many = torch.randint(0, V, (30000,), generator=g, device="cuda", dtype=torch.int32)
    dy = torch.randn((30000, 40), generator=g, device="cuda")

    def go():
        y = tokens.embed(ids, w, 0.3)
        dw = tokens.embed_grad(ids, y, V, 0.3)
        r = tokens.logprobs(x, ids, 0.9, 10)
        dx = tokens.logprobs_grad(x, ids, r.stats, r.entropy, g1, g1, 0.9)
        t = tokens.distill(x, *q, 1.4, g1)
        s = tokens.logprobs(long, None, 1.0, 7)
        dm = tokens.embed_grad(many, dy, V)
        return [y, dw, *r, dx, *t, *s[1:], dm]

    return go


def _larger(seed):
    """As _everything, for the paths of many ids and of many long rows."""
    from paper_2302_03851_amd import tokens
    g = _gen(seed)
    V, n = 66001, 300
    ids = _some_ids(70000, V, g, True)
    dy = torch.randn((70000, 36), generator=g, device="cuda").to(BF16)
    x = _rows("masked", n, V, BF16, g)
    q = _teacher(n, V, 12, g, "short")
    w = torch.randn(n, generator=g, device="cuda")

    def go():
        return [tokens.embed_grad(ids, dy, V), *tokens.distill(x, *q, 1.4, w), *tokens.logprobs(x, None, 1.0, 40)[1:]]

    return go


def _same(a, b):
    return all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(a, b))


@gpu
def test_tokens_streams():
    """The current stream's work, several streams at once."""
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
@pytest.mark.parametrize("calls", [_everything, _larger])
def test_tokens_captured(calls):
    """All calls in one HIP graph, replayed between eager calls."""
    go = calls(7)
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


@gpu
def test_word_model_example():
    """Every operator in one program: both of its losses fall."""
    from examples import word_model
    said = []
    distilled, tuned = word_model.run(instances=6, vocab=1003, steps=12, report=said.append)
    assert np.isfinite(distilled + tuned).all() and min(distilled) >= 0 and min(tuned) >= 0
    assert distilled[-1] < 0.7 * distilled[0] and tuned[-1] < 0.5 * tuned[0]
    assert len(said) == 6


# ---- refusals ----------------------------------------------------------------

A = 1 << 20      # addresses that are never read: every call below is refused first


def _embed(**k):
    a = dict(ids=A, n=4, table=2 * A, td=L.F32, V=10, E=8, ts=8, scale=1.0, out=3 * A, od=L.F32, os=8)
    a.update(k)
    return L.load().edb_embed(*a.values(), None)


def _embed_grad(**k):
    a = dict(ids=A, n=4, dout=2 * A, dd=L.F32, V=10, E=8, ds=8, scale=1.0, acc=0, out=3 * A, od=L.F32, os=8, ws=4 * A, wb=1 << 40)
    a.update(k)
    return L.load().edb_embed_grad(*a.values(), None)


def _logprobs(**k):
    a = dict(x=A, d=L.F32, n=4, V=10, s=10, ids=2 * A, T=1.0, top=2, lp=3 * A, h=3 * A, st=3 * A, ti=3 * A, tl=3 * A, ws=4 * A, wb=1 << 40)
    a.update(k)
    return L.load().edb_logprobs(*a.values(), None)


def _lp_grad(**k):
    a = dict(x=A, d=L.F32, n=4, V=10, s=10, ids=2 * A, T=1.0, st=3 * A, h=3 * A, g1=3 * A, g2=3 * A, out=4 * A, os=10)
    a.update(k)
    return L.load().edb_logprobs_grad(*a.values(), None)


def _distill(**k):
    a = dict(x=A, d=L.F32, n=4, V=10, s=10, ti=2 * A, tl=3 * A, top=2, T=1.0, w=3 * A, loss=3 * A, out=4 * A, os=10,
             ws=5 * A, wb=1 << 40)
    a.update(k)
    return L.load().edb_distill(*a.values(), None)


INVALID, UNSUPPORTED = L.EDB_ERR_INVALID, L.EDB_ERR_UNSUPPORTED
ROWS_BAD = [(dict(x=None), INVALID), (dict(d=7), INVALID), (dict(n=-1), INVALID), (dict(V=0), INVALID), (dict(s=9), INVALID),
            (dict(s=1 << 47), INVALID), (dict(V=(1 << 30) + 1, s=1 << 31, os=1 << 31), UNSUPPORTED), (dict(T=0.0), INVALID),
            (dict(T=-1.0), INVALID), (dict(T=INF), INVALID), (dict(T=float("nan")), INVALID), (dict(T=1e-45), INVALID),
            (dict(x=A + 2), INVALID), (dict(d=L.BF16, x=A + 1), INVALID)]
REFUSED = (
    [(_embed, k, e) for k, e in [
        (dict(ids=None), INVALID), (dict(table=None), INVALID), (dict(out=None), INVALID), (dict(td=2), INVALID),
        (dict(od=-1), INVALID), (dict(n=-1), INVALID), (dict(V=0), INVALID), (dict(E=0), INVALID), (dict(ts=7), INVALID),
        (dict(os=7), INVALID), (dict(scale=INF), INVALID), (dict(V=(1 << 30) + 1), UNSUPPORTED),
        (dict(E=(1 << 20) + 1, ts=1 << 21, os=1 << 21), UNSUPPORTED), (dict(table=2 * A + 2), INVALID), (dict(out=3 * A + 1), INVALID),
        (dict(out=2 * A + 64), INVALID), (dict(n=1 << 30, E=1 << 10, ts=1 << 10, os=1 << 10, out=1 << 45), UNSUPPORTED)]]
    + [(_embed_grad, k, e) for k, e in [
        (dict(ids=None), INVALID), (dict(dout=None), INVALID), (dict(out=None), INVALID), (dict(out=None, n=0), INVALID),
        (dict(dd=3), INVALID), (dict(od=3), INVALID), (dict(n=-1), INVALID), (dict(V=0), INVALID), (dict(E=0), INVALID),
        (dict(ds=7), INVALID), (dict(os=7), INVALID), (dict(scale=float("nan")), INVALID), (dict(out=2 * A + 64), INVALID),
        (dict(dout=2 * A + 2), INVALID), (dict(n=5000, wb=0), INVALID), (dict(n=5000, ws=None), INVALID),
        (dict(n=5000, ws=4 * A + 8), INVALID)]]
    + [(_logprobs, k, e) for k, e in [(q, e) for q, e in ROWS_BAD if "os" not in q] + [
        (dict(top=-1), UNSUPPORTED), (dict(top=65), UNSUPPORTED), (dict(ids=None), INVALID), (dict(ti=None), INVALID),
        (dict(tl=None), INVALID), (dict(n=1, V=100000, s=100000, wb=0), INVALID), (dict(n=1, V=100000, s=100000, ws=None), INVALID),
        (dict(n=1, V=100000, s=100000, ws=4 * A + 4), INVALID)]]
    + [(_lp_grad, k, e) for k, e in ROWS_BAD + [
        (dict(ids=None), INVALID), (dict(st=None), INVALID), (dict(h=None), INVALID), (dict(out=None), INVALID), (dict(os=9), INVALID),
        (dict(out=A + 4), INVALID), (dict(out=A, os=12), INVALID), (dict(out=4 * A + 2), INVALID)]]
    + [(_distill, k, e) for k, e in ROWS_BAD + [
        (dict(ti=None), INVALID), (dict(tl=None), INVALID), (dict(loss=None), INVALID), (dict(top=0), UNSUPPORTED),
        (dict(top=257), UNSUPPORTED), (dict(os=9), INVALID), (dict(out=A + 4), INVALID), (dict(out=A, os=12), INVALID),
        (dict(n=1, V=200000, s=200000, os=200000, wb=0), INVALID), (dict(n=1, V=200000, s=200000, os=200000, ws=None), INVALID),
        (dict(n=1, V=200000, s=200000, os=200000, ws=5 * A + 8), INVALID)]])


@pytest.mark.parametrize("call,changed,status", REFUSED, ids=[f"{f.__name__[1:]}-{i}" for i, (f, _, _) in enumerate(REFUSED)])
def test_refusals(call, changed, status):
    """Refused on the host, with a message, before any launch (no GPU needed)."""
    assert call(**changed) == status
    assert L.load().edb_last_error()


# arguments apart from each other; n = 4, V = 10, rows 40 bytes and 1 MB apart in `far`
LP_APART = dict(lp=3 * A, h=3 * A + 64, st=3 * A + 128, ti=3 * A + 192, tl=3 * A + 256)
DI_APART = dict(loss=6 * A)
OVERLAPS = (
    [(_embed, k) for k in [dict(out=A + 8), dict(out=A - 32 * 4 + 4), dict(out=A - 256 - 28, os=64), dict(ids=2), dict(ids=A + 1)]]
    + [(_embed_grad, k) for k in [dict(out=A - 316), dict(out=A + 12), dict(ids=A + 2), dict(n=5000, ids=4 * A + 160),
                                  dict(n=5000, out=4 * A - 64), dict(n=5000, dout=4 * A + 16, out=64 * A),
                                  dict(n=5000, dout=4 * A - 159996, out=64 * A)]]
    + [(_logprobs, dict(LP_APART, **k)) for k in [
        dict(lp=A), dict(h=A + 156), dict(st=A - 28), dict(ti=A + 40), dict(tl=A + 128), dict(lp=2 * A + 12), dict(h=2 * A - 12),
        dict(h=3 * A + 12), dict(st=3 * A + 76), dict(tl=3 * A + 220), dict(s=A // 4, lp=2 * A + 36, ids=9 * A),
        dict(s=A // 4, lp=4 * A - 12, ids=9 * A), dict(lp=3 * A + 1), dict(h=3 * A + 66), dict(st=3 * A + 131), dict(ti=3 * A + 193),
        dict(tl=3 * A + 258), dict(ids=2 * A + 2), dict(n=1, V=100000, s=100000, ids=9 * A, ws=3 * A),
        dict(n=1, V=100000, s=100000, ids=9 * A, ws=A + 399984), dict(n=1, V=100000, s=100000, ids=4 * A + 64)]]
    + [(_lp_grad, k) for k in [dict(out=2 * A - 156), dict(out=3 * A + 28), dict(out=2 * A + 12), dict(ids=2 * A + 1), dict(st=3 * A + 2),
                               dict(h=3 * A + 1), dict(g1=3 * A + 3), dict(g2=3 * A + 2), dict(g1=4 * A + 144),
                               dict(g2=4 * A + 36, os=20), dict(h=4 * A - 12), dict(st=4 * A - 28)]]
    + [(_distill, dict(DI_APART, **k)) for k in [
        dict(loss=3 * A), dict(loss=A + 156), dict(loss=2 * A + 28), dict(loss=4 * A + 120), dict(w=4 * A + 8), dict(ti=4 * A - 28),
        dict(tl=4 * A + 156), dict(loss=6 * A + 2), dict(w=3 * A + 1), dict(ti=2 * A + 2), dict(tl=3 * A + 2),
        dict(n=1, V=200000, s=200000, os=200000, ws=6 * A), dict(n=1, V=200000, s=200000, os=200000, ws=2 * A),
        dict(n=1, V=200000, s=200000, os=200000, ws=4 * A + 799984)]])


@pytest.mark.parametrize("call,changed", OVERLAPS, ids=[f"{f.__name__[1:]}-{i}" for i, (f, _) in enumerate(OVERLAPS)])
def test_refused_overlaps(call, changed):
    """Results and workspaces in another argument's memory, by one word at either end, and arrays off their words."""
    assert call(**changed) == INVALID


BESIDE = [(_embed, dict(table=A, ts=30, os=30, out=A + k, ids=9 * A)) for k in (28, -28, 92, 4 * 30 * 3 + 28)] + \
         [(_embed_grad, dict(dout=A, ds=30, os=30, out=A + k, ids=9 * A)) for k in (28, -28, 92)] + \
         [(_lp_grad, dict(s=30, os=30, out=A + k)) for k in (36, -36, 84)] + \
         [(_distill, dict(DI_APART, s=30, os=30, out=A + k)) for k in (36, -36, 84)]


@pytest.mark.parametrize("call,changed", BESIDE, ids=[f"{f.__name__[1:]}-{i}" for i, (f, _) in enumerate(BESIDE)])
def test_refused_columns(call, changed):
    """Columns of one buffer that share one with the others."""
    assert call(**changed) == INVALID


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E,gap", [(10, 0), (513, 1), (64, 0), (4099, 0)])
def test_columns_beside(E, gap, dtype):
    """Inputs and results as columns of one buffer, right beside each other, give the bits of separate ones."""
    from paper_2302_03851_amd import tokens
    g = _gen(E)
    n, V = 70, 70
    buf = torch.full((n, 3 * (E + gap)), float("nan"), dtype=dtype, device="cuda")
    left, mid, right = (buf[:, i * (E + gap):i * (E + gap) + E] for i in range(3))
    one = torch.randn((n, E), generator=g, device="cuda").to(dtype)
    ids = _some_ids(n, min(V, E), g, True)
    u = _teacher(n, E, 5, g, "equal")
    w = torch.rand(n, generator=g, device="cuda")
    r = tokens.logprobs(one, ids)
    loss = torch.empty(n, device="cuda")
    for x, y in ((mid, right), (mid, left), (left, right), (right, left)):
        for f, ref in ((lambda: tokens.embed(ids, x, 0.7, out=y), tokens.embed(ids, one, 0.7)),
                       (lambda: tokens.embed_grad(ids, x, V, 0.7, out=y), tokens.embed_grad(ids, one, V, 0.7, dtype=dtype)),
                       (lambda: tokens.logprobs_grad(x, ids, r.stats, r.entropy, w, w, out=y),
                        tokens.logprobs_grad(one, ids, r.stats, r.entropy, w, w)),
                       (lambda: tokens.distill(x, *u, 1.3, w, out=tokens.Distilled(loss, y)).dlogits,
                        tokens.distill(one, *u, 1.3, w).dlogits)):
            buf.fill_(float("nan"))
            x.copy_(one)
            f()
            assert torch.equal(y, ref) and torch.equal(x, one)
            x.fill_(float("nan"))
            y.fill_(float("nan"))
            assert bool(torch.isnan(buf).all())


@gpu
def test_arrays_between_rows():
    """Results may lie between the rows of a matrix, right up to them."""
    from paper_2302_03851_amd import tokens
    g = _gen(8)
    n, V = 3, 10
    mem = torch.zeros(200, device="cuda")
    x = mem.as_strided((n, V), (60, 1), 8)
    x.copy_(torch.randn((n, V), generator=g, device="cuda"))
    ids = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    ref = tokens.logprobs(x.contiguous(), ids, top=2)
    out = tokens.LogProbs(mem[5:8], mem[18:21], mem[21:27].view(3, 2), mem[62:68].view(torch.int32).view(3, 2), mem[138:144].view(3, 2))
    got = tokens.logprobs(x, ids, top=2, out=out)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


@pytest.mark.parametrize("call", [_logprobs, _lp_grad, _distill])
def test_refused_temperatures(call):
    """Where 1 / T is finite and the exponents' factor log2(e) / T is not."""
    for n in (0, 4):
        assert call(n=n, T=3e-39) == INVALID and call(n=n, T=4.2e-39) == INVALID
    assert call(n=0, T=4.3e-39) == L.EDB_OK and call(n=0, T=3.4e38) == L.EDB_OK


@pytest.mark.parametrize("call", [_embed, _logprobs, _lp_grad, _distill])
def test_nothing_to_do(call):
    assert call(n=0) == L.EDB_OK


def test_workspace_sizes():
    lib, nb = L.load(), C.c_int64(-1)
    assert lib.edb_logprobs_bytes(5, 1000, L.BF16, 3, C.byref(nb)) == L.EDB_OK and nb.value >= 0
    assert lib.edb_embed_grad_bytes(9000, 500, 64, C.byref(nb)) == L.EDB_OK and nb.value > 0
    assert lib.edb_logprobs_bytes(1, 1 << 30, L.F32, 64, C.byref(nb)) == L.EDB_OK and nb.value > 0
    assert lib.edb_logprobs_bytes(5, 1000, L.BF16, 65, C.byref(nb)) == UNSUPPORTED
    assert lib.edb_logprobs_bytes(5, 1000, 9, 3, C.byref(nb)) == INVALID
    assert lib.edb_logprobs_bytes(5, 1000, L.F32, 3, None) == INVALID
    assert lib.edb_distill_bytes(5, 1000, L.BF16, 3, C.byref(nb)) == L.EDB_OK and nb.value >= 0
    assert lib.edb_distill_bytes(1, 1 << 30, L.F32, 256, C.byref(nb)) == L.EDB_OK and nb.value > 0
    assert lib.edb_distill_bytes(5, 1000, L.BF16, 0, C.byref(nb)) == UNSUPPORTED
    assert lib.edb_distill_bytes(5, 1000, 4, 3, C.byref(nb)) == INVALID
    assert lib.edb_distill_bytes(5, 1000, L.F32, 3, None) == INVALID
    assert lib.edb_embed_grad_bytes(-1, 500, 64, C.byref(nb)) == INVALID
    assert lib.edb_embed_grad_bytes(1, 500, 64, None) == INVALID


def test_python_checks():
    """Tensors that no call may take (CPU tensors, wrong types and shapes)."""
    from paper_2302_03851_amd import tokens
    w, ids = torch.zeros((4, 8)), torch.zeros(3, dtype=torch.int32)
    for bad in (w, w.double(), w.view(-1), w.t()):
        with pytest.raises(ValueError):
            tokens.embed(ids, bad)
        with pytest.raises(ValueError):
            tokens.embed_grad(ids, bad, 5)
        with pytest.raises(ValueError):
            tokens.logprobs(bad, ids)
        with pytest.raises(ValueError):
            tokens.logprobs_grad(bad, ids, torch.zeros((4, 2)))
        with pytest.raises(ValueError):
            tokens.distill(bad, ids.view(1, 3), torch.zeros((1, 3)))


def test_python_sizes():
    """Sizes past 31 bits, which the C calls would see cut off (meta tensors: nothing is allocated)."""
    from paper_2302_03851_amd import tokens
    ids = torch.empty(1, dtype=torch.int32, device="meta")
    for shape in ((1, 2 ** 32 + 5), (2 ** 32 + 1, 5), (2 ** 31, 1)):
        big = torch.empty(shape, dtype=BF16, device="meta")
        one = torch.empty(1, device="meta")
        for f in (lambda: tokens.embed(ids, big), lambda: tokens.embed_grad(ids, big, 5), lambda: tokens.logprobs(big),
                  lambda: tokens.logprobs_grad(big, ids, one), lambda: tokens.distill(big, ids.view(1, 1), one.view(1, 1))):
            with pytest.raises(ValueError, match="2147483647"):
                f()


@gpu
def test_python_sizes_gpu():
    """The sizes that are arguments of their own, before anything is allocated by them."""
    from paper_2302_03851_amd import tokens
    w = torch.zeros((4, 8), device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    far = torch.zeros(1, dtype=torch.int32, device="cuda").expand(2 ** 32 + 2)
    for f in (lambda: tokens.embed_grad(ids, w, 2 ** 32 + 3), lambda: tokens.embed_grad(ids, w, -1),
              lambda: tokens.logprobs(w, ids, top=2 ** 32 + 2), lambda: tokens.logprobs(w, ids, top=-1),
              lambda: tokens.embed(far, w), lambda: tokens.distill(w, far[None].expand(4, -1), w)):
        with pytest.raises(ValueError, match="2147483647"):
            f()


@gpu
def test_python_checks_gpu():
    from paper_2302_03851_amd import tokens
    w = torch.zeros((4, 8), device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    two = torch.zeros((4, 2), device="cuda")
    bad = [lambda: tokens.embed(ids.long(), w), lambda: tokens.embed(ids.cpu(), w), lambda: tokens.embed(ids[::2], w),
           lambda: tokens.embed(ids, w, out=w[:3]), lambda: tokens.embed(ids, w, dtype=F32, out=w.to(BF16)),
           lambda: tokens.embed(ids, w.t()), lambda: tokens.embed(ids, w[:1].expand(4, 8)),
           lambda: tokens.embed_grad(ids, w, 5, accumulate=True), lambda: tokens.embed_grad(ids[:3], w, 5),
           lambda: tokens.embed_grad(ids, w, 5, out=w), lambda: tokens.logprobs(w, ids[:3]),
           lambda: tokens.logprobs(w, ids, out=tokens.logprobs(w)), lambda: tokens.logprobs(w, ids, top=2, out=tokens.logprobs(w, ids)),
           lambda: tokens.logprobs_grad(w, ids, two[:3]), lambda: tokens.logprobs_grad(w, ids, two.double()),
           lambda: tokens.logprobs_grad(w, ids, two, out=w.to(BF16)), lambda: tokens.distill(w, ids, two),
           lambda: tokens.distill(w, ids.view(4, 1), two), lambda: tokens.distill(w, ids.view(4, 1), two[:, :1].to(BF16)),
           lambda: tokens.distill(w, ids.view(4, 1), two[:, :1].contiguous(), weight=ids)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: tokens.logprobs(w, ids, temperature=0.0), lambda: tokens.logprobs(w, ids, top=65),
              lambda: tokens.embed(ids, w, out=w)):
        with pytest.raises(L.EdbError):
            f()
