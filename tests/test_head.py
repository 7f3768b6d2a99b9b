"""Layer norm and linear layers against their definitions in 64 bits, their
gradients also against differences, and their refusals.

Tolerances.  u = 2^-24 is fp32's rounding unit; a result's own rounding adds
half a unit in its last place, 2^-8 of the value for bf16.
* Layer norm: differences d from a value of the row are off by u, sums of at
  most 8 of them (or of their squares, a unit more each) by 3 u, the rest is in
  64 bits.  So the mean is off by 4 u of the average |d| and its own rounding;
  the variance by 6 u of the average d^2, which is at most 4 times it where
  sums are in 32 bits: 24 u, rstd by half of that and its rounding, 13 u.
  |d| is at most what it is from the farthest element, and its average at most
  twice the deviation where sums are in 32 bits (average d^2 <= 4 variances).
  h = (x - mean) rstd takes 4 roundings of itself and what the mean is off,
  8 u deviations; h w + b one more.
* Its gradients: h is off by 2 u, g = dy w by u of itself; the row's averages
  add up at most 24 terms a thread (dim / 1024 + 8 for rows past 8192), then a
  tree, waves and a division: DEPTH = dim / 1024 + 56 roundings of sum |term|.
  A column's sum takes at most n / 256 + 64 rows and parts one after another (n
  for rows past 8192).
* A product's sum of K terms in fp32, in any order, is off by K u sum |x w|;
  six partial products a term at most double the roundings, and leave out
  2^-24 of it: (2 K + 16) u sum |x w|.
* Activations move by at most 1.13 of what their argument moves; their own
  evaluation is off by some units, of the exponential's argument z by z more.
* bf16 gradients are formed from g rounded to bf16.
"""
import ctypes as C
import math

import pytest

from paper_2302_03851_amd import _lib as L

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
INF = math.inf
TINY = 2.0 ** -149      # below the normal numbers the last place is this


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _half(ref, dtype):
    return ref.abs() * (2.0 ** -8 if dtype == BF16 else U) + (2.0 ** -133 if dtype == BF16 else TINY)


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


def _only(mem, before, view, old):
    """Nothing beside the view was written."""
    kept = view.clone()
    view.copy_(old)
    assert torch.equal(mem.view(torch.uint8), before.view(torch.uint8))
    view.copy_(kept)


# ---- layer norm ------------------------------------------------------------------

# every way that a row is held, and every way that it ends
DIMS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 1024,
        1025, 2047, 2048, 2051, 4096, 4097, 8192, 8193, 16384, 16385, 32771, 70001]


def _norm_reference(x, w, b, eps):
    x = x.double()
    mean = torch.where(torch.isfinite(x).all(1, keepdim=True), x.mean(1, keepdim=True), math.nan)
    # from the first element on: the mean's own rounding does not count then
    d = x - x[:, :1]
    mean_d = d.mean(1, keepdim=True)
    var = (d - mean_d).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    h = (d - mean_d) * rstd
    w = torch.ones_like(x[0]) if w is None else w.double()
    b = torch.zeros_like(x[0]) if b is None else b.double()
    return mean, rstd, h, h * w + b, w


def _check_norm(x, w, b, eps, r):
    mean, rstd, h, y, wd = _norm_reference(x, w, b, eps)
    D = x.shape[1]
    spread = 2 * (x.double() - mean).square().mean(1, keepdim=True).sqrt()
    # 64-bit sums of D terms, themselves rounded
    wide = D * 2.0 ** -50
    _close(r.stats[:, :1], mean, _half(mean, F32) + 4 * U * spread + wide * (spread + mean.abs()))
    _close(r.stats[:, 1:], rstd, _half(rstd, F32) + (13 * U + wide) * rstd)
    _close(r.out, y, (18 * U + wide) * (h * wd).abs() + (8 * U + wide) * (spread * rstd * wd).abs() + U * y.abs() + _half(y, r.out.dtype))


@gpu
@pytest.mark.parametrize("T,O", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("dim", DIMS)
def test_layer_norm(dim, T, O):
    from paper_2302_03851_amd import head
    g = _gen(dim)
    for n, pad, shift, w, b in [(1, 0, 0, None, None), (3, 3, 1, F32, F32), (37 if dim < 5000 else 9, 8, 0, BF16, BF16),
                                (300 if dim < 5000 else 17, 0, 3, F32, None)]:
        x, _ = _view((torch.randn((n, dim), generator=g, device="cuda") + 2.0).to(T), pad, shift)
        wt = None if w is None else torch.randn(dim, generator=g, device="cuda").to(w)
        bt = None if b is None else torch.randn(dim, generator=g, device="cuda").to(b)
        dst, mem = _view(torch.zeros((n, dim), dtype=O, device="cuda"), pad, shift)
        before, old = mem.clone(), dst.clone()
        r = head.layer_norm(x, wt, bt, 1e-5, out=head.Normed(dst, torch.empty((n, 2), device="cuda")))
        _check_norm(x, wt, bt, 1e-5, r)
        _only(mem, before, dst, old)


@gpu
@pytest.mark.parametrize("dim", [7, 100, 512, 4099, 20000])
@pytest.mark.parametrize("T", [F32, BF16])
def test_layer_norm_values(dim, T):
    """Means far above the spread, constant rows, very large and very small rows, rows with infinities and NaN."""
    from paper_2302_03851_amd import head
    g = _gen(dim)
    x = torch.randn((12, dim), generator=g, device="cuda")
    x[1] += 30000.0
    x[2] = 3.0
    x[3] *= 1e30
    x[4] *= 1e-30
    x[5] = torch.where(x[5] > 0, 3.3e38, -3.3e38)
    x[6, dim // 2] = INF
    x[7, 0] = -INF
    x[8, dim - 1] = float("nan")
    x[9] = 0.0
    x[10, 1:] = 5.0
    x[10, 0] = -1e9
    x = x.to(T)
    for eps in (1e-5, 1e-12):
        r = head.layer_norm(x, None, None, eps, dtype=F32)
        _check_norm(x, None, None, eps, r)
        assert torch.isnan(r.out[6:9]).all() and not r.out[2].any() and not r.out[9].any()
        if eps == 1e-5:
            good = [0, 1, 2, 3, 4, 5, 9, 10, 11]
            dy = torch.randn((9, dim), generator=g, device="cuda").to(T)
            xs = x[good].contiguous()
            xs[5, 0], xs[5, 1:] = -3.3e38, 3.3e38      # differences past fp32's range
            st = head.layer_norm(xs).stats
            _check_norm_grad(xs, st, dy, None, head.layer_norm_grad(xs, st, dy))
            q = head.layer_norm_grad(x, r.stats, torch.ones_like(x))
            assert torch.isnan(q.dx[6:9]).all() and torch.isnan(q.dweight).all() and (q.dbias == 12).all()
    assert torch.isnan(head.layer_norm(x[2:3], eps=0.0).out).all()


@gpu
def test_layer_norm_rows():
    """Many rows, none, and rows past 32 bits of elements."""
    from paper_2302_03851_amd import head
    g = _gen(1)
    x = torch.randn((3000001, 5), generator=g, device="cuda")
    r = head.layer_norm(x)
    _check_norm(x, None, None, 1e-5, r)
    q = head.layer_norm_grad(x, r.stats, x)
    _check_norm_grad(x, r.stats, x, None, q)
    none = head.layer_norm(x[:0])
    assert none.out.shape == (0, 5)
    q = head.layer_norm_grad(x[:0], none.stats, x[:0], torch.ones(5, device="cuda"))
    assert q.dx.shape == (0, 5) and not q.dweight.any() and not q.dbias.any()
    far = 1 << 31
    mem = torch.empty(2 * far + 64, dtype=BF16, device="cuda")
    rows = mem.as_strided((3, 64), (far, 1))
    rows.copy_(torch.randn((3, 64), generator=g, device="cuda"))
    near = rows.clone()
    r = head.layer_norm(rows)
    assert torch.equal(r.out, head.layer_norm(near).out)
    dy = torch.randn((3, 64), generator=g, device="cuda")
    ref = head.layer_norm_grad(near, r.stats, dy)
    got = head.layer_norm_grad(near, r.stats, dy, out=head.NormGrad(rows, torch.empty(64, device="cuda"), torch.empty(64, device="cuda")))
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    head.layer_norm(near, out=head.Normed(rows, r.stats))
    assert torch.equal(rows, head.layer_norm(near).out)


def _check_norm_grad(x, stats, dy, w, r):
    n, D = x.shape
    mean, rstd = stats.double().unbind(1)
    h = (x.double() - mean[:, None]) * rstd[:, None]
    dy = dy.double()
    wd = torch.ones(D, device="cuda", dtype=torch.float64) if w is None else w.double()
    gg = dy * wd
    c1, c2 = gg.mean(1, keepdim=True), (gg * h).mean(1, keepdim=True)
    a1, a2 = gg.abs().mean(1, keepdim=True), (gg * h).abs().mean(1, keepdim=True)
    if r.dx is not None:
        ref = rstd[:, None] * (gg - c1 - h * c2)
        deep = D / 1024 + 56
        tol = U * rstd[:, None] * (5 * (gg.abs() + c1.abs() + 2 * (h * c2).abs()) + (deep + 4) * a1 + (deep + 8) * h.abs() * a2)
        _close(r.dx, ref, tol + _half(ref, r.dx.dtype))
    if r.dweight is not None:
        rows = n / 256 + 64 if D <= 8192 else n + 64
        ref = (dy * h).sum(0)
        _close(r.dweight, ref, (rows + 4) * U * (dy * h).abs().sum(0) + _half(ref, F32))
        ref = dy.sum(0)
        _close(r.dbias, ref, rows * U * dy.abs().sum(0) + _half(ref, F32))


@gpu
@pytest.mark.parametrize("T,O", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("dim", DIMS)
def test_layer_norm_grad(dim, T, O):
    from paper_2302_03851_amd import head
    g = _gen(dim + 1)
    for n, pad, shift, w in [(1, 0, 0, None), (3, 3, 1, F32), (37 if dim < 5000 else 9, 8, 0, BF16), (700 if dim < 5000 else 33, 0, 3, F32)]:
        x, _ = _view((torch.randn((n, dim), generator=g, device="cuda") + 1.0).to(T), pad, shift)
        dy, _ = _view(torch.randn((n, dim), generator=g, device="cuda").to(O), shift, pad)
        wt = None if w is None else torch.randn(dim, generator=g, device="cuda").to(w)
        stats = head.layer_norm(x).stats
        dst, mem = _view(torch.zeros((n, dim), dtype=T, device="cuda"), pad, shift)
        before, old = mem.clone(), dst.clone()
        sums = [torch.full((dim,), float("nan"), device="cuda") for _ in range(2)]
        r = head.layer_norm_grad(x, stats, dy, wt, out=head.NormGrad(dst, *sums))
        _check_norm_grad(x, stats, dy, wt, r)
        _only(mem, before, dst, old)
        only = head.layer_norm_grad(x, stats, dy, wt, sums=False)
        assert only.dweight is None and torch.equal(only.dx, r.dx)
        only = head.layer_norm_grad(x, stats, dy, wt, dx=False)
        assert only.dx is None and torch.equal(only.dweight, r.dweight) and torch.equal(only.dbias, r.dbias)


@gpu
@pytest.mark.parametrize("n", [1024, 2047, 8191, 8193, 40001])
@pytest.mark.parametrize("dim,T", [(40, F32), (512, BF16), (1030, F32), (9000, F32), (12000, BF16)])
def test_layer_norm_grad_rows(n, dim, T):
    """More rows than the work-groups take in one turn."""
    from paper_2302_03851_amd import head
    if n * dim > 1 << 27:
        n //= 8
    g = _gen(n)
    x = torch.randn((n, dim), generator=g, device="cuda").to(T)
    dy = torch.randn((n, dim), generator=g, device="cuda").to(T)
    w = torch.randn(dim, generator=g, device="cuda")
    r = head.layer_norm(x, w)
    _check_norm(x, w, None, 1e-5, r)
    _check_norm_grad(x, r.stats, dy, w, head.layer_norm_grad(x, r.stats, dy, w))


@gpu
def test_layer_norm_differences():
    """The gradients against central differences of the kernel's own results: steps of 2^-6, so an
    error of up to step^2 / 6 times the third derivative and u |y| sum / step."""
    from paper_2302_03851_amd import head
    g = _gen(4)
    n, D, step = 4, 24, 2.0 ** -6
    x, dy = torch.randn((n, D), generator=g, device="cuda"), torch.randn((n, D), generator=g, device="cuda")
    w, b = torch.randn(D, generator=g, device="cuda"), torch.randn(D, generator=g, device="cuda")

    def f(x, w, b):
        return float((head.layer_norm(x, w, b).out.double() * dy.double()).sum())

    r = head.layer_norm_grad(x, head.layer_norm(x, w, b).stats, dy, w)
    noise = U * float((head.layer_norm(x, w, b).out.abs() * dy.abs()).sum()) / step
    for got, t, at in [(r.dx, x, (1, 5)), (r.dx, x, (3, 0)), (r.dweight, w, (7,)), (r.dbias, b, (23,))]:
        up, down = t.clone(), t.clone()
        up[at] += step
        down[at] -= step
        args = [(up if t is q else q, down if t is q else q) for q in (x, w, b)]
        slope = (f(*(a for a, _ in args)) - f(*(a for _, a in args))) / (2 * step)
        # third derivatives in x: of order sum |dy w| / std^3, some units
        bend = step ** 2 * 10 * float((dy * w).abs().sum(1).max()) if t is x else 0.0
        assert abs(float(got[at]) - slope) <= bend + 2 * noise + 1e-5


# ---- linear layers ---------------------------------------------------------------

ACTS = ["none", "relu", "gelu", "silu", "tanh"]
SQRT_HALF = math.sqrt(0.5)


def _act(v, act):
    """Value, derivative, and what the evaluation of either is off by, in units u."""
    if act == "none":
        return v, torch.ones_like(v), 0 * v, 0 * v
    if act == "relu":
        return v.clamp(min=0), (v > 0).double(), 0 * v, 0 * v
    if act == "gelu":
        p, d = 0.5 * torch.erfc(-v * SQRT_HALF), torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
        return v * p, p + v * d, (v * p).abs() * (10 + 2 * v * v), p * (10 + 2 * v * v) + (v * d).abs() * (10 + v * v)
    if act == "silu":
        p = torch.sigmoid(v)
        return v * p, p * (1 + v * (1 - p)), (v * p).abs() * (10 + v.abs()), p * (1 + v.abs()) * (12 + 2 * v.abs())
    t = torch.tanh(v)
    return t, 1 / torch.cosh(v) ** 2, 8 * t.abs(), (12 + 4 * v.abs()) / torch.cosh(v) ** 2


def _check_linear(x, w, bias, act, res, r):
    K = x.shape[1]
    v = torch.mm(x.double(), w.double())
    tol = (2 * K + 16) * U * torch.mm(x.double().abs(), w.double().abs())
    if bias is not None:
        v = v + bias.double()
    tol = tol + U * v.abs()
    if r.pre is not None:
        _close(r.pre, v, tol + _half(v, r.pre.dtype))
    y, _, off, _ = _act(v, act)
    tol = 1.14 * tol + U * off
    if res is not None:
        y = y + res.double()
    _close(r.out, y, tol + U * y.abs() + _half(y, r.out.dtype))


# (n, k, m): single rows, every tile's edges, split sums, odd lengths
SHAPES = [(1, 1, 1), (1, 64, 300), (2, 7, 5), (3, 513, 1030), (16, 512, 2048), (17, 100, 77), (33, 31, 129), (64, 64, 64),
          (65, 65, 65), (100, 2000, 40), (128, 33, 256), (130, 700, 131), (260, 96, 1000), (1000, 40, 1), (2500, 130, 1300)]


@gpu
@pytest.mark.parametrize("T", [F32, BF16])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_linear(shape, T, turned):
    from paper_2302_03851_amd import head
    n, k, m = shape
    g = _gen(n + k + m)
    for i, (pad, shift, act, O, b, res) in enumerate([(0, 0, "none", T, None, None), (8, 8, "gelu", T, F32, T), (3, 1, "silu", F32, BF16, BF16),
                                                     (1, 3, "tanh", BF16, T, F32), (5, 0, "relu", T, F32, T)]):
        x, _ = _view(torch.randn((n, k), generator=g, device="cuda").to(T), pad, shift)
        w = (torch.randn((m, k) if turned else (k, m), generator=g, device="cuda") * (2 / math.sqrt(k))).to(T)
        w, _ = _view(w, pad, shift)
        w = w.t() if turned else w
        bias = None if b is None else torch.randn(m, generator=g, device="cuda").to(b)
        r = None if res is None else _view(torch.randn((n, m), generator=g, device="cuda").to(res), pad, shift)[0]
        dst, mem = _view(torch.zeros((n, m), dtype=O, device="cuda"), pad, shift)
        pre, pmem = _view(torch.zeros((n, m), dtype=T, device="cuda"), shift, pad)
        before, pbefore, old, pold = mem.clone(), pmem.clone(), dst.clone(), pre.clone()
        got = head.linear(x, w, bias, act, r, keep=i % 2 == 1, out=head.Linear(dst, pre))
        _check_linear(x, w, bias, act, r, head.Linear(got.out, got.pre if i % 2 == 1 else None))
        _only(mem, before, dst, old)
        if i % 2 == 1:
            _only(pmem, pbefore, pre, pold)
        else:
            assert torch.equal(pmem.view(torch.uint8), pbefore.view(torch.uint8))


@gpu
@pytest.mark.parametrize("T", [F32, BF16])
@pytest.mark.parametrize("m", list(range(1, 20)) + [63, 66, 255, 258])
@pytest.mark.parametrize("n,k", [(5, 9), (70, 41)])
def test_linear_widths(n, k, m, T):
    """Every way that a row of results can end."""
    from paper_2302_03851_amd import head
    g = _gen(m)
    x = torch.randn((n, k), generator=g, device="cuda").to(T)
    w = torch.randn((k, m), generator=g, device="cuda").to(T)
    b = torch.randn(m, generator=g, device="cuda")
    dst, mem = _view(torch.zeros((n, m), dtype=T, device="cuda"), 2, 1)
    before, old = mem.clone(), dst.clone()
    r = head.linear(x, w, b, "tanh", out=head.Linear(dst, None))
    _check_linear(x, w, b, "tanh", None, r)
    _only(mem, before, dst, old)
    _check_linear_grad(x, w, r.out, "none", None, head.linear_grad(x, w, r.out))


def _check_linear_grad(x, w, dy, act, pre, r):
    (n, k), m, T = x.shape, w.shape[1], x.dtype
    g, off = dy.double(), 0.0
    if act != "none":
        _, d, _, doff = _act(pre.double(), act)
        off = U * g.abs() * (doff + d.abs())
        g = g * d
    size = g.abs()
    if r.dbias is not None:
        ref = g.sum(0)
        rows = n / 8 + 8 + 32
        _close(r.dbias, ref, (off.sum(0) if act != "none" else 0.0) + rows * U * size.sum(0) + _half(ref, F32))
    if T == BF16 and (act != "none" or dy.dtype != BF16):
        off = off + 2.0 ** -8 * size + 2.0 ** -133
    off = torch.as_tensor(off, device="cuda", dtype=torch.float64).expand_as(g).contiguous()
    xd, wd = x.double(), w.double()
    if r.dx is not None:
        ref = torch.mm(g, wd.t())
        tol = torch.mm(off, wd.t().abs()) + (2 * m + 16) * U * torch.mm(size + off, wd.t().abs())
        _close(r.dx, ref, tol + _half(ref, T))
    if r.dweight is not None:
        ref = torch.mm(xd.t(), g)
        tol = torch.mm(xd.t().abs(), off) + (2 * n + 16) * U * torch.mm(xd.t().abs(), size + off)
        _close(r.dweight, ref, tol + _half(ref, T))


@gpu
@pytest.mark.parametrize("T", [F32, BF16])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("shape", SHAPES + [(5000, 40, 72)])
def test_linear_grad(shape, T, turned):
    from paper_2302_03851_amd import head
    n, k, m = shape
    g = _gen(n + k * m)
    for pad, shift, act, O in [(0, 0, "none", T), (8, 8, "gelu", T), (3, 1, "silu", F32), (1, 3, "tanh", BF16), (5, 0, "relu", T),
                               (3, 1, "none", BF16 if T == F32 else F32)]:
        x, _ = _view(torch.randn((n, k), generator=g, device="cuda").to(T), pad, shift)
        w = (torch.randn((m, k) if turned else (k, m), generator=g, device="cuda") * (2 / math.sqrt(k))).to(T)
        w, _ = _view(w, pad, shift)
        dy, _ = _view(torch.randn((n, m), generator=g, device="cuda").to(O), pad, shift)
        pre = None if act == "none" else _view(torch.randn((n, m), generator=g, device="cuda").to(T) * 2, shift, pad)[0]
        dx, xmem = _view(torch.zeros((n, k), dtype=T, device="cuda"), pad, shift)
        dw, wmem = _view(torch.zeros_like(w, memory_format=torch.contiguous_format), pad, shift)
        before, wbefore, old, wold = xmem.clone(), wmem.clone(), dx.clone(), dw.clone()
        turn = (lambda t: t.t()) if turned else (lambda t: t)
        r = head.linear_grad(x, turn(w), dy, act, pre, out=head.LinearGrad(dx, turn(dw), torch.empty(m, device="cuda")))
        _check_linear_grad(x, turn(w), dy, act, pre, r)
        _only(xmem, before, dx, old)
        _only(wmem, wbefore, dw, wold)
        for one in ("dx", "dweight", "dbias"):
            only = head.linear_grad(x, turn(w), dy, act, pre, **{q: q == one for q in ("dx", "dweight", "dbias")})
            assert [q is not None for q in only] == [q == one for q in ("dx", "dweight", "dbias")]
            if one == "dbias":      # added up by the weight's product or by itself
                _check_linear_grad(x, turn(w), dy, act, pre, only)
            else:
                assert torch.equal(getattr(only, one), getattr(r, one))
            assert one != "dweight" or 1 in (k, m) or only.dweight.stride() == turn(torch.empty((m, k) if turned else (k, m))).stride()


@gpu
@pytest.mark.parametrize("n,k,m,T", [(1, 512, 60000, BF16), (16, 500, 9001, BF16), (15, 1000, 9001, F32), (4100, 512, 1536, BF16),
                                     (1627, 100, 8011, F32), (3000, 256, 768, F32), (257, 4099, 300, BF16), (20000, 64, 64, F32)])
@pytest.mark.parametrize("turned", [False, True])
def test_linear_larger(n, k, m, T, turned):
    """The sizes at which tiles, splits and layouts change, in use."""
    from paper_2302_03851_amd import head
    g = _gen(n)
    x = torch.randn((n, k), generator=g, device="cuda").to(T)
    w = (torch.randn((m, k) if turned else (k, m), generator=g, device="cuda") / math.sqrt(k)).to(T)
    w = w.t() if turned else w
    b = torch.randn(m, generator=g, device="cuda")
    r = head.linear(x, w, b, "gelu", keep=True)
    _check_linear(x, w, b, "gelu", None, r)
    _check_linear_grad(x, w, r.out, "gelu", r.pre, head.linear_grad(x, w, r.out, "gelu", r.pre))


@gpu
@pytest.mark.parametrize("T", [F32, BF16])
def test_linear_values(T):
    """Infinities, NaN and the largest and smallest numbers: a row affects itself only."""
    from paper_2302_03851_amd import head
    g = _gen(9)
    n, k, m = 40, 70, 50
    x = torch.randn((n, k), generator=g, device="cuda")
    x[1, 3], x[2, 69], x[3, 0], x[4, 7], x[4, 9] = INF, -INF, float("nan"), INF, -INF
    x[5] *= 1e30
    x[6] = 0.0
    x[6, 5] = torch.finfo(F32).max
    x[7] = 0.0
    x[7, 5] = -torch.finfo(F32).max
    x[8] *= 1e-30
    x = x.to(T)
    w = torch.randn((k, m), generator=g, device="cuda").to(T)
    w[5] = w[5].abs().clamp(max=0.5)
    w[0] = 0.0       # infinity times zero is none
    x[3, 0], x[9, 0] = 1.0, INF
    x[3, 1] = float("nan")
    for turned in (False, True):
        wt = w.t().contiguous().t() if turned else w
        r = head.linear(x, wt, dtype=F32)
        _check_linear(x, wt, None, "none", None, r)
        assert torch.isnan(r.out[9]).all() and torch.isnan(r.out[3]).all() and torch.isinf(r.out[1]).all()
        q = head.linear_grad(x, wt, r.out, dx=False, dweight=False)
        _close(q.dbias, r.out.double().sum(0), 1e30)
        # and as the other operand: columns of the weight
        s = head.linear(wt.t().contiguous(), x.t().contiguous(), dtype=F32)
        ok = torch.isfinite(r.out)
        assert torch.equal(ok, torch.isfinite(s.out.t()))
    v = torch.tensor([[-INF, -1e4, -100.0, -20.0, -5.0, 0.0, 5.0, 20.0, 100.0, 1e4, INF, float("nan")]], device="cuda").to(T)
    one = torch.eye(12, device="cuda").to(T)
    x = torch.zeros_like(one)
    for act, left in [("relu", 0.0), ("tanh", -1.0)]:
        y = head.linear(torch.zeros((1, 12), device="cuda", dtype=T), one, v[0], act).out[0]
        assert y[0] == left and y[5] == 0 and torch.isnan(y[11]) and y[10] == (INF if act == "relu" else 1.0)
    for act in ACTS[1:]:
        dy = torch.ones_like(v)
        q = head.linear_grad(x[:1], one, dy, act, v, dx=False, dweight=False).dbias
        assert torch.isfinite(q[1:10]).all() and float(q[1:5].abs().max()) <= 0.1 and torch.isnan(q[11])


@gpu
@pytest.mark.parametrize("T", [F32, BF16])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("n,k,m", [(40, 70, 50), (700, 33, 300), (9001, 1000, 1000)])
def test_linear_grad_values(n, k, m, T, turned):
    """Infinities, NaN and large numbers of dout reach the sums of their own columns only, with the weight's gradient and
    alone, and a NaN row of x all of the weight's gradient; the product of the transposes has the same values."""
    from paper_2302_03851_amd import head
    g = _gen(n)
    x, w = torch.randn((n, k), generator=g, device="cuda").to(T), torch.randn((k, m), generator=g, device="cuda").to(T)
    wt = w.t().contiguous().t() if turned else w
    dy = torch.randn((n, m), generator=g, device="cuda")
    dy[3, 0], dy[n - 1, 1], dy[7, 2], dy[8, 2] = INF, -INF, INF, -INF
    dy[n // 2, 4] = float("nan")
    dy[:, 5] *= 1e30
    dy[5, m - 1] = INF
    dy = dy.to(T)
    inner = [c for c in range(m) if c not in (0, 1, 2, 4, m - 1)]
    for want in (dict(), dict(dx=False), dict(dx=False, dweight=False)):
        q = head.linear_grad(x, wt, dy, **want)
        _check_linear_grad(x, w, dy, "none", None, head.LinearGrad(None, None, q.dbias))
        assert q.dbias[0] == INF and q.dbias[1] == -INF and torch.isnan(q.dbias[2]) and torch.isnan(q.dbias[4]) and q.dbias[m - 1] == INF
        if q.dweight is not None:      # the other columns know nothing of it
            _check_linear_grad(x, w[:, inner], dy[:, inner], "none", None, head.LinearGrad(None, q.dweight[:, inner], None))
            assert not torch.isfinite(q.dweight[:, [0, 1, 2, 4, m - 1]]).any()
    bad = x.clone()
    bad[n // 3] = float("nan")
    q = head.linear_grad(bad, wt, dy, dx=False)
    assert torch.isnan(q.dweight).all()
    _check_linear_grad(bad, w, dy, "none", None, head.LinearGrad(None, None, q.dbias))
    # as the right operand: a column of the results each
    s = head.linear(wt.t().contiguous(), x.t().contiguous() if turned else x.t(), dtype=F32)
    _check_linear(w.t(), x.t(), None, "none", None, s)
    far = x.clone()
    far[1, 3], far[2, k - 1], far[4, 0], far[4, 1], far[6, 2] = INF, -INF, INF, -INF, float("nan")
    s = head.linear(wt.t().contiguous(), far.t().contiguous() if turned else far.t(), dtype=F32)
    _check_linear(w.t(), far.t(), None, "none", None, s)


@gpu
@pytest.mark.parametrize("n,k,m", [(6, 40, 30), (600, 3000, 520)])
def test_linear_ends_of_the_range(n, k, m):
    """fp32 terms up to 2^128 - 2^121, whose first pieces' product is the largest (1 + 2^-8)^2 of it, and infinities
    times the smallest numbers that are not taken for zeros."""
    from paper_2302_03851_amd import head
    g = _gen(k)
    x, w = torch.zeros((n, k), device="cuda"), torch.zeros((k, m), device="cuda")
    # mantissas just above the middle between two bf16 values: their first pieces are rounded up by the most
    up = 1 + 2.0 ** -8 + 2.0 ** -23
    x[0, 3], w[3, 0], w[3, 1] = up * 2.0 ** 64, 2.0 ** 63 * 1.976, -(2.0 ** 63) * 1.976
    x[1, 4], w[4, 0], w[4, 1] = up * 2.0 ** 100, up * 2.0 ** 27, -up * 2.0 ** 27
    x[2, 5], w[5, 0], w[5, 1] = 1.98 * 2.0 ** 127, 1.0, -1.0
    assert float((x.double() @ w.double()).abs().max()) <= 2.0 ** 128 - 2.0 ** 121
    r = head.linear(x, w)
    _check_linear(x, w, None, "none", None, r)
    assert torch.isfinite(r.out).all()
    x, w = torch.zeros((n, k), device="cuda"), torch.zeros((k, m), device="cuda")
    x[0, 7], x[1, 7] = INF, -INF
    w[7, :4] = torch.tensor([2.0 ** -133, -(2.0 ** -133), 2.0 ** -126, 1.5 * 2.0 ** -133], device="cuda")
    for a, b in ((x, w), (w.t().contiguous(), x.t().contiguous())):
        _check_linear(a, b, None, "none", None, head.linear(a, b))


@gpu
@pytest.mark.parametrize("scale", [1e-30, 1e-33, 1e-35, 1e-37, 1e-39])
@pytest.mark.parametrize("T", [F32, BF16])
def test_linear_small(T, scale):
    """Factors down to below the normal numbers: fp32 ones are off by 2^-134 each (half of bf16's least number)."""
    from paper_2302_03851_amd import head
    g = _gen(11)
    x = (torch.randn((70, 96), generator=g, device="cuda").double() * scale).to(T)
    w = (torch.randn((96, 130), generator=g, device="cuda") * 1e4).to(T)
    for a, b in ((x, w), (w.t().contiguous(), x.t().contiguous())):
        v, size = torch.mm(a.double(), b.double()), torch.mm(a.double().abs(), b.double().abs())
        tol = (2 * 96 + 16) * U * size + _half(v, F32)
        if T == F32:
            tol = tol + 2.0 ** -134 * (a.double().abs().sum(1, keepdim=True) + b.double().abs().sum(0, keepdim=True))
        _close(head.linear(a, b, dtype=F32).out, v, tol)


@gpu
def test_linear_in_place():
    """The residual's place may take the result; columns of one buffer; nothing to do."""
    from paper_2302_03851_amd import head
    g = _gen(2)
    for n, k, m, T in [(5, 40, 30, F32), (700, 64, 200, BF16), (1, 512, 33, BF16), (40, 3000, 50, F32)]:
        x = torch.randn((n, k), generator=g, device="cuda").to(T)
        w = torch.randn((k, m), generator=g, device="cuda").to(T)
        r = torch.randn((n, m), generator=g, device="cuda").to(T)
        ref = head.linear(x, w, None, "silu", r).out
        place = r.clone()
        head.linear(x, w, None, "silu", place, out=head.Linear(place, None))
        assert torch.equal(place, ref)
        buf = torch.zeros((n, k + 2 * m), dtype=T, device="cuda")
        buf[:, :k] = x
        buf[:, k:k + m] = r
        head.linear(buf[:, :k], w, None, "silu", buf[:, k:k + m], out=head.Linear(buf[:, k + m:], None))
        assert torch.equal(buf[:, k + m:], ref) and torch.equal(buf[:, k:k + m], r)
        none = head.linear(x[:0], w)
        assert none.out.shape == (0, m)
        q = head.linear_grad(x[:0], w, r[:0])
        assert q.dx.shape == (0, k) and not q.dweight.any() and not q.dbias.any()


@gpu
@pytest.mark.parametrize("T", [F32, BF16])
def test_linear_offsets_past_32_bits(T):
    from paper_2302_03851_amd import head
    g = _gen(3)
    far, n, k, m = 1 << 31, 3, 40, 24
    mem = torch.zeros(2 * far + 64, dtype=T, device="cuda")
    rows = mem.as_strided((n, k), (far, 1))
    x = torch.randn((n, k), generator=g, device="cuda").to(T)
    w = torch.randn((k, m), generator=g, device="cuda").to(T)
    rows.copy_(x)
    ref = head.linear(x, w).out
    assert torch.equal(head.linear(rows, w).out, ref)
    grads = head.linear_grad(x, w, ref)
    assert all(torch.equal(a, b) for a, b in zip(head.linear_grad(rows, w, ref), grads))
    out = mem.as_strided((n, m), (far, 1))
    head.linear(x, w, out=head.Linear(out, None))
    assert torch.equal(out, ref)
    assert torch.equal(head.linear_grad(x, w, out).dx, grads.dx)
    # a weight of three far lines, either way round
    few = torch.randn((5, n), generator=g, device="cuda").to(T)
    lines = mem.as_strided((n, k), (far, 1))
    lines.copy_(x)
    assert torch.equal(head.linear(few, lines).out, head.linear(few, x).out)
    many = torch.randn((5, k), generator=g, device="cuda").to(T)
    assert torch.equal(head.linear(many, lines.t()).out, head.linear(many, x.t()).out)


@gpu
@pytest.mark.parametrize("n,k,m,T", [(5000001, 3, 5, F32), (2100000, 9, 70, BF16), (3, 1300001, 2, F32), (2, 3, 3000003, BF16)])
def test_linear_long(n, k, m, T):
    """Millions of rows, of terms and of columns."""
    from paper_2302_03851_amd import head
    g = _gen(n)
    x = torch.randn((n, k), generator=g, device="cuda").to(T)
    w = torch.randn((k, m), generator=g, device="cuda").to(T)
    b = torch.randn(m, generator=g, device="cuda")
    r = head.linear(x, w, b, "relu", keep=True)
    _check_linear(x, w, b, "relu", None, r)
    _check_linear_grad(x, w, r.out, "relu", r.pre, head.linear_grad(x, w, r.out, "relu", r.pre))
    _check_linear_grad(x, w, r.out, "none", None, head.linear_grad(x, w, r.out))


@gpu
def test_linear_differences():
    """The gradients against central differences of the results in fp32: the step is 2^-5; bends are
    below 3 step^2 / 6 of the terms, noise (2 k + 16) u of them over the step."""
    from paper_2302_03851_amd import head
    g = _gen(6)
    n, k, m, step = 6, 10, 9, 2.0 ** -5
    x, w = torch.randn((n, k), generator=g, device="cuda") / 2, torch.randn((k, m), generator=g, device="cuda") / 2
    b, dy = torch.randn(m, generator=g, device="cuda"), torch.randn((n, m), generator=g, device="cuda")

    for act in ["none", "gelu", "silu", "tanh"]:
        def f(x, w, b):
            return float((head.linear(x, w, b, act).out.double() * dy.double()).sum())

        pre = None if act == "none" else head.linear(x, w, b, act, keep=True).pre
        r = head.linear_grad(x, w, dy, act, pre)
        for got, t, at in [(r.dx, x, (2, 3)), (r.dx, x, (5, 9)), (r.dweight, w, (1, 8)), (r.dbias, b, (4,))]:
            up, down = t.clone(), t.clone()
            up[at] += step
            down[at] -= step
            args = [(up if t is q else q, down if t is q else q) for q in (x, w, b)]
            slope = (f(*(a for a, _ in args)) - f(*(a for _, a in args))) / (2 * step)
            size = float(dy.abs().sum()) * 4       # |dy| times the cube of what moves, which is below 2
            assert abs(float(got[at]) - slope) <= step ** 2 / 2 * size + (2 * k + 16) * U * size / step


@gpu
@pytest.mark.parametrize("n,k,m,T", [(262144, 2048, 2048, F32), (262144, 512, 1024, BF16), (300001, 40, 72, F32), (40000, 300, 20000, BF16),
                                     (70001, 515, 4104, BF16)])
@pytest.mark.parametrize("turned", [False, True])
def test_linear_grad_bias_of_one_sign(n, k, m, T, turned):
    """The bias's gradient of numbers of one sign, with the weight's and alone: column c adds up numbers whose sum loses
    nearly half a place at every addition while it is between 2^(c % 18) and twice that.  Summed with the weight's
    gradient, a thread adds up at most 256 pieces at a time and n / 2048 such sums, then come 32 threads and 64 parts;
    alone, 64 rows at a time, n m / 2^28 such sums and the rest of it."""
    from paper_2302_03851_amd import head
    x, w = torch.zeros((n, k), device="cuda", dtype=T), torch.zeros((m, k) if turned else (k, m), device="cuda", dtype=T)
    w = w.t() if turned else w
    column = 1 + 0.49 * 2.0 ** (torch.arange(m, device="cuda", dtype=torch.float64) % 18 - 23)
    if T == BF16:
        column = 0.5 + torch.rand(m, generator=_gen(m), device="cuda")
    dy = column.to(T).expand(n, m).contiguous()
    if T == BF16:
        dy *= torch.rand((n, 1), generator=_gen(n), device="cuda").to(T) + 0.5
    ref = torch.zeros(m, dtype=torch.float64, device="cuda")
    for part in dy.split(65536):
        ref += part.double().sum(0)
    for adds, got in ((n / 2048 + 360, head.linear_grad(x, w, dy).dbias), (n / 2048 + 360, head.linear_grad(x, w, dy, dx=False).dbias),
                      (n * m / 2.0 ** 28 + 360, head.linear_grad(x, w, dy, dx=False, dweight=False).dbias)):
        _close(got, ref, adds * U * ref + _half(ref, F32))


# ---- streams and graphs ------------------------------------------------------------


def _everything(seed):
    """Inputs of each operator and a function that runs them into new results."""
    from paper_2302_03851_amd import head
    g = _gen(seed)

    def normal(*shape, dtype=F32):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    cases = []
    for n, k, m, T in [(700, 100, 333, F32), (3, 600, 2000, BF16), (20000, 64, 40, BF16), (257, 4099, 70, F32)]:
        cases.append((normal(n, k, dtype=T), normal(k, m, dtype=T), normal(m), normal(n, m, dtype=T), normal(k)))
    long = normal(5, 40003)

    def go():
        got = []
        for x, w, b, dy, scale in cases:
            y = head.layer_norm(x, scale)
            r = head.linear(y.out, w, b, "gelu", dy, keep=True)
            q = head.linear_grad(y.out, w, dy, "gelu", r.pre)
            got += [*y, *r, *q, *head.layer_norm_grad(x, y.stats, q.dx, scale)]
        y = head.layer_norm(long)
        return got + [*y, *head.layer_norm_grad(long, y.stats, long)]

    return go


def _same(a, b):
    return all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(a, b))


@gpu
def test_head_streams():
    """The current stream's work, several streams at once; the same bits in every run."""
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
def test_head_captured():
    """All calls in one HIP graph, replayed between eager calls."""
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

A = 1 << 30      # addresses that are never read: every call below is refused first
INVALID, UNSUPPORTED = L.EDB_ERR_INVALID, L.EDB_ERR_UNSUPPORTED


def _norm(**k):
    a = dict(x=A, xd=L.F32, n=4, D=10, xs=10, w=2 * A, b=3 * A, wd=L.F32, eps=1e-5, out=4 * A, od=L.F32, os=10, st=5 * A)
    a.update(k)
    return L.load().edb_layer_norm(*a.values(), None)


def _norm_grad(**k):
    a = dict(x=A, xd=L.F32, n=4, D=10, xs=10, st=2 * A, dy=3 * A, dd=L.F32, ds=10, w=4 * A, wd=L.F32, dx=5 * A, dxs=10, dw=6 * A,
             db=7 * A, ws=8 * A, wb=1 << 29)
    a.update(k)
    return L.load().edb_layer_norm_grad(*a.values(), None)


def _linear(**k):
    a = dict(x=A, w=2 * A, d=L.F32, n=4, k=10, m=12, xs=10, wst=12, turned=0, b=3 * A, bd=L.F32, act=0, r=4 * A, rd=L.F32, rs=12,
             out=5 * A, od=L.F32, os=12, pre=6 * A, ps=12, ws=7 * A, wb=1 << 29)
    a.update(k)
    return L.load().edb_linear(*a.values(), None)


def _linear_grad(**k):
    a = dict(x=A, w=2 * A, d=L.F32, n=4, k=10, m=12, xs=10, wst=12, turned=0, dy=3 * A, dd=L.F32, ds=12, act=1, pre=4 * A, ps=12,
             dx=5 * A, dxs=10, dw=6 * A, dws=12, db=7 * A, ws=8 * A, wb=1 << 29)
    a.update(k)
    return L.load().edb_linear_grad(*a.values(), None)


REFUSED = (
    [(_norm, k, e) for k, e in [
        (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(xd=2), INVALID), (dict(od=-1), INVALID), (dict(wd=5), INVALID),
        (dict(n=-1), INVALID), (dict(D=0), INVALID), (dict(xs=9), INVALID), (dict(os=9), INVALID), (dict(eps=-1e-9), INVALID),
        (dict(eps=INF), INVALID), (dict(eps=float("nan")), INVALID), (dict(D=(1 << 20) + 1, xs=1 << 21, os=1 << 21), UNSUPPORTED),
        (dict(xs=1 << 47), INVALID), (dict(x=A + 2), INVALID), (dict(w=2 * A + 1), INVALID), (dict(b=3 * A + 2), INVALID),
        (dict(st=5 * A + 2), INVALID), (dict(out=A), INVALID), (dict(out=A + 156), INVALID), (dict(out=2 * A + 36), INVALID),
        (dict(out=3 * A - 156), INVALID), (dict(st=4 * A + 156), INVALID), (dict(st=A - 28), INVALID), (dict(st=2 * A), INVALID)]]
    + [(_norm_grad, k, e) for k, e in [
        (dict(x=None), INVALID), (dict(st=None), INVALID), (dict(dy=None), INVALID), (dict(xd=2), INVALID), (dict(dd=2), INVALID),
        (dict(wd=2), INVALID), (dict(n=-1), INVALID), (dict(D=0), INVALID), (dict(xs=9), INVALID), (dict(ds=9), INVALID),
        (dict(dxs=9), INVALID), (dict(ws=None), INVALID), (dict(wb=0), INVALID), (dict(ws=8 * A + 8), INVALID),
        (dict(D=(1 << 20) + 1, xs=1 << 21, ds=1 << 21, dxs=1 << 21), UNSUPPORTED), (dict(dx=A), INVALID), (dict(dx=3 * A), INVALID),
        (dict(dx=4 * A + 36), INVALID), (dict(dw=7 * A + 36), INVALID), (dict(dw=2 * A + 28), INVALID), (dict(db=3 * A + 156), INVALID),
        (dict(ws=A + 144), INVALID), (dict(ws=6 * A + 32), INVALID), (dict(dw=6 * A + 2), INVALID), (dict(st=2 * A + 1), INVALID)]]
    + [(_linear, k, e) for k, e in [
        (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(out=None), INVALID), (dict(d=2), INVALID), (dict(od=2), INVALID),
        (dict(bd=2), INVALID), (dict(rd=2), INVALID), (dict(n=-1), INVALID), (dict(k=0), INVALID), (dict(m=0), INVALID),
        (dict(act=-1), INVALID), (dict(act=5), INVALID), (dict(xs=9), INVALID), (dict(wst=11), INVALID), (dict(turned=1, wst=9), INVALID),
        (dict(os=11), INVALID), (dict(rs=11), INVALID), (dict(ps=11), INVALID), (dict(x=A + 1), INVALID), (dict(w=2 * A + 2), INVALID),
        (dict(b=3 * A + 2), INVALID), (dict(r=4 * A + 1), INVALID), (dict(out=5 * A + 2), INVALID), (dict(pre=6 * A + 2), INVALID),
        (dict(k=(1 << 24) + 1, xs=1 << 25), UNSUPPORTED), (dict(m=(1 << 24) + 1, wst=1 << 25, os=1 << 25, rs=1 << 25, ps=1 << 25), UNSUPPORTED),
        (dict(n=(1 << 30) + 1, k=129, xs=129), UNSUPPORTED), (dict(k=4000, xs=4000, wb=0), INVALID),
        (dict(k=4000, xs=4000, ws=None), INVALID), (dict(k=4000, xs=4000, ws=7 * A + 8), INVALID),
        (dict(out=A), INVALID), (dict(out=2 * A + 476), INVALID), (dict(out=3 * A + 44), INVALID), (dict(out=4 * A, os=24), INVALID),
        (dict(out=4 * A + 4), INVALID), (dict(out=4 * A, od=L.BF16), INVALID), (dict(out=6 * A + 188), INVALID), (dict(pre=4 * A), INVALID),
        (dict(pre=A + 156), INVALID), (dict(pre=3 * A), INVALID), (dict(k=4000, xs=4000, ws=5 * A), INVALID),
        (dict(k=4000, xs=4000, ws=4 * A), INVALID)]]
    + [(_linear_grad, k, e) for k, e in [
        (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(dy=None), INVALID), (dict(pre=None), INVALID), (dict(d=2), INVALID),
        (dict(dd=2), INVALID), (dict(n=-1), INVALID), (dict(k=0), INVALID), (dict(m=0), INVALID), (dict(act=9), INVALID),
        (dict(xs=9), INVALID), (dict(wst=11), INVALID), (dict(ds=11), INVALID), (dict(ps=11), INVALID), (dict(dxs=9), INVALID),
        (dict(dws=11), INVALID), (dict(turned=1, wst=10, dws=9), INVALID), (dict(wb=0), INVALID), (dict(ws=None), INVALID),
        (dict(ws=8 * A + 4), INVALID), (dict(db=7 * A + 2), INVALID), (dict(dx=A + 4), INVALID), (dict(dx=3 * A + 188), INVALID),
        (dict(dx=4 * A), INVALID), (dict(dw=2 * A), INVALID), (dict(dw=5 * A + 156), INVALID), (dict(db=6 * A + 476), INVALID),
        (dict(db=3 * A), INVALID), (dict(ws=3 * A + 176), INVALID), (dict(ws=7 * A + 32), INVALID)]])


@pytest.mark.parametrize("call,changed,status", REFUSED, ids=[f"{f.__name__[1:]}-{i}" for i, (f, _, _) in enumerate(REFUSED)])
def test_refusals(call, changed, status):
    """Refused on the host, with a message, before any launch (no GPU needed)."""
    assert call(**changed) == status
    assert L.load().edb_last_error()


@pytest.mark.parametrize("call", [_norm, _linear])
def test_nothing_to_do(call):
    assert call(n=0) == L.EDB_OK
    assert _norm_grad(n=0, dw=None, db=None) == L.EDB_OK and _norm_grad(dx=None, dw=None, db=None) == L.EDB_OK
    assert _linear_grad(n=0, dw=None, db=None) == L.EDB_OK and _linear_grad(dx=None, dw=None, db=None) == L.EDB_OK


def test_workspace_sizes():
    lib, nb = L.load(), C.c_int64(-1)
    assert lib.edb_layer_norm_grad_bytes(500, 64, L.F32, C.byref(nb)) == L.EDB_OK and nb.value > 0
    assert lib.edb_layer_norm_grad_bytes(0, 64, L.F32, C.byref(nb)) == L.EDB_OK and nb.value == 0
    assert lib.edb_layer_norm_grad_bytes(2 ** 31 - 1, 1 << 20, L.BF16, C.byref(nb)) == L.EDB_OK and nb.value > 0
    assert lib.edb_layer_norm_grad_bytes(500, 0, L.F32, C.byref(nb)) == INVALID
    assert lib.edb_layer_norm_grad_bytes(500, 64, 3, C.byref(nb)) == INVALID
    assert lib.edb_layer_norm_grad_bytes(500, 64, L.F32, None) == INVALID
    assert lib.edb_linear_bytes(10, 5000, 64, L.F32, C.byref(nb)) == L.EDB_OK and nb.value > 0
    assert lib.edb_linear_bytes(0, 5000, 64, L.F32, C.byref(nb)) == L.EDB_OK and nb.value == 0
    assert lib.edb_linear_bytes(10, 5000, 64, 2, C.byref(nb)) == INVALID
    assert lib.edb_linear_bytes(10, 0, 64, L.F32, C.byref(nb)) == INVALID
    assert lib.edb_linear_bytes(10, 5000, 64, L.F32, None) == INVALID
    assert lib.edb_linear_grad_bytes(10, 50, 64, L.BF16, L.F32, 1, 7, C.byref(nb)) == L.EDB_OK and nb.value > 0
    assert lib.edb_linear_grad_bytes(10, 50, 64, L.BF16, L.F32, 1, 8, C.byref(nb)) == INVALID
    assert lib.edb_linear_grad_bytes(10, 50, 64, L.BF16, L.F32, 7, 7, C.byref(nb)) == INVALID
    assert lib.edb_linear_grad_bytes(10, 50, 64, L.BF16, 9, 1, 7, C.byref(nb)) == INVALID
    assert lib.edb_linear_grad_bytes(10, 50, 64, L.BF16, L.F32, 1, 7, None) == INVALID
    assert lib.edb_linear_grad_bytes(2 ** 31 - 1, 1 << 24, 64, L.BF16, L.F32, 1, 7, C.byref(nb)) == UNSUPPORTED


def test_python_checks():
    """Tensors that no call may take (CPU tensors, wrong types and shapes), and sizes past 31 bits."""
    from paper_2302_03851_amd import head
    w = torch.zeros((4, 8))
    big = torch.empty((2 ** 31, 1), dtype=BF16, device="meta")
    for bad in (w, w.double(), w.view(-1), w.t(), big):
        for f in (lambda: head.layer_norm(bad), lambda: head.layer_norm_grad(bad, w, w), lambda: head.linear(bad, w),
                  lambda: head.linear_grad(bad, w, w)):
            with pytest.raises(ValueError):
                f()


@gpu
def test_python_checks_gpu():
    from paper_2302_03851_amd import head
    x, w = torch.zeros((4, 8), device="cuda"), torch.zeros((8, 6), device="cuda")
    y, st, h = torch.zeros((4, 6), device="cuda"), torch.zeros((4, 2), device="cuda"), torch.zeros(8, device="cuda")
    bad = [lambda: head.layer_norm(x, h[:7]), lambda: head.layer_norm(x, h.double()), lambda: head.layer_norm(x, h, h.to(BF16)),
           lambda: head.layer_norm(x, out=head.Normed(y, st)), lambda: head.layer_norm(x, dtype=BF16, out=head.Normed(x.clone(), st)),
           lambda: head.layer_norm(x, h.cpu()), lambda: head.layer_norm(x[:, ::2]), lambda: head.layer_norm_grad(x, st[:3], x),
           lambda: head.layer_norm_grad(x, st, y), lambda: head.layer_norm_grad(x, st, x, out=head.NormGrad(None, h, h)),
           lambda: head.layer_norm_grad(x, st, x, out=head.NormGrad(x.clone(), None, h)), lambda: head.linear(x, w.t()),
           lambda: head.linear(x, w.to(BF16)), lambda: head.linear(x, w, h), lambda: head.linear(x, w, act="sine"),
           lambda: head.linear(x, w, residual=x), lambda: head.linear(x, w, residual=y.cpu()), lambda: head.linear(x, w[:, ::2]),
           lambda: head.linear(x, w, keep=True, out=head.Linear(y, None)), lambda: head.linear(x, w, out=head.Linear(x, None)),
           lambda: head.linear_grad(x, w, x), lambda: head.linear_grad(x, w, y, "relu"), lambda: head.linear_grad(x, w, y, "none", y),
           lambda: head.linear_grad(x, w, y, "relu", y.to(BF16)), lambda: head.linear_grad(x, w, y, out=head.LinearGrad(None, w, h[:6])),
           lambda: head.linear_grad(x, w, y, out=head.LinearGrad(x, w.t(), h[:6]))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: head.layer_norm(x, eps=-1.0), lambda: head.layer_norm(x, out=head.Normed(x, st)),
              lambda: head.linear(x, w, out=head.Linear(x[:, :6], None))):
        with pytest.raises(L.EdbError):
            f()
