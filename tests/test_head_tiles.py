"""Every tile of the linear layers' products in every layout, with k whole and split: odd sizes in all three directions,
row strides of odd lengths with NaN between the rows, the bias's gradient within the weight's product and beside it, a
residual that is the result's place.

Dense products have the tolerances of test_head.py.  Those grow with the number of terms, so products with one term a
result are there besides: whatever the sizes, such a result is that term to the last bit (fp32 factors are the sum of
three bf16 pieces, and each of the pieces' products and sums on the way is exact)."""
import ctypes as C

import pytest

from paper_2302_03851_amd import _lib as L

torch = pytest.importorskip("torch")
from test_head import BF16, F32, _check_linear, _check_linear_grad, _gen, _only, _view   # noqa: E402

gpu = pytest.mark.gpu
SHAPES = {
    BF16: [(31, 65, 63), (19713, 327, 333), (193, 1169, 12425), (467, 6393, 1031), (1529, 357, 9383), (6053, 5055, 231), (10825, 3515, 65),
           (6611, 411, 5423), (5647, 6253, 393), (411, 5647, 6035)],
    F32: [(31, 67, 61), (137, 129, 131), (4737, 3687, 67), (193, 453, 28423)],
}
FEW = [(13, 63, 16391), (13, 2051, 16391), (11, 16387, 61), (11, 16387, 2053), (59, 9, 16399), (2055, 9, 16399), (59, 16395, 7), (2055, 16395, 7)]
for _shapes in SHAPES.values():
    _shapes.extend(FEW)
CASES = [pytest.param(*s, T, id=f"{'-'.join(map(str, s))}-{'bf16' if T == BF16 else 'fp32'}") for T in SHAPES for s in SHAPES[T]]


def _plan(n, k, m, T):
    """Tile and number of parts of a product of n x k by k x m."""
    rows, cols, splits = C.c_int32(), C.c_int32(), C.c_int32()
    L.check(L.load().edb_linear_plan(n, k, m, L.BF16 if T == BF16 else L.F32, C.byref(rows), C.byref(cols), C.byref(splits)), "edb_linear_plan")
    return rows.value, cols.value, splits.value


def _products(n, k, m, T):
    return {"out": _plan(n, k, m, T), "dx": _plan(n, m, k, T), "dweight": _plan(k, n, m, T), "dweight turned": _plan(m, n, k, T)}


def test_every_tile_is_there():
    """The shapes below reach every tile with every layout of its operands, with k in one part and in several."""
    tiles = {BF16: [(128, 128), (64, 64), (16, 256), (256, 256), (256, 128)], F32: [(128, 128), (64, 64), (16, 256)]}
    for T in SHAPES:
        there = {(name, p[:2], p[2] > 1) for s in SHAPES[T] for name, p in _products(*s, T).items()}
        wanted = {(name, tile, split) for name in ("out", "dx", "dweight", "dweight turned") for tile in tiles[T] for split in (False, True)}
        assert not wanted - there, sorted(wanted - there)


def test_plan_refusals():
    r = [C.c_int32() for _ in range(3)]
    f = L.load().edb_linear_plan
    assert f(10, 20, 30, L.F32, *map(C.byref, r)) == L.EDB_OK and all(x.value > 0 for x in r)
    assert f(10, 20, 30, 7, *map(C.byref, r)) == L.EDB_ERR_INVALID and f(10, 0, 30, L.F32, *map(C.byref, r)) == L.EDB_ERR_INVALID
    assert f(10, (1 << 24) + 1, 30, L.F32, *map(C.byref, r)) == L.EDB_ERR_UNSUPPORTED
    for i in range(3):
        assert f(10, 20, 30, L.F32, *(None if i == j else C.byref(x) for j, x in enumerate(r))) == L.EDB_ERR_INVALID


def _normal(g, *shape, T):
    return torch.randn(shape, generator=g, device="cuda").to(T)


def _turn(w, turned, pad, shift):
    """The same weight, stored either way in a buffer with NaN between its lines."""
    return _view(w.t().contiguous(), pad, shift)[0].t() if turned else _view(w, pad, shift)[0]


@gpu
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("n,k,m,T", CASES)
def test_products(n, k, m, T, turned):
    from paper_2302_03851_amd import head
    g = _gen(n + k + m)
    x, _ = _view(_normal(g, n, k, T=T), 5, 3)
    w = _turn(_normal(g, k, m, T=T) / k ** 0.5, turned, 9, 1)
    bias = _normal(g, m, T=F32)
    # the residual's place takes the result; what stands before the activation is kept
    res = _normal(g, n, m, T=T)
    place, mem = _view(res, 1, 5)
    before = mem.clone()
    pre, _ = _view(torch.zeros_like(res), 3, 1)
    r = head.linear(x, w, bias, "silu", place, keep=True, out=head.Linear(place, pre))
    _check_linear(x, w, bias, "silu", res, r)
    _only(mem, before, place, res)
    other = F32 if T == BF16 else BF16
    r = head.linear(x, w, None, "none", dtype=other)
    _check_linear(x, w, None, "none", None, r)
    # gradients: summed within the weight's product, of another type, and through an activation
    for act, O in (("none", T), ("none", other), ("gelu", T)):
        dy, _ = _view(_normal(g, n, m, T=O), 7, 2)
        v = None if act == "none" else _view(_normal(g, n, m, T=T) * 2, 1, 1)[0]
        dx, xmem = _view(torch.zeros((n, k), dtype=T, device="cuda"), 3, 1)
        dw, wmem = _view(torch.zeros((m, k) if turned else (k, m), dtype=T, device="cuda"), 5, 7)
        xbefore, wbefore, xold, wold = xmem.clone(), wmem.clone(), dx.clone(), dw.clone()
        q = head.linear_grad(x, w, dy, act, v, out=head.LinearGrad(dx, dw.t() if turned else dw, torch.empty(m, device="cuda")))
        _check_linear_grad(x, w, dy, act, v, q)
        _only(xmem, xbefore, dx, xold)
        _only(wmem, wbefore, dw, wold)


def _ones(g, rows, cols, T):
    """A matrix of one +-2^e in every column, the rows that they stand in, and the numbers."""
    at = torch.randint(0, rows, (cols,), generator=g, device="cuda")
    v = torch.ldexp(torch.ones(cols, device="cuda"), torch.randint(-3, 4, (cols,), generator=g, device="cuda"))
    v = v * (torch.randint(0, 2, (cols,), generator=g, device="cuda") * 2 - 1)
    o = torch.zeros((rows, cols), device="cuda")
    o[at, torch.arange(cols, device="cuda")] = v
    return o.to(T), at, v


@gpu
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("n,k,m,T", CASES)
def test_products_of_one_term(n, k, m, T, turned):
    from paper_2302_03851_amd import head
    g = _gen(n + k * m)
    x, _ = _view(_normal(g, n, k, T=T), 3, 1)
    dy, _ = _view(_normal(g, n, m, T=T), 1, 3)
    # out[:, j] = x[:, at[j]] v[j]
    w, at, v = _ones(g, k, m, T)
    w = _turn(w, turned, 1, 1)
    assert torch.equal(head.linear(x, w).out, (x[:, at].double() * v).to(T))
    # dx[:, i] = dy[:, at[i]] v[i]
    w, at, v = _ones(g, m, k, T)
    w = _turn(w.t().contiguous(), turned, 3, 5)
    assert torch.equal(head.linear_grad(x, w, dy, dweight=False, dbias=False).dx, (dy[:, at].double() * v).to(T))
    # dweight[i, :] = dy[at[i], :] v[i], and the other way round
    one, at, v = _ones(g, n, k, T)
    assert torch.equal(head.linear_grad(_view(one, 3, 1)[0], w, dy, dx=False).dweight, (dy[at].double() * v[:, None]).to(T))
    one, at, v = _ones(g, n, m, T)
    q = head.linear_grad(x, w, _view(one, 5, 1)[0], dx=False)
    assert torch.equal(q.dweight, (x[at].double() * v[:, None]).to(T).t())
    assert torch.equal(q.dbias, v)


@gpu
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("n,k,m,T", CASES)
def test_products_repeat_themselves(n, k, m, T, turned):
    """The same bits in every run."""
    from paper_2302_03851_amd import head
    g = _gen(n * k + m)
    x, dy = _normal(g, n, k, T=T), _normal(g, n, m, T=T)
    w = _turn(_normal(g, k, m, T=T), turned, 1, 1)
    bias = _normal(g, m, T=F32)

    def go():
        r = head.linear(x, w, bias, "tanh", keep=True)
        return [*r, *head.linear_grad(x, w, dy), *head.linear_grad(x, w, dy, "tanh", r.pre)]
    ref = go()
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(go(), ref))
