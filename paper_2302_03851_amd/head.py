"""The head on the cells' states, on torch tensors: layer norm and linear layers
(matrix product with bias, activation and residual), with their gradients
(include/edb.h holds the definitions).  Between the states and the vocabulary
logits of ``tokens``, and in its manner: every call checks its tensors,
enqueues libedb's kernels on the current stream of the tensors' device and
returns without waiting.

Matrices are 2-D fp32 or bf16 tensors whose rows are contiguous (any row
stride).  ``out`` takes the result of an earlier call of the same sizes to be
written again; without it a new one is allocated.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import _lib as L
from .tokens import _DTYPE, _array, _bytes, _call, _matrix, _optional, _workspace

_ACT = {"none": L.ACT_NONE, "relu": L.ACT_RELU, "gelu": L.ACT_GELU, "silu": L.ACT_SILU, "tanh": L.ACT_TANH}


class Normed(NamedTuple):
    out: torch.Tensor                      # [n, dim]
    stats: torch.Tensor                    # float32 [n, 2]: mean and rstd, for layer_norm_grad


class NormGrad(NamedTuple):
    dx: Optional[torch.Tensor]             # like x
    dweight: Optional[torch.Tensor]        # float32 [dim]
    dbias: Optional[torch.Tensor]          # float32 [dim]


class Linear(NamedTuple):
    out: torch.Tensor                      # [n, m]
    pre: Optional[torch.Tensor]            # [n, m] like x: before the activation, for linear_grad


class LinearGrad(NamedTuple):
    dx: Optional[torch.Tensor]             # like x
    dweight: Optional[torch.Tensor]        # like the weight, stored as it is
    dbias: Optional[torch.Tensor]          # float32 [m]


def _shaped(t, name, n, m, dtype, dev):
    """Row stride of a matrix operand of known sizes (and type, if given)."""
    on, om, stride = _matrix(t, name, dev)
    if (on, om) != (n, m) or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name}: {n} x {m}{'' if dtype is None else f' {dtype}'} is needed, not {on} x {om} {t.dtype}")
    return stride


def _vector(t, name, m, dev):
    """Address and type of a vector operand, fp32 or bf16; None for none."""
    if t is None:
        return None, L.F32
    if t.dtype not in _DTYPE:
        raise ValueError(f"{name}: float32 or bfloat16 is needed, not {t.dtype}")
    return _array(t, name, (m,), t.dtype, dev), _DTYPE[t.dtype]


def _pair(weight, bias, dim, dev):
    wp, wt = _vector(weight, "weight", dim, dev)
    bp, bt = _vector(bias, "bias", dim, dev)
    if wp is not None and bp is not None and wt != bt:
        raise ValueError(f"bias: {weight.dtype} is needed, not {bias.dtype}")
    return wp, bp, bt if wp is None else wt


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, dtype=None, out: Optional[Normed] = None) -> Normed:
    """Rows of `x` [n, dim] less their mean, by their deviation, times `weight`
    [dim], plus `bias` [dim], as `dtype` (x's by default)."""
    n, dim, stride = _matrix(x, "x")
    dev = x.device
    if out is None:
        out = Normed(torch.empty((n, dim), dtype=dtype or x.dtype, device=dev),
                     torch.empty((n, 2), dtype=torch.float32, device=dev))
    ostride = _shaped(out.out, "out.out", n, dim, dtype, dev)
    wp, bp, wt = _pair(weight, bias, dim, dev)
    _call("edb_layer_norm", dev, x.data_ptr(), _DTYPE[x.dtype], n, dim, stride, wp, bp, wt, eps, out.out.data_ptr(),
          _DTYPE[out.out.dtype], ostride, _array(out.stats, "out.stats", (n, 2), torch.float32, dev))
    return out


def layer_norm_grad(x, stats, dout, weight=None, dx: bool = True, sums: bool = True,
                    out: Optional[NormGrad] = None) -> NormGrad:
    """Gradients of ``layer_norm`` from that of its result, with the stats that
    it left: of `x` (with `dx`), and of the weight and the bias (with `sums`)."""
    n, dim, stride = _matrix(x, "x")
    dev, f32 = x.device, torch.float32
    dstride = _shaped(dout, "dout", n, dim, None, dev)
    wp, wt = _vector(weight, "weight", dim, dev)
    if out is None:
        out = NormGrad(torch.empty((n, dim), dtype=x.dtype, device=dev) if dx else None,
                       *(torch.empty(dim, dtype=f32, device=dev) if sums else None for _ in range(2)))
    xstride = dim
    if dx:
        if out.dx is None:
            raise ValueError("out: has no dx to write")
        xstride = _shaped(out.dx, "out.dx", n, dim, x.dtype, dev)
    if sums and (out.dweight is None or out.dbias is None):
        raise ValueError("out: has no sums to write")
    nb = _bytes("edb_layer_norm_grad_bytes", n, dim, _DTYPE[x.dtype]) if sums else 0
    ws = _workspace(dev, nb)
    _call("edb_layer_norm_grad", dev, x.data_ptr(), _DTYPE[x.dtype], n, dim, stride,
          _array(stats, "stats", (n, 2), f32, dev), dout.data_ptr(), _DTYPE[dout.dtype], dstride, wp, wt,
          out.dx.data_ptr() if dx else None, xstride, _array(out.dweight, "out.dweight", (dim,), f32, dev) if sums else None,
          _array(out.dbias, "out.dbias", (dim,), f32, dev) if sums else None, ws.data_ptr() if nb else None, nb)
    return out


def _weight(w, name, dev):
    """Rows and columns of a weight, whether it is stored column by column, and
    the stride of what it is stored by."""
    if w.dim() == 2 and w.stride(1) != 1 and w.shape[1] > 1 and (w.stride(0) == 1 or w.shape[0] == 1):
        m, k, stride = _matrix(w.t(), name, dev)
        return k, m, 1, stride
    k, m, stride = _matrix(w, name, dev)
    return k, m, 0, stride


def _like(w, turned):
    k, m = w.shape
    return torch.empty((m, k), dtype=w.dtype, device=w.device).t() if turned else torch.empty((k, m), dtype=w.dtype, device=w.device)


def _act(act):
    if act not in _ACT:
        raise ValueError(f"act: one of {', '.join(_ACT)} is needed, not {act}")
    return _ACT[act]


def _operands(x, weight):
    n, k, stride = _matrix(x, "x")
    wk, m, turned, wstride = _weight(weight, "weight", x.device)
    if wk != k or weight.dtype != x.dtype:
        raise ValueError(f"weight: {k} rows of {x.dtype} are needed, not {wk} of {weight.dtype}")
    return n, k, m, stride, turned, wstride


def linear(x, weight, bias=None, act: str = "none", residual=None, dtype=None, keep: bool = False,
           out: Optional[Linear] = None) -> Linear:
    """act(x weight + bias) + residual, as `dtype` (x's by default): `x` [n, k],
    `weight` [k, m] of the same type, stored row by row or column by column (the
    transpose of an [m, k] tensor), `bias` [m], `residual` [n, m].  `act` is
    "none", "relu", "gelu", "silu" or "tanh".  With `keep` the values before the
    activation are kept for ``linear_grad``.  ``out.out`` may be the residual
    itself."""
    n, k, m, stride, turned, wstride = _operands(x, weight)
    dev, dt, code = x.device, _DTYPE[x.dtype], _act(act)
    if out is None:
        out = Linear(torch.empty((n, m), dtype=dtype or x.dtype, device=dev),
                     torch.empty((n, m), dtype=x.dtype, device=dev) if keep else None)
    ostride = _shaped(out.out, "out.out", n, m, dtype, dev)
    pstride = m
    if keep:
        if out.pre is None:
            raise ValueError("out: has no pre to write")
        pstride = _shaped(out.pre, "out.pre", n, m, x.dtype, dev)
    bp, bt = _vector(bias, "bias", m, dev)
    rp, rt, rstride = None, L.F32, m
    if residual is not None:
        rp, rstride = residual.data_ptr(), _shaped(residual, "residual", n, m, None, dev)
        rt = _DTYPE[residual.dtype]
    nb = _bytes("edb_linear_bytes", n, k, m, dt)
    ws = _workspace(dev, nb)
    _call("edb_linear", dev, x.data_ptr(), weight.data_ptr(), dt, n, k, m, stride, wstride, turned, bp, bt, code, rp, rt,
          rstride, out.out.data_ptr(), _DTYPE[out.out.dtype], ostride, out.pre.data_ptr() if keep else None, pstride,
          ws.data_ptr() if nb else None, nb)
    return out


def linear_grad(x, weight, dout, act: str = "none", pre=None, dx: bool = True, dweight: bool = True, dbias: bool = True,
                out: Optional[LinearGrad] = None) -> LinearGrad:
    """Gradients of ``linear`` from that of its result `dout` [n, m], with the
    values before the activation that it kept: of `x`, of the weight (stored as
    the weight is) and of the bias, each where wanted.  The residual's is `dout`."""
    n, k, m, stride, turned, wstride = _operands(x, weight)
    dev, dt, code, f32 = x.device, _DTYPE[x.dtype], _act(act), torch.float32
    dstride = _shaped(dout, "dout", n, m, None, dev)
    if (pre is None) != (act == "none"):
        raise ValueError("pre: needed with an activation, and only then")
    pp, pstride = (None, m) if pre is None else (pre.data_ptr(), _shaped(pre, "pre", n, m, x.dtype, dev))
    if out is None:
        out = LinearGrad(torch.empty((n, k), dtype=x.dtype, device=dev) if dx else None, _like(weight, turned) if dweight else None,
                         torch.empty(m, dtype=f32, device=dev) if dbias else None)
    xp, xstride, wp, wgstride = None, k, None, k if turned else m
    if dx:
        if out.dx is None:
            raise ValueError("out: has no dx to write")
        xp, xstride = out.dx.data_ptr(), _shaped(out.dx, "out.dx", n, k, x.dtype, dev)
    if dweight:
        if out.dweight is None:
            raise ValueError("out: has no dweight to write")
        stored = out.dweight.t() if turned else out.dweight
        wp, wgstride = stored.data_ptr(), _shaped(stored, "out.dweight", m if turned else k, k if turned else m, x.dtype, dev)
    if dbias and out.dbias is None:
        raise ValueError("out: has no dbias to write")
    results = (L.LINEAR_DX if dx else 0) | (L.LINEAR_DWEIGHT if dweight else 0) | (L.LINEAR_DBIAS if dbias else 0)
    nb = _bytes("edb_linear_grad_bytes", n, k, m, dt, _DTYPE[dout.dtype], code, results)
    ws = _workspace(dev, nb)
    _call("edb_linear_grad", dev, x.data_ptr(), weight.data_ptr(), dt, n, k, m, stride, wstride, turned, dout.data_ptr(),
          _DTYPE[dout.dtype], dstride, code, pp, pstride, xp, xstride, wp, wgstride,
          _array(out.dbias, "out.dbias", (m,), f32, dev) if dbias else None, ws.data_ptr() if nb else None, nb)
    return out
