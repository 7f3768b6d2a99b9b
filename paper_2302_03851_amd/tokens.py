"""Token operators on torch tensors: embedding lookup and its gradient, log
probabilities of given tokens with entropy and alternatives and their
gradient, and distillation from a teacher's best logits (include/edb.h holds
the definitions).  PyTorch provides device memory and the stream only: every
call checks its tensors, enqueues libedb's kernels on the current stream of
the tensors' device and returns without waiting.

Matrices are 2-D fp32 or bf16 tensors whose rows are contiguous (any row
stride); ids are int32, -1 for no token.  ``out`` takes the result of an
earlier call of the same sizes to be written again; without it a new one is
allocated.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import NamedTuple, Optional

import torch

from . import _lib as L

_DTYPE = {torch.float32: L.F32, torch.bfloat16: L.BF16}


class LogProbs(NamedTuple):
    logprob: Optional[torch.Tensor]        # float32 [n], None without ids
    entropy: torch.Tensor                  # float32 [n]
    stats: torch.Tensor                    # float32 [n, 2], for logprobs_grad
    top_ids: torch.Tensor                  # int32 [n, top]
    top_logprobs: torch.Tensor             # float32 [n, top]


class Distilled(NamedTuple):
    loss: torch.Tensor                     # float32 [n]
    dlogits: Optional[torch.Tensor]        # like the logits, None for the loss alone


_MOST = 2 ** 31 - 1     # of a size: the C calls take int32, and ctypes would cut off the rest


def _size(v, name):
    """A size that the C calls can take."""
    if not 0 <= v <= _MOST:
        raise ValueError(f"{name}: {v} is not a size from 0 to {_MOST}")
    return v


def _matrix(t, name, dev=None):
    """Rows, columns and row stride in elements of a matrix operand."""
    if t.dim() != 2 or t.dtype not in _DTYPE:
        raise ValueError(f"{name}: a 2-D float32 or bfloat16 tensor is needed, not {t.dim()}-D {t.dtype}")
    n, m = t.shape
    if n > _MOST or m > _MOST:
        raise ValueError(f"{name}: {n} x {m} is more than {_MOST} rows or columns")
    if dev is None or t.device != dev:
        _on(t, name, dev)
    s, one = t.stride()
    if one != 1 and m > 1:
        raise ValueError(f"{name}: the rows must be contiguous")
    if s >= m:
        return n, m, s
    if n > 1:
        raise ValueError(f"{name}: the rows overlap")
    return n, m, m


def _on(t, name, dev):
    if not t.is_cuda:
        raise ValueError(f"{name}: must be on the GPU")
    if dev is not None and t.device != dev:
        raise ValueError(f"{name}: must be on {dev}, not {t.device}")


def _array(t, name, shape, dtype, dev):
    """Address of a dense operand of one type (no copies are made)."""
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {shape} is needed, not {t.dtype} {tuple(t.shape)}")
    if t.device != dev:
        _on(t, name, dev)
    return t.data_ptr()


# the current stream's handle; the public call builds a Stream object first (2.5 us a call, this 0.1)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_entry = {}


def _call(name, dev, *args):
    """Run one entry point on the current stream of `dev`."""
    fn = _entry.get(name)
    if fn is None:
        fn = _entry[name] = getattr(L.load(), name)
    index = dev.index
    if torch.cuda.current_device() == index:
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _raw_stream(index))
    if status:
        L.check(status, name)


@functools.lru_cache(maxsize=1024)
def _bytes(name, *args):
    nb = C.c_int64()
    L.check(getattr(L.load(), name)(*args, C.byref(nb)), name)
    return nb.value


def _workspace(dev, nb):
    """Scratch memory of the current stream: torch hands it to later work of that stream only."""
    if not nb:
        return None
    if torch.cuda.current_device() == dev.index:
        return torch.empty(nb, dtype=torch.uint8, device=dev)
    with torch.cuda.device(dev):   # its stream, not the current device's
        return torch.empty(nb, dtype=torch.uint8, device=dev)


def embed(ids, table, scale: float = 1.0, dtype=None, out=None) -> torch.Tensor:
    """Rows of `table` [vocab, dim] at `ids` [n], times `scale`, as `dtype`
    (the table's by default); a zero row where an id is no token."""
    vocab, dim, stride = _matrix(table, "table")
    dev = table.device
    n = _size(ids.numel(), "ids")
    ip = _array(ids, "ids", (n,), torch.int32, dev)
    if out is None:
        out = torch.empty((n, dim), dtype=dtype or table.dtype, device=dev)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError(f"out: {dtype} is asked for, not {out.dtype}")
    on, om, ostride = _matrix(out, "out", dev)
    if (on, om) != (n, dim):
        raise ValueError(f"out: {n} x {dim} is needed, not {on} x {om}")
    _call("edb_embed", dev, ip, n, table.data_ptr(), _DTYPE[table.dtype], vocab, dim, stride, scale, out.data_ptr(),
          _DTYPE[out.dtype], ostride)
    return out


def embed_grad(ids, dout, vocab: int, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False) -> torch.Tensor:
    """Gradient [vocab, dim] of the table of ``embed(ids, table, scale)`` from
    `dout` [n, dim], as `dtype` (float32 by default); with `accumulate` it is
    added to `out`."""
    n, dim, stride = _matrix(dout, "dout")
    _size(vocab, "vocab")
    dev = dout.device
    ip = _array(ids, "ids", (n,), torch.int32, dev)
    if out is None:
        if accumulate:
            raise ValueError("out: needed to accumulate")
        out = torch.empty((vocab, dim), dtype=dtype or torch.float32, device=dev)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError(f"out: {dtype} is asked for, not {out.dtype}")
    on, om, ostride = _matrix(out, "out", dev)
    if (on, om) != (vocab, dim):
        raise ValueError(f"out: {vocab} x {dim} is needed, not {on} x {om}")
    nb = _bytes("edb_embed_grad_bytes", n, vocab, dim)
    ws = _workspace(dev, nb)
    _call("edb_embed_grad", dev, ip, n, dout.data_ptr(), _DTYPE[dout.dtype], vocab, dim, stride, scale,
          1 if accumulate else 0, out.data_ptr(), _DTYPE[out.dtype], ostride, ws.data_ptr() if nb else None, nb)
    return out


def logprobs(logits, ids=None, temperature: float = 1.0, top: int = 0, out: Optional[LogProbs] = None) -> LogProbs:
    """Log probabilities of the tokens `ids` [n] under softmax(logits /
    temperature), the rows' entropies and the `top` best alternatives."""
    n, vocab, stride = _matrix(logits, "logits")
    _size(top, "top")
    dev, dt = logits.device, _DTYPE[logits.dtype]
    ip = None if ids is None else _array(ids, "ids", (n,), torch.int32, dev)
    f32 = torch.float32
    if out is None:
        out = LogProbs(None if ids is None else torch.empty(n, dtype=f32, device=dev),
                       torch.empty(n, dtype=f32, device=dev), torch.empty((n, 2), dtype=f32, device=dev),
                       torch.empty((n, top), dtype=torch.int32, device=dev),
                       torch.empty((n, top), dtype=f32, device=dev))
    if (out.logprob is None) != (ids is None):
        raise ValueError("out: made with ids and used without, or the other way round")
    lp = None if ids is None else _array(out.logprob, "out.logprob", (n,), f32, dev)
    nb = _bytes("edb_logprobs_bytes", n, vocab, dt, top)
    ws = _workspace(dev, nb)
    _call("edb_logprobs", dev, logits.data_ptr(), dt, n, vocab, stride, ip, temperature, top, lp,
          _array(out.entropy, "out.entropy", (n,), f32, dev), _array(out.stats, "out.stats", (n, 2), f32, dev),
          _array(out.top_ids, "out.top_ids", (n, top), torch.int32, dev),
          _array(out.top_logprobs, "out.top_logprobs", (n, top), f32, dev), ws.data_ptr() if nb else None, nb)
    return out


def logprobs_grad(logits, ids, stats, entropy=None, g_logprob=None, g_entropy=None, temperature: float = 1.0,
                  out=None) -> torch.Tensor:
    """Gradient of the logits from those of ``logprobs``' log probabilities and
    entropies ([n] each, None for zero); `out` may be the logits themselves."""
    n, vocab, stride = _matrix(logits, "logits")
    dev, dt = logits.device, _DTYPE[logits.dtype]
    f32 = torch.float32
    if out is None:
        out = torch.empty((n, vocab), dtype=logits.dtype, device=dev)
    on, om, ostride = _matrix(out, "out", dev)
    if (on, om) != (n, vocab) or out.dtype != logits.dtype:
        raise ValueError(f"out: {n} x {vocab} {logits.dtype} is needed, not {on} x {om} {out.dtype}")
    if out.data_ptr() == logits.data_ptr():
        ostride = stride if on <= 1 else ostride
    _call("edb_logprobs_grad", dev, logits.data_ptr(), dt, n, vocab, stride,
          _array(ids, "ids", (n,), torch.int32, dev), temperature, _array(stats, "stats", (n, 2), f32, dev),
          None if entropy is None else _array(entropy, "entropy", (n,), f32, dev),
          None if g_logprob is None else _array(g_logprob, "g_logprob", (n,), f32, dev),
          None if g_entropy is None else _array(g_entropy, "g_entropy", (n,), f32, dev), out.data_ptr(), ostride)
    return out


def distill(logits, top_ids, top_logits, temperature: float = 1.0, weight=None, grad: bool = True,
            out: Optional[Distilled] = None) -> Distilled:
    """Loss of every row against the teacher's listed logits ([n, top] ids and
    float32 logits) and, with `grad`, the logits' gradient of the losses' sum
    weighted by `weight` [n]; ``out.dlogits`` may be the logits themselves."""
    n, vocab, stride = _matrix(logits, "logits")
    dev, dt = logits.device, _DTYPE[logits.dtype]
    f32 = torch.float32
    if top_ids.dim() != 2:
        raise ValueError("top_ids: a 2-D tensor is needed")
    top = _size(top_ids.shape[1], "top_ids")
    if out is None:
        out = Distilled(torch.empty(n, dtype=f32, device=dev),
                        torch.empty((n, vocab), dtype=logits.dtype, device=dev) if grad else None)
    dp, ostride = None, vocab
    if grad:
        if out.dlogits is None:
            raise ValueError("out: has no gradient to write")
        d = out.dlogits
        on, om, ostride = _matrix(d, "out.dlogits", dev)
        if (on, om) != (n, vocab) or d.dtype != logits.dtype:
            raise ValueError(f"out.dlogits: {n} x {vocab} {logits.dtype} is needed, not {on} x {om} {d.dtype}")
        dp = d.data_ptr()
        if dp == logits.data_ptr():
            ostride = stride if on <= 1 else ostride
    nb = _bytes("edb_distill_bytes", n, vocab, dt, top) if top else 0
    ws = _workspace(dev, nb)
    _call("edb_distill", dev, logits.data_ptr(), dt, n, vocab, stride,
          _array(top_ids, "top_ids", (n, top), torch.int32, dev),
          _array(top_logits, "top_logits", (n, top), f32, dev), top, temperature,
          None if weight is None else _array(weight, "weight", (n,), f32, dev),
          _array(out.loss, "out.loss", (n,), f32, dev), dp, ostride, ws.data_ptr() if nb else None, nb)
    return out
