"""The two ends of a decoder on its vocabulary: the embedding of token ids and
the softmax cross entropy, each with its gradient (include/ultramem.h, "the two
ends of a decoder on its vocabulary").

    x = embedding(table, ids, scale)                        # [T] ids -> [T, D]
    loss, lse = cross_entropy(h, w_out, labels)             # [T] fp32 each, no logits kept
    dh, dw_out = cross_entropy_backward(h, w_out, labels, lse, dloss)
    dtable = embedding_backward(ids, dx, vocab, scale)      # summed in a fixed order

With one table at both ends, dw_out is the table's gradient from the loss and
``embedding_backward(..., dtable=dw_out, accumulate=True)`` adds the other part.

As in binding.py, these functions marshal arguments only; there is no fallback,
and an argument that the library cannot take raises.  They launch on the
current stream of the current device, where every tensor has to lie, and
autograd does not see them.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.F32, torch.bfloat16: _b.BF16}
_INTS = {torch.int32: 4, torch.int64: 8}


def _matrix(name, t, dev):
    """A [rows, columns] tensor whose rows may be strided apart, its sizes and
    the rows' distance."""
    shape = t.shape
    if len(shape) != 2 or t.dtype not in _DTYPES or t.get_device() != dev:
        raise ValueError(f"{name} must be a tensor [rows, columns], fp32 or bf16, on the current "
                         "device")
    rows, columns = shape
    if columns < 1:
        raise ValueError(f"{name} must have columns")
    _b._fits_int32(rows, columns)
    s0, s1 = t.stride()
    if s0 >= columns and (s1 == 1 or columns == 1):
        return t, rows, columns, s0
    if rows > 1 or (s1 != 1 and columns > 1):
        t = t.contiguous()
    return t, rows, columns, columns


def _ids(name, t, n, dev):
    if t.dtype not in _INTS or t.get_device() != dev or not t.is_contiguous() or \
            t.shape != (n,):
        raise ValueError(f"{name} must be a contiguous int32 or int64 tensor of {n} entries on the "
                         "current device")
    return t.data_ptr(), _INTS[t.dtype]


def _floats(name, t, n, dev):
    if t.dtype != torch.float32 or t.get_device() != dev or not t.is_contiguous() or \
            t.shape != (n,):
        raise ValueError(f"{name} must be a contiguous fp32 tensor of {n} entries on the current "
                         "device")
    return t.data_ptr()


def _output(name, t, shape, dtype, dev):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name} must be a contiguous tensor {tuple(shape)} of {dtype} on the "
                         "current device")
    return t


def _gradient(name, t, shape, dtype, dev, device):
    """An output asked for (True), given, or left out (None or False)."""
    if t is True:
        return torch.empty(shape, dtype=dtype, device=device)
    return None if t is None or t is False else _output(name, t, shape, dtype, dev)


def embedding(table, ids, scale: float = 1.0, out=None):
    """out [T, D] = scale * table[ids] for ids [T] (int32 or int64) into table
    [V, D]; a zero row for an id outside [0, V)."""
    dev = _b._on_device("table", table)
    table, V, D, ld = _matrix("table", table, dev)
    T = ids.numel()
    _b._fits_int32(T)
    p_ids, ids_bytes = _ids("ids", ids, T, dev)
    dtype = table.dtype
    if out is None:
        out = torch.empty((T, D), dtype=dtype, device=table.device)
    else:
        _output("out", out, (T, D), dtype, dev)
    lib = _b._lib or _b.load()
    status = lib.ultramem_embedding(table.data_ptr(), ld, _DTYPES[dtype], V, D, p_ids,
                                    ids_bytes, T, scale, out.data_ptr(), _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_embedding")
    return out


@functools.lru_cache(maxsize=256)
def _workspace(dev, name, *sizes):
    """Bytes of a call's workspace, a function of the sizes and the (current)
    device alone."""
    return int(getattr(_b.load(), name)(*sizes))


def embedding_backward(ids, dout, vocab: int, scale: float = 1.0, dtable=None,
                       accumulate: bool = False):
    """The gradient of the table: dtable [vocab, D] with row v = scale times the
    sum of dout [T, D] over the tokens with ids[t] = v, in dout's type unless
    ``dtable`` (fp32 or bf16) is given.  With ``accumulate`` the sums are added
    to what the given dtable holds.  The sums have an order that the sizes and
    the tensors' alignment fix."""
    dev = _b._on_device("dout", dout)
    dout, T, D, ld = _matrix("dout", dout, dev)
    _b._fits_int32(vocab)
    p_ids, ids_bytes = _ids("ids", ids, T, dev)
    if dtable is not None:
        if dtable.dtype not in _DTYPES:
            raise ValueError("dtable must be fp32 or bf16")
        _output("dtable", dtable, (vocab, D), dtable.dtype, dev)
    elif accumulate:
        raise ValueError("accumulate needs a dtable to add to")
    elif vocab < 1:
        raise ValueError("vocab must be positive")
    else:
        dtable = torch.empty((vocab, D), dtype=dout.dtype, device=dout.device)
    lib = _b._lib or _b.load()
    nbytes = _workspace(dev, "ultramem_embedding_backward_workspace", T, D)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dout.device)
    status = lib.ultramem_embedding_backward(
        p_ids, ids_bytes, T, dout.data_ptr(), ld, _DTYPES[dout.dtype], vocab, D, scale,
        dtable.data_ptr(), _DTYPES[dtable.dtype], 1 if accumulate else 0, ws.data_ptr(), nbytes,
        _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_embedding_backward")
    return dtable


def _ce_args(x, w, labels, logit_scale):
    dev = _b._on_device("x", x)
    x, T, D, ld_x = _matrix("x", x, dev)
    w, V, w_dim, ld_w = _matrix("w", w, dev)
    dtype = x.dtype
    if w_dim != D or w.dtype != dtype:
        raise ValueError("w must be [vocab, dim] of x's type")
    p_labels, labels_bytes = _ids("labels", labels, T, dev)
    code = _DTYPES[dtype]
    a = _b.CrossEntropyArgs(x.data_ptr(), w.data_ptr(), p_labels, ld_x, ld_w, T, V, D, code,
                            labels_bytes, logit_scale)
    return a, x, w, dev, (code, T, V, D)


def cross_entropy(x, w, labels, logit_scale: float = 1.0):
    """(loss, lse), fp32 [T], of hidden states x [T, D] against the output
    weights w [V, D]: z = logit_scale * x w^T, lse = log sum e^z, loss = lse -
    z[label], at least 0.  A label outside [0, V) marks a token that does not
    count (loss 0).  The logits are not kept."""
    a, x, w, dev, sizes = _ce_args(x, w, labels, logit_scale)
    device = x.device
    loss = torch.empty(sizes[1], dtype=torch.float32, device=device)
    lse = torch.empty(sizes[1], dtype=torch.float32, device=device)
    lib = _b._lib or _b.load()
    nbytes = _workspace(dev, "ultramem_cross_entropy_workspace", *sizes)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    status = lib.ultramem_cross_entropy(C.byref(a), loss.data_ptr(), lse.data_ptr(),
                                        ws.data_ptr(), nbytes, _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_cross_entropy")
    return loss, lse


def cross_entropy_backward(x, w, labels, lse, dloss, logit_scale: float = 1.0, dx=True, dw=True):
    """(dx, dw) [T, D] and [V, D] in x's type, at the lse of ``cross_entropy``
    and for the gradients dloss [T] (fp32) of its losses.  ``dx`` and ``dw``
    may be contiguous tensors to write, or False to leave that one out
    (None is returned for it)."""
    a, x, w, dev, sizes = _ce_args(x, w, labels, logit_scale)
    _, T, V, D = sizes
    dtype, device = x.dtype, x.device
    p_lse, p_dloss = _floats("lse", lse, T, dev), _floats("dloss", dloss, T, dev)
    dx = _gradient("dx", dx, (T, D), dtype, dev, device)
    dw = _gradient("dw", dw, (V, D), dtype, dev, device)
    lib = _b._lib or _b.load()
    nbytes = _workspace(dev, "ultramem_cross_entropy_backward_workspace", *sizes)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    status = lib.ultramem_cross_entropy_backward(
        C.byref(a), p_lse, p_dloss, None if dx is None else dx.data_ptr(),
        None if dw is None else dw.data_ptr(), ws.data_ptr(), nbytes, _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_cross_entropy_backward")
    return dx, dw
