"""The paged key/value cache of a decoder block: pages for a step's new
tokens, the cache write, and the attention that reads it (include/ultramem.h,
"the decoder block around the layer").

A cache is two tensors k_cache, v_cache [n_pages, kv_heads, page_size,
head_dim] (fp32 or bf16).  The requests' lengths, the block table and the free
list are int32 device tensors; no call waits for the GPU.  One step:

    q_start, kv_lens, slots, balance = paged_plan(ctx_lens, new_lens, block_table, free_pages,
                                                  free_count, page_size, n_tokens, free_left)
    paged_append(k_cache, v_cache, k, v, slots)            # in every block
    out = paged_attention(q, k_cache, v_cache, block_table, q_start, kv_lens, max_new)

A training step, whose requests are whole sequences, takes its gradient with
paged_attention_backward.

As in binding.py, these functions marshal arguments only; there is no
fallback, and an argument that the library cannot take raises.  They launch on
the current stream of the current device, where every tensor has to lie, and
autograd does not see them.
"""
from __future__ import annotations

import ctypes as C
import functools
import math

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.F32, torch.bfloat16: _b.BF16}


def _int32(name, t, dev):
    if t.dtype != torch.int32 or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor on the current device")
    return t.data_ptr()


def _cache(k_cache, v_cache):
    shape, dtype = k_cache.shape, k_cache.dtype
    if len(shape) != 4 or shape != v_cache.shape or dtype != v_cache.dtype:
        raise ValueError("k_cache and v_cache must be [n_pages, kv_heads, page_size, head_dim] "
                         "of one type")
    code = _DTYPES.get(dtype)
    dev = _b._on_device("k_cache", k_cache)
    if code is None or v_cache.get_device() != dev:
        raise ValueError("the cache must be fp32 or bf16 CUDA tensors on the current device")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("the cache must be contiguous")
    return _b.KVCache(k_cache.data_ptr(), v_cache.data_ptr(), *shape, code), shape, dtype, dev


def _rows(name, t, heads, dim, dtype, dev):
    """A [tokens, heads, dim] tensor whose tokens may be strided apart, and
    their distance."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != dim or (heads and shape[1] != heads) or \
            t.dtype != dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be a tensor [tokens, {heads or 'heads'}, {dim}] of the "
                         f"cache's type and device")
    s0, s1, s2 = t.stride()
    row = shape[1] * dim
    if s2 == 1 and s1 == dim and s0 >= row:
        return t, s0
    t = t.contiguous()
    return t, row


def paged_plan(ctx_lens, new_lens, block_table, free_pages, free_count, page_size: int,
               n_tokens: int, free_left=None):
    """Pages and slots for new_lens [R] new tokens after ctx_lens [R] cached
    ones: writes the new pages into block_table [R, width] and returns
    (q_start [R+1], kv_lens [R], slots [n_tokens], balance [1]), int32.
    New pages come from the end of free_pages[:free_count], whose length
    after the call goes to free_left [1] (the next call's free_count, another
    tensor than this call's).  A request that does not fit is refused (slots
    -1, kv_len 0).  balance is free_count less the pages that requests up to
    the last served one asked for, refused ones among them: it is neither the
    next free_count nor a count of what refused requests lack."""
    R = ctx_lens.numel()
    table_shape = block_table.shape
    if new_lens.numel() != R or len(table_shape) != 2 or table_shape[0] != R or \
            free_count.numel() != 1:
        raise ValueError("ctx_lens, new_lens and block_table must have a row for each request, "
                         "free_count one element")
    if n_tokens < 0:
        raise ValueError("n_tokens must not be negative")
    _b._fits_int32(n_tokens, R, table_shape[1], free_pages.numel(), page_size)
    dev = _b._on_device("ctx_lens", ctx_lens)
    free_ptr = None
    if free_left is not None:
        free_ptr = _int32("free_left", free_left, dev)
        if free_left.numel() != 1:
            raise ValueError("free_left must have one element")
    device = ctx_lens.device
    q_start = torch.empty(R + 1, dtype=torch.int32, device=device)
    kv_lens = torch.empty(R, dtype=torch.int32, device=device)
    slots = torch.empty(n_tokens, dtype=torch.int32, device=device)
    balance = torch.empty(1, dtype=torch.int32, device=device)
    lib = _b._lib or _b.load()
    status = lib.ultramem_paged_plan(
        _int32("ctx_lens", ctx_lens, dev), _int32("new_lens", new_lens, dev), R, page_size,
        _int32("block_table", block_table, dev), table_shape[1],
        _int32("free_pages", free_pages, dev), _int32("free_count", free_count, dev),
        free_pages.numel(), n_tokens, q_start.data_ptr(),
        kv_lens.data_ptr(), slots.data_ptr(), free_ptr, balance.data_ptr(), _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_paged_plan")
    return q_start, kv_lens, slots, balance


def paged_append(k_cache, v_cache, k, v, slots):
    """Writes k, v [tokens, kv_heads, head_dim] (tokens may be strided, as
    slices of one projection's output) into their slots [tokens]."""
    c, shape, dtype, dev = _cache(k_cache, v_cache)
    heads, dim = shape[1], shape[3]
    k, ks = _rows("k", k, heads, dim, dtype, dev)
    v, vs = _rows("v", v, heads, dim, dtype, dev)
    T = k.shape[0]
    if v.shape[0] != T or slots.numel() != T:
        raise ValueError("k, v and slots must have a row for each token")
    _b._fits_int32(T)
    lib = _b._lib or _b.load()
    status = lib.ultramem_paged_append(C.byref(c), k.data_ptr(), ks, v.data_ptr(), vs,
                                       _int32("slots", slots, dev), T, _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_paged_append")


@functools.lru_cache(maxsize=256)
def _workspace(dev, dtype, q_heads, kv_heads, head_dim, max_new):
    """Bytes of the attention's workspace, a function of the sizes and the
    (current) device alone."""
    return int(_b.load().ultramem_paged_attention_workspace(dtype, q_heads, kv_heads, head_dim,
                                                            max_new))


def paged_attention(q, k_cache, v_cache, block_table, q_start, kv_lens, max_new: int, scale=None,
                    out=None, with_lse=False):
    """Causal attention of q [tokens, q_heads, head_dim] (requests packed by
    q_start [R+1]) over the pages of block_table [R, width]: out like q, and
    the rows' log-sum-exp [tokens, q_heads] fp32 when ``with_lse``.  max_new:
    the most new tokens a request has (a host number, which chooses one kernel
    for the whole call); scale: default
    1 / sqrt(head_dim).  Rows that belong to no request (past q_start[R]) are
    not written.  ``out`` may be a contiguous q itself."""
    c, shape, dtype, dev = _cache(k_cache, v_cache)
    heads, dim = shape[1], shape[3]
    q, qs = _rows("q", q, 0, dim, dtype, dev)
    q_shape, device = q.shape, q.device
    T, H, _ = q_shape
    R = kv_lens.numel()
    table_shape = block_table.shape
    if q_start.numel() != R + 1 or len(table_shape) != 2 or table_shape[0] != R:
        raise ValueError("block_table and kv_lens must have a row for each request, q_start one "
                         "more")
    _b._fits_int32(T, R, table_shape[1], max_new)
    if out is None:
        out = torch.empty(q_shape, dtype=dtype, device=device)
    elif out.shape != q_shape or out.dtype != dtype or not out.is_contiguous() or \
            out.get_device() != dev:
        raise ValueError("out must be a contiguous tensor of q's shape, type and device")
    lse = torch.empty((T, H), dtype=torch.float32, device=device) if with_lse else None
    lib = _b._lib or _b.load()
    nbytes = _workspace(dev, c.dtype, H, heads, dim, max_new)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    status = lib.ultramem_paged_attention(
        C.byref(c), q.data_ptr(), qs, H, _int32("q_start", q_start, dev),
        _int32("kv_lens", kv_lens, dev), _int32("block_table", block_table, dev), table_shape[1], R,
        T, max_new,
        1.0 / math.sqrt(dim) if scale is None else scale, out.data_ptr(),
        None if lse is None else lse.data_ptr(), ws.data_ptr(), nbytes, _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_paged_attention")
    return (out, lse) if with_lse else out


@functools.lru_cache(maxsize=256)
def _grad_workspace(dev, dtype, T, R, q_heads, kv_heads, head_dim):
    """Bytes of the gradient's workspace, by the sizes and the (current)
    device alone."""
    return int(_b.load().ultramem_paged_attention_backward_workspace(dtype, T, R, q_heads,
                                                                     kv_heads, head_dim))


def _grad_rows(name, t, n, heads, dim, dtype, dev, device):
    """An output [tokens, heads, dim], new or given, whose tokens may be strided
    apart, and their distance."""
    shape, row = (n, heads, dim), heads * dim
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device), row
    s0, s1, s2 = t.stride() if t.dim() == 3 else (0, 0, 0)
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or s2 != 1 or \
            s1 != dim or (s0 < row and n > 1):
        raise ValueError(f"{name} must be a tensor {shape} of q's type and device, a token's "
                         "heads contiguous")
    return t, max(s0, row)


def paged_attention_backward(q, k, v, out, lse, dout, q_start, scale=None, dq=None, dk=None,
                             dv=None):
    """(dq, dk, dv) of the attention of whole sequences: requests without cached
    tokens, packed by q_start [R+1], at q [tokens, q_heads, head_dim], the k
    and v [tokens, kv_heads, head_dim] that were appended, and the out and lse
    that ``paged_attention`` gave for them, for the gradient dout of out.
    scale as there.  Tokens of all but lse may be strided apart, as slices of
    one projection's output; dq, dk and dv may be given, slices of one
    gradient among them.  Rows that belong to no sequence are not written.
    Tensors of bf16 that start or step off 16 bytes, and heads wider than 128,
    take the CUDA cores, many times slower where sequences are long."""
    dev = _b._on_device("q", q)
    if q.dim() != 3 or k.dim() != 3 or q.dtype not in _DTYPES:
        raise ValueError("q, k and v must be [tokens, heads, head_dim], fp32 or bf16")
    T, H, D = q.shape
    heads, dtype = k.shape[1], q.dtype
    R = q_start.numel() - 1
    if R < 0 or q_start.dim() != 1:
        raise ValueError("q_start must have an entry more than there are sequences")
    _b._fits_int32(T, R, k.shape[0])
    q, qs = _rows("q", q, H, D, dtype, dev)
    out, os = _rows("out", out, H, D, dtype, dev)
    dout, ds = _rows("dout", dout, H, D, dtype, dev)
    k, ks = _rows("k", k, heads, D, dtype, dev)
    v, vs = _rows("v", v, heads, D, dtype, dev)
    if not (out.shape[0] == dout.shape[0] == k.shape[0] == v.shape[0] == T):
        raise ValueError("q, k, v, out and dout must have a row for each token")
    if lse.shape != (T, H) or lse.dtype != torch.float32 or lse.get_device() != dev or \
            not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor [tokens, q_heads] on q's device")
    starts = _int32("q_start", q_start, dev)
    device = q.device
    dq, dqs = _grad_rows("dq", dq, T, H, D, dtype, dev, device)
    dk, dks = _grad_rows("dk", dk, T, heads, D, dtype, dev, device)
    dv, dvs = _grad_rows("dv", dv, T, heads, D, dtype, dev, device)
    code = _DTYPES[dtype]
    a = _b.AttentionGrad(
        q.data_ptr(), out.data_ptr(), dout.data_ptr(), k.data_ptr(), v.data_ptr(), dq.data_ptr(),
        dk.data_ptr(), dv.data_ptr(), lse.data_ptr(), starts, qs, os, ds, ks, vs, dqs, dks, dvs, T,
        R, H, heads, D, code, 1.0 / math.sqrt(D) if scale is None else scale)
    lib = _b._lib or _b.load()
    nbytes = _grad_workspace(dev, code, T, R, H, heads, D)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    status = lib.ultramem_paged_attention_backward(C.byref(a), ws.data_ptr(), nbytes,
                                                   _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_paged_attention_backward")
    return dq, dk, dv


def paged_check() -> int:
    """Syncs the current stream and returns the attention kernels' status on
    the current device since the last check, whatever stream they ran on."""
    return int(_b.load().ultramem_paged_check(_b._stream()))
