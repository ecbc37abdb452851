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

As in binding.py, these functions marshal arguments only; there is no
fallback, and an argument that the library cannot take raises.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.F32, torch.bfloat16: _b.BF16}


def _device_int32(name, t):
    if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
    return t


def _cache(k_cache, v_cache):
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype:
        raise ValueError("k_cache and v_cache must be [n_pages, kv_heads, page_size, head_dim] "
                         "of one type")
    if k_cache.dtype not in _DTYPES or not (k_cache.is_cuda and v_cache.is_cuda):
        raise ValueError("the cache must be fp32 or bf16 CUDA tensors")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("the cache must be contiguous")
    n, h, p, d = k_cache.shape
    return _b.KVCache(k_cache.data_ptr(), v_cache.data_ptr(), n, h, p, d, _DTYPES[k_cache.dtype])


def _rows(name, t, heads, dim, dtype):
    """A [tokens, heads, dim] tensor whose tokens may be strided apart."""
    if t.dim() != 3 or t.shape[2] != dim or (heads and t.shape[1] != heads) or \
            t.dtype != dtype or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor [tokens, {heads or 'heads'}, {dim}] "
                         f"of the cache's type")
    s = t.stride()
    if t.numel() and (s[2] != 1 or s[1] != dim or (s[0] < t.shape[1] * dim and t.shape[0] > 1)):
        t = t.contiguous()
    return t, max(t.stride(0), t.shape[1] * dim)


def paged_plan(ctx_lens, new_lens, block_table, free_pages, free_count, page_size: int,
               n_tokens: int, free_left=None):
    """Pages and slots for new_lens [R] new tokens after ctx_lens [R] cached
    ones: writes the new pages into block_table [R, width] and returns
    (q_start [R+1], kv_lens [R], slots [n_tokens], balance [1]), int32.
    New pages come from the end of free_pages[:free_count], whose length
    after the call goes to free_left [1] (the next call's free_count, another
    tensor than this call's).  A request that does not fit is refused (slots
    -1, kv_len 0); balance is free_count less the pages asked for up to the
    last request served, so below zero what the step was short of."""
    lib = _b.load()
    R = ctx_lens.numel()
    if new_lens.numel() != R or block_table.dim() != 2 or block_table.shape[0] != R or \
            free_count.numel() != 1:
        raise ValueError("ctx_lens, new_lens and block_table must have a row for each request, "
                         "free_count one element")
    for name, t in (("ctx_lens", ctx_lens), ("new_lens", new_lens), ("block_table", block_table),
                    ("free_pages", free_pages), ("free_count", free_count)):
        _device_int32(name, t)
    n_tokens = int(n_tokens)
    if n_tokens < 0:
        raise ValueError("n_tokens must not be negative")
    if free_left is not None and _device_int32("free_left", free_left).numel() != 1:
        raise ValueError("free_left must have one element")
    # one allocation for the outputs, each on a 16-byte boundary
    at = [0, (R + 4) & ~3]
    at.append(at[1] + ((R + 3) & ~3))
    at.append(at[2] + ((n_tokens + 3) & ~3))
    buf = torch.empty(at[3] + 2, dtype=torch.int32, device=ctx_lens.device)
    q_start, kv_lens = buf[:R + 1], buf[at[1]:at[1] + R]
    slots, balance = buf[at[2]:at[2] + n_tokens], buf[at[3]:at[3] + 1]
    base = buf.data_ptr()
    _b._check(lib.ultramem_paged_plan(
        ctx_lens.data_ptr(), new_lens.data_ptr(), R, int(page_size), block_table.data_ptr(),
        block_table.shape[1], free_pages.data_ptr(), free_count.data_ptr(), n_tokens, base,
        base + 4 * at[1], base + 4 * at[2],
        base + 4 * at[3] + 4 if free_left is None else free_left.data_ptr(), base + 4 * at[3],
        _b._stream()), "ultramem_paged_plan")
    return q_start, kv_lens, slots, balance


def paged_append(k_cache, v_cache, k, v, slots):
    """Writes k, v [tokens, kv_heads, head_dim] (tokens may be strided, as
    slices of one projection's output) into their slots [tokens]."""
    lib = _b.load()
    c = _cache(k_cache, v_cache)
    k, ks = _rows("k", k, c.kv_heads, c.head_dim, k_cache.dtype)
    v, vs = _rows("v", v, c.kv_heads, c.head_dim, k_cache.dtype)
    T = k.shape[0]
    if v.shape[0] != T or slots.numel() != T:
        raise ValueError("k, v and slots must have a row for each token")
    _device_int32("slots", slots)
    _b._check(lib.ultramem_paged_append(C.byref(c), k.data_ptr(), ks, v.data_ptr(), vs,
                                        slots.data_ptr(), T, _b._stream()),
              "ultramem_paged_append")


def paged_attention(q, k_cache, v_cache, block_table, q_start, kv_lens, max_new: int, scale=None,
                    out=None, with_lse=False):
    """Causal attention of q [tokens, q_heads, head_dim] (requests packed by
    q_start [R+1]) over the pages of block_table [R, width]: out like q, and
    the rows' log-sum-exp [tokens, q_heads] fp32 when ``with_lse``.  max_new:
    the most new tokens a request has (a host number); scale: default
    1 / sqrt(head_dim)."""
    lib = _b.load()
    c = _cache(k_cache, v_cache)
    q, qs = _rows("q", q, 0, c.head_dim, k_cache.dtype)
    T, H, D = q.shape
    R = kv_lens.numel()
    if q_start.numel() != R + 1 or block_table.dim() != 2 or block_table.shape[0] != R:
        raise ValueError("block_table and kv_lens must have a row for each request, q_start one "
                         "more")
    for name, t in (("block_table", block_table), ("q_start", q_start), ("kv_lens", kv_lens)):
        _device_int32(name, t)
    if out is None:
        out = torch.empty((T, H, D), dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise ValueError("out must be contiguous, of q's shape and type")
    lse = torch.empty((T, H), dtype=torch.float32, device=q.device) if with_lse else None
    max_new = int(max_new)
    nbytes = lib.ultramem_paged_attention_workspace(c.dtype, H, c.kv_heads, D, max_new)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    _b._check(lib.ultramem_paged_attention(
        C.byref(c), q.data_ptr(), qs, H, q_start.data_ptr(), kv_lens.data_ptr(),
        block_table.data_ptr(), block_table.shape[1], R, T, max_new,
        1.0 / math.sqrt(D) if scale is None else float(scale), out.data_ptr(),
        None if lse is None else lse.data_ptr(), ws.data_ptr(), nbytes, _b._stream()),
        "ultramem_paged_attention")
    return (out, lse) if with_lse else out


def paged_check() -> int:
    """Syncs the current stream and returns the attention kernels' status."""
    return int(_b.load().ultramem_paged_check(_b._stream()))
