"""The norms after one block and before the next, fused with the block's gate
and the residual scale, and their gradient (include/ultramem.h,
ultramem_block_norm):

    z = N_post(y),  u = res_scale r + out_scale gate (.) z,  n = N_pre(u)

As in binding.py, these functions marshal arguments only.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.F32, torch.bfloat16: _b.BF16}
_KINDS = {"rms": 0, "layer": 1}
GATE_NONE, GATE_CHANNEL, GATE_TOKEN, GATE_FULL = 0, 1, 2, 3


def _rows(name, t, like):
    """A [T, D] tensor like ``like``; its rows may be strided apart."""
    if t.shape != like.shape or t.dtype != like.dtype or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor of y's shape {tuple(like.shape)} and type")
    s, d = t.stride(), t.shape[1]
    if s[1] != 1 or (s[0] < d and t.shape[0] > 1):
        t = t.contiguous()
    return t, max(t.stride(0), d)


def _vector(name, t, d):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != d or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 CUDA tensor of {d} entries")
    return t.data_ptr()


def _args(y, gate, w_post, b_post, w_pre, b_pre, kind, eps, res_scale, out_scale, post, pre):
    if y.dim() != 2 or y.dtype not in _DTYPES or not y.is_cuda:
        raise ValueError("y must be a CUDA tensor [tokens, dim], fp32 or bf16")
    if kind not in _KINDS:
        raise ValueError(f"kind must be one of {tuple(_KINDS)}")
    T, D = y.shape
    y, ld_y = _rows("y", y, y)
    mode = GATE_NONE
    if gate is not None:
        if not gate.is_cuda or not gate.is_contiguous():
            raise ValueError("gate must be a contiguous CUDA tensor")
        if gate.shape == (D,) and gate.dtype == torch.float32:
            mode = GATE_CHANNEL
        elif gate.shape == (T, D) and gate.dtype == y.dtype:
            mode = GATE_FULL
        elif gate.shape == (T, 1) and gate.dtype == y.dtype:
            mode = GATE_TOKEN
        else:
            raise ValueError("gate must be fp32 [dim], or [tokens, 1] or [tokens, dim] of y's "
                             "type")
    a = _b.BlockNormArgs(
        y.data_ptr(), None if gate is None else gate.data_ptr(), _vector("w_post", w_post, D),
        _vector("b_post", b_post, D), _vector("w_pre", w_pre, D), _vector("b_pre", b_pre, D),
        ld_y, 0, T, D, _DTYPES[y.dtype], _KINDS[kind], int(bool(post)), int(bool(pre)), mode,
        float(res_scale), float(out_scale), float(eps))
    return a, y, mode


def block_norm(y, residual, w_post=None, b_post=None, gate=None, w_pre=None, b_pre=None,
               kind="rms", eps=1e-5, res_scale=1.0, out_scale=1.0, post=True, pre=True, u=None,
               n=None):
    """(u, n) for a block's output y [T, D] and the residual stream before it
    (n is None without ``pre``).  gate: fp32 [D], or [T, 1] or [T, D] in y's
    type.  ``u`` and ``n`` may be given; u may be the residual itself and n
    may be y, updated in place."""
    lib = _b.load()
    a, y, _ = _args(y, gate, w_post, b_post, w_pre, b_pre, kind, eps, res_scale, out_scale, post,
                    pre)
    residual, a.ld_r = _rows("residual", residual, y)
    for name, t in (("u", u), ("n", n)):
        if t is not None and (t.shape != y.shape or t.dtype != y.dtype or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous, of y's shape and type")
    u = torch.empty(y.shape, dtype=y.dtype, device=y.device) if u is None else u
    if not pre:
        n = None
    elif n is None:
        n = torch.empty(y.shape, dtype=y.dtype, device=y.device)
    _b._check(lib.ultramem_block_norm(C.byref(a), residual.data_ptr(), u.data_ptr(),
                                      None if n is None else n.data_ptr(), _b._stream()),
              "ultramem_block_norm")
    return u, n


def block_norm_backward(y, u, du, dn=None, w_post=None, b_post=None, gate=None, w_pre=None,
                        b_pre=None, kind="rms", eps=1e-5, res_scale=1.0, out_scale=1.0, post=True,
                        pre=True):
    """The gradient of ``block_norm`` at its y and stored u, for the gradients
    du of u (may be None) and dn of n (with ``pre``): a dict of dy, dr,
    dw_post, db_post, dw_pre, db_pre, dgate (None where the forward has no such
    input; gains and biases are fp32, and absent gains get no gradient)."""
    lib = _b.load()
    a, y, mode = _args(y, gate, w_post, b_post, w_pre, b_pre, kind, eps, res_scale, out_scale,
                       post, pre)
    T, D = y.shape
    u, a.ld_r = _rows("u", u, y)
    ld_du = ld_dn = 0
    if du is not None:
        du, ld_du = _rows("du", du, y)
    if dn is not None:
        dn, ld_dn = _rows("dn", dn, y)
    rows = torch.empty((2, T, D), dtype=y.dtype, device=y.device)
    got = {"dy": rows[0], "dr": rows[1]}
    want = [("dw_post", post and w_post is not None), ("db_post", post and b_post is not None),
            ("dw_pre", pre and w_pre is not None), ("db_pre", pre and b_pre is not None)]
    nbytes = int(lib.ultramem_block_norm_backward_workspace(T, D))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=y.device)
    for name, on in want:
        got[name] = torch.empty(D, dtype=torch.float32, device=y.device) if on else None
    got["dgate"] = None if gate is None else torch.empty_like(gate)
    ptr = {k: None if v is None else v.data_ptr() for k, v in got.items()}
    _b._check(lib.ultramem_block_norm_backward(
        C.byref(a), u.data_ptr(), None if du is None else du.data_ptr(), ld_du,
        None if dn is None else dn.data_ptr(), ld_dn, ptr["dy"], ptr["dr"], ptr["dgate"],
        ptr["dw_post"], ptr["db_post"], ptr["dw_pre"], ptr["db_pre"], ws.data_ptr(), nbytes,
        _b._stream()), "ultramem_block_norm_backward")
    return got
