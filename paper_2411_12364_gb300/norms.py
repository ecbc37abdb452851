"""The norms after one block and before the next, fused with the block's gate
and the residual scale, and their gradient (include/ultramem.h,
ultramem_block_norm):

    z = N_post(y),  u = res_scale r + out_scale gate (.) z,  n = N_pre(u)

As in binding.py, these functions marshal arguments only.  They launch on the
current stream of the current device, where every tensor has to lie.  Autograd
does not see them: their outputs require no gradient, whatever the inputs do;
a training step calls block_norm_backward.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.F32, torch.bfloat16: _b.BF16}
_KINDS = {"rms": 0, "layer": 1}
GATE_NONE, GATE_CHANNEL, GATE_TOKEN, GATE_FULL = 0, 1, 2, 3


def _rows(name, t, shape, dtype, dev):
    """A [T, D] tensor; its rows may be strided apart.  Returns it and the
    distance of its rows."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be a tensor of y's shape {tuple(shape)}, type and device")
    s0, s1 = t.stride()
    d = shape[1]
    if s1 == 1 and s0 >= d:
        return t, s0
    if (s1 == 1 or d == 1) and shape[0] == 1:
        return t, d
    return t.contiguous(), d


def _vector(name, t, d, dev):
    if t.dtype != torch.float32 or t.numel() != d or t.get_device() != dev or \
            not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor of {d} entries on y's device")
    return t.data_ptr()


def _args(y, gate, w_post, b_post, w_pre, b_pre, kind, eps, res_scale, out_scale, post, pre):
    shape, dtype = y.shape, y.dtype
    code, kind_code = _DTYPES.get(dtype), _KINDS.get(kind)
    if len(shape) != 2 or code is None:
        raise ValueError("y must be a CUDA tensor [tokens, dim], fp32 or bf16")
    if kind_code is None:
        raise ValueError(f"kind must be one of {tuple(_KINDS)}")
    dev = _b._on_device("y", y)
    _b._fits_int32(*shape)
    y, ld_y = _rows("y", y, shape, dtype, dev)
    T, D = shape
    mode, gate_ptr = GATE_NONE, None
    if gate is not None:
        if gate.get_device() != dev or not gate.is_contiguous():
            raise ValueError("gate must be a contiguous tensor on y's device")
        gate_shape = gate.shape
        if gate_shape == (D,) and gate.dtype == torch.float32:
            mode = GATE_CHANNEL
        elif gate_shape == shape and gate.dtype == dtype:
            mode = GATE_FULL
        elif gate_shape == (T, 1) and gate.dtype == dtype:
            mode = GATE_TOKEN
        else:
            raise ValueError("gate must be fp32 [dim], or [tokens, 1] or [tokens, dim] of y's "
                             "type")
        gate_ptr = gate.data_ptr()
    a = _b.BlockNormArgs(
        y.data_ptr(), gate_ptr, None if w_post is None else _vector("w_post", w_post, D, dev),
        None if b_post is None else _vector("b_post", b_post, D, dev),
        None if w_pre is None else _vector("w_pre", w_pre, D, dev),
        None if b_pre is None else _vector("b_pre", b_pre, D, dev), ld_y, 0, T, D, code, kind_code,
        1 if post else 0, 1 if pre else 0, mode, res_scale, out_scale, eps)
    return a, y, dev


@functools.lru_cache(maxsize=256)
def _workspace(dev, T, D):
    """Bytes of the backward's workspace, a function of the sizes and the
    (current) device alone."""
    return int(_b.load().ultramem_block_norm_backward_workspace(T, D))


def _given(name, t, y, dev):
    if t.shape != y.shape or t.dtype != y.dtype or not t.is_contiguous() or \
            t.get_device() != dev:
        raise ValueError(f"{name} must be contiguous, of y's shape, type and device")
    return t


def block_norm(y, residual, w_post=None, b_post=None, gate=None, w_pre=None, b_pre=None,
               kind="rms", eps=1e-5, res_scale=1.0, out_scale=1.0, post=True, pre=True, u=None,
               n=None):
    """(u, n) for a block's output y [T, D] and the residual stream before it
    (n is None without ``pre``).  gate: fp32 [D], or [T, 1] or [T, D] in y's
    type.  ``u`` and ``n`` may be given; u may be the residual itself and n
    may be y, updated in place (or the other way round), but they must not
    overlap each other."""
    a, y, dev = _args(y, gate, w_post, b_post, w_pre, b_pre, kind, eps, res_scale, out_scale, post,
                      pre)
    shape, dtype = y.shape, y.dtype
    residual, a.ld_r = _rows("residual", residual, shape, dtype, dev)
    u = torch.empty(shape, dtype=dtype, device=y.device) if u is None else _given("u", u, y, dev)
    if not pre:
        n = None
    elif n is None:
        n = torch.empty(shape, dtype=dtype, device=y.device)
    else:
        n = _given("n", n, y, dev)
    lib = _b._lib or _b.load()
    status = lib.ultramem_block_norm(C.byref(a), residual.data_ptr(), u.data_ptr(),
                                     None if n is None else n.data_ptr(), _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_block_norm")
    return u, n


def block_norm_backward(y, u, du, dn=None, w_post=None, b_post=None, gate=None, w_pre=None,
                        b_pre=None, kind="rms", eps=1e-5, res_scale=1.0, out_scale=1.0, post=True,
                        pre=True):
    """The gradient of ``block_norm`` at its y and stored u, for the gradients
    du of u (may be None) and dn of n (with ``pre``): a dict of dy, dr,
    dw_post, db_post, dw_pre, db_pre, dgate (None where the forward has no such
    input; gains and biases are fp32, and absent gains get no gradient)."""
    a, y, dev = _args(y, gate, w_post, b_post, w_pre, b_pre, kind, eps, res_scale, out_scale, post,
                      pre)
    shape, dtype, device = y.shape, y.dtype, y.device
    T, D = shape
    u, a.ld_r = _rows("u", u, shape, dtype, dev)
    du_ptr = dn_ptr = None
    ld_du = ld_dn = 0
    if du is not None:
        du, ld_du = _rows("du", du, shape, dtype, dev)
        du_ptr = du.data_ptr()
    if dn is not None:
        dn, ld_dn = _rows("dn", dn, shape, dtype, dev)
        dn_ptr = dn.data_ptr()
    lib = _b._lib or _b.load()
    dy = torch.empty(shape, dtype=dtype, device=device)
    dr = torch.empty(shape, dtype=dtype, device=device)
    dw_post = db_post = dw_pre = db_pre = dgate = None
    p_wpost = p_bpost = p_wpre = p_bpre = p_gate = None
    if post and w_post is not None:
        dw_post = torch.empty(D, dtype=torch.float32, device=device)
        p_wpost = dw_post.data_ptr()
    if post and b_post is not None:
        db_post = torch.empty(D, dtype=torch.float32, device=device)
        p_bpost = db_post.data_ptr()
    if pre and w_pre is not None:
        dw_pre = torch.empty(D, dtype=torch.float32, device=device)
        p_wpre = dw_pre.data_ptr()
    if pre and b_pre is not None:
        db_pre = torch.empty(D, dtype=torch.float32, device=device)
        p_bpre = db_pre.data_ptr()
    if gate is not None:
        dgate = torch.empty_like(gate)
        p_gate = dgate.data_ptr()
    nbytes = _workspace(dev, T, D)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    status = lib.ultramem_block_norm_backward(
        C.byref(a), u.data_ptr(), du_ptr, ld_du, dn_ptr, ld_dn, dy.data_ptr(), dr.data_ptr(),
        p_gate, p_wpost, p_bpost, p_wpre, p_bpre, ws.data_ptr(), nbytes, _b._stream(dev))
    if status:
        raise _b.UltraMemError(status, "ultramem_block_norm_backward")
    return {"dy": dy, "dr": dr, "dw_post": dw_post, "db_post": db_post, "dw_pre": dw_pre,
            "db_pre": db_pre, "dgate": dgate}
