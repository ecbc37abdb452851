"""The block norms with outputs in the place of inputs give the bits of the
same call with outputs of their own."""
import ctypes as C

import pytest
import torch

from paper_2411_12364_gb300 import binding
from paper_2411_12364_gb300.norms import block_norm, block_norm_backward

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def make(T, D, dtype, gate):
    gen = torch.Generator(device="cuda").manual_seed(T + D)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    p = {k: randn(T, D).to(dtype) for k in ("y", "u", "du", "dn")}
    p.update({k: randn(D) for k in ("w_post", "b_post", "w_pre", "b_pre")})
    p["gate"] = {"channel": lambda: randn(D), "token": lambda: randn(T, 1).to(dtype),
                 "full": lambda: randn(T, D).to(dtype)}[gate]()
    return p


@pytest.mark.parametrize("dtype,D", [(BF16, 256), (BF16, 333), (BF16, 2048), (F32, 1000),
                                     (BF16, 8192)])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (False, False)])
def test_forward_in_any_row_tensors_place(dtype, D, post, pre, gpu_lib):
    p = make(700, D, dtype, "full")
    w = {k: p[k] for k in ("w_post", "b_post", "w_pre", "b_pre")}

    def call(u=None, n=None):
        t = {k: p[k].clone() for k in ("y", "u", "gate")}
        return block_norm(t["y"], t["u"], gate=t["gate"], kind="layer", post=post, pre=pre,
                          u=u and t[u], n=n and t[n], **w)

    want = call()
    for u, n in (("u", "y"), ("y", "u"), ("gate", "y"), ("y", "gate"), ("u", "gate")):
        got = call(u, n if pre else None)
        assert torch.equal(got[0], want[0])
        assert not pre or torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype,D", [(BF16, 256), (BF16, 333), (F32, 2048), (BF16, 8192)])
@pytest.mark.parametrize("gate", ["channel", "token", "full"])
def test_gradient_in_its_inputs_place(dtype, D, gate, gpu_lib):
    T = 700
    p = make(T, D, dtype, gate)
    want = block_norm_backward(kind="layer", **p)
    mode = {"channel": 1, "token": 2, "full": 3}[gate]
    for dy, dr in (("du", "dn"), ("dn", "y"), ("y", "u")):
        t = {k: v.clone() for k, v in p.items()}
        a = binding.BlockNormArgs(
            t["y"].data_ptr(), t["gate"].data_ptr(), t["w_post"].data_ptr(),
            t["b_post"].data_ptr(), t["w_pre"].data_ptr(), t["b_pre"].data_ptr(), D, D, T, D,
            binding.BF16 if dtype == BF16 else binding.F32, 1, 1, 1, mode, 1.0, 1.0, 1e-5)
        need = gpu_lib.ultramem_block_norm_backward_workspace(T, D)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        st = gpu_lib.ultramem_block_norm_backward(
            C.byref(a), t["u"].data_ptr(), t["du"].data_ptr(), D, t["dn"].data_ptr(), D,
            t[dy].data_ptr(), t[dr].data_ptr(), t["gate"].data_ptr(), t["w_post"].data_ptr(),
            t["b_post"].data_ptr(), t["w_pre"].data_ptr(), t["b_pre"].data_ptr(), ws.data_ptr(),
            need, torch.cuda.current_stream().cuda_stream)
        assert st == binding.OK
        got = dict(dy=t[dy], dr=t[dr], dgate=t["gate"], dw_post=t["w_post"], db_post=t["b_post"],
                   dw_pre=t["w_pre"], db_pre=t["b_pre"])
        for name, x in got.items():
            assert torch.equal(x, want[name]), (name, dy, dr)


def test_overlapping_outputs_are_refused(gpu_lib):
    x = torch.randn(8, 64, device="cuda")
    both = torch.empty(8, 64, device="cuda")
    for kw in (dict(u=both, n=both), dict(u=x, n=x)):
        with pytest.raises(binding.UltraMemError) as e:
            block_norm(x, x.clone(), **kw)
        assert e.value.status == binding.EINVAL
