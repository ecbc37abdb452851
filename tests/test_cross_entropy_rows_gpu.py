"""What lies beside the rows of the cross entropy's operands stays out of its
copies of them."""
import ctypes as C

import pytest
import torch

from paper_2411_12364_gb300 import binding as b
from paper_2411_12364_gb300 import vocab
from tests.test_cross_entropy_gpu import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [8, 40, 56, 64, 72, 200])
def test_copies_end_with_their_rows(gpu_lib, dtype, D):
    """The gradient's copy of x stands first in its workspace: zeros behind each
    row, where the memory beside the rows holds NaN."""
    T, V, ld = 20, 33, 256
    g = torch.Generator(device="cuda").manual_seed(D)
    x = torch.full((T + 1, ld), float("nan"), dtype=dtype, device="cuda")
    w = torch.full((V + 1, ld), float("nan"), dtype=dtype, device="cuda")
    x[:T, :D] = torch.randn(T, D, generator=g, device="cuda").to(dtype)
    w[:V, :D] = torch.randn(V, D, generator=g, device="cuda").to(dtype)
    labels = torch.arange(T, device="cuda")
    lse, dloss = torch.full((T,), 5.0, device="cuda"), torch.ones(T, device="cuda")
    dx, dw = (torch.empty(n, D, dtype=dtype, device="cuda") for n in (T, V))
    code = b.BF16 if dtype == BF16 else b.F32
    need = gpu_lib.ultramem_cross_entropy_backward_workspace(code, T, V, D)
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device="cuda")
    ws = ws[-ws.data_ptr() % 256:]
    a = b.CrossEntropyArgs(x.data_ptr(), w.data_ptr(), labels.data_ptr(), ld, ld, T, V, D, code, 8,
                           1.0)
    assert gpu_lib.ultramem_cross_entropy_backward(
        C.byref(a), lse.data_ptr(), dloss.data_ptr(), dx.data_ptr(), dw.data_ptr(), ws.data_ptr(),
        need, b._stream(x.get_device())) == b.OK
    planes, width = (1 if dtype == BF16 else 3), -(-D // 64) * 64
    copy = ws[:planes * T * width * 2].view(BF16).view(planes, T, width)
    assert torch.equal(copy.double().sum(0)[:, :D], x[:T, :D].double())
    assert not bool(copy[:, :, D:].any())
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())


@pytest.mark.parametrize("T,V", [(4095, 4200), (4100, 4200), (4200, 4095)])
@pytest.mark.parametrize("D", [72, 128])
def test_rows_where_they_lie_and_copied(gpu_lib, T, V, D):
    """bf16 rows off 128 bytes: read where they lie, or copied where both sides are long."""
    x, w, labels, dloss = inputs(T, V, D, BF16)
    loss, lse = vocab.cross_entropy(x, w, labels)
    check_forward(x, w, labels, 1.0, (loss, lse))
    grads = vocab.cross_entropy_backward(x, w, labels, lse, dloss)
    check_backward(x, w, labels, lse, dloss, 1.0, grads)
    only = vocab.cross_entropy_backward(x, w, labels, lse, dloss, dw=False)
    assert torch.equal(only[0], grads[0])
