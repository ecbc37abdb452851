"""The cross entropy of rows of more than 2048 entries, whose sums are cut in the
tensor cores, against 64 bits in both directions."""
import pytest
import torch

from paper_2411_12364_gb300 import paged, vocab
from tests.test_cross_entropy_gpu import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,D", [(300, 1003, 4096), (270, 515, 2049), (513, 777, 2112),
                                   (5, 3001, 4096), (2300, 301, 2500), (260, 40, 8200),
                                   (1, 1, 2049), (129, 257, 16384)])
def test_wide_rows(gpu_lib, dtype, T, V, D):
    x, w, labels, dloss = inputs(T, V, D, dtype)
    for s in (1.0, -0.37):
        got = vocab.cross_entropy(x, w, labels, logit_scale=s)
        check_forward(x, w, labels, s, got)
        again = vocab.cross_entropy(x, w, labels, logit_scale=s)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        grads = vocab.cross_entropy_backward(x, w, labels, got[1], dloss, logit_scale=s)
        check_backward(x, w, labels, got[1], dloss, s, grads)
    assert paged.paged_check() == 0


@pytest.mark.parametrize("D", [4096, 4099])
def test_wide_rows_are_as_exact_as_narrow_ones(gpu_lib, D):
    """lse to 1e-6 of its size, where sums truncated all along lose 1.4e-6."""
    x, w, labels, _ = inputs(700, 5003, D, BF16)
    _, lse = vocab.cross_entropy(x, w, labels)
    want = torch.logsumexp(x.double() @ w.double().T, 1)
    assert float((lse.double() - want).norm() / want.norm()) <= 1e-6
