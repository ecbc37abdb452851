"""Losses of tokens whose label holds nearly all the probability: never below 0,
and with the digits that a sum near 1 has."""
import pytest
import torch

from paper_2411_12364_gb300 import vocab
from tests.test_cross_entropy_gpu import check_forward, z_error

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,D", [(300, 1000, 64), (70, 33, 100), (260, 900, 2112)])
@pytest.mark.parametrize("logit", [8.0, 60.0, 300.0])
@pytest.mark.parametrize("s", [1.0, 0.37, -1.0])
def test_sure_labels(gpu_lib, dtype, T, V, D, logit, s):
    g = torch.Generator(device="cuda").manual_seed(T + V + D)
    w = torch.nn.functional.normalize(torch.randn(V, D, generator=g, device="cuda"), dim=1)
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    x = (w[labels] * (logit / s)).to(dtype)          # the label's logit, by the rows' unit length
    w = w.to(dtype)
    loss, lse = vocab.cross_entropy(x, w, labels, logit_scale=s)
    check_forward(x, w, labels, s, (loss, lse))
    assert float(loss.min()) >= 0.0
    z = (x.double() @ w.double().T) * s
    z -= z.gather(1, labels[:, None])
    others = torch.exp(z).sum(1) - 1.0
    want = torch.log1p(others)
    sure = z.amax(1) <= 0                            # the label's is the largest logit
    assert int(sure.sum()) > T // 2
    # The largest term is 1 and takes part in at most 8 additions of a chunk's pairs
    # and 2 of their sums, 4 of chunks, 1 of a warp's tiles in the join (V < 32
    # tiles), 5 between warps, and the logarithm adds 2 roundings: below 32
    # roundings of 2^-24 of a value below 2; each of the others is off by its logit's
    # error and the label's, and by that of e^ (2^-20).
    err = 2 * z_error(x, w, s).amax(1) + 2.0 ** -20
    tol = 64 * 2.0 ** -24 + others * torch.expm1(err)
    assert bool(((loss.double() - want).abs() <= tol)[sure].all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("s", [1.0, 0.3, -2.7, 0.0])
def test_a_vocabulary_of_one(gpu_lib, dtype, s):
    """The only logit is the largest and the label's: the loss is 0, and lse the logit."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(200, 72, generator=g, device="cuda").to(dtype)
    w = torch.randn(1, 72, generator=g, device="cuda").to(dtype)
    labels = torch.zeros(200, dtype=torch.int64, device="cuda")
    loss, lse = vocab.cross_entropy(x, w, labels, logit_scale=s)
    assert not bool(loss.any())
    check_forward(x, w, labels, s, (loss, lse))
