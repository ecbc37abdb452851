"""Logits of plus and minus infinity: lse and loss as their definitions give them."""
import pytest
import torch

from paper_2411_12364_gb300 import vocab

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("D", [64, 100, 4096])
@pytest.mark.parametrize("V", [1, 40, 700])
@pytest.mark.parametrize("s", [1.0, -0.5])
def test_infinite_logits(gpu_lib, D, V, s):
    T = 140
    g = torch.Generator(device="cuda").manual_seed(D + V)
    x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    w = (torch.randn(V, D, generator=g, device="cuda") / D ** 0.5).bfloat16()
    x[:, 5] = torch.where(torch.arange(T, device="cuda") % 3 == 0, 1.0, -1.0)
    w[V // 2, 5] = INF                   # a logit of either sign for every token
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    labels[:6] = V // 2
    loss, lse = vocab.cross_entropy(x, w, labels, logit_scale=s)
    z = (x.double() @ w.double().T) * s
    want = torch.logsumexp(z, 1)
    assert int(torch.isinf(want).sum()) >= T // 3
    # an infinity is one exactly; finite values as in the other tests, loosely
    inf = torch.isinf(want)
    assert torch.equal(lse[inf].double(), want[inf])
    assert bool(((lse - want).abs() <= 1e-4)[~inf].all())
    pick = want - z.gather(1, labels[:, None])[:, 0]
    assert torch.equal(torch.isnan(loss), torch.isnan(pick))
    assert torch.equal(loss == INF, pick == INF)
    ok = torch.isfinite(pick)
    assert bool(((loss - pick).abs() <= 1e-4)[ok].all())
