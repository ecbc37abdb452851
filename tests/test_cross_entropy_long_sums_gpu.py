"""Gradients of the cross entropy whose sums run over more than 65536 terms of one
sign, where the truncation of the tensor cores' sums adds up."""
import math

import pytest
import torch

from paper_2411_12364_gb300 import vocab

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
# half a step of bf16 for the result, and what 65536 terms lose (2^-23 of the sum
# every 16) before they are joined; the joins' own roundings are 2^-24 each
TOL = 2.0 ** -8 + 2.0 ** -11 + 64 * 2.0 ** -24


def positive(rows, columns, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (1 + torch.rand(rows, columns, generator=g, device="cuda")).to(BF16)


def weights_of_2_to_minus_16(T):
    """lse and dloss that make every G but the labels' 2^-16 where all logits are 0."""
    return (torch.full((T,), 16 * math.log(2), device="cuda"), torch.ones(T, device="cuda"),
            torch.zeros(T, dtype=torch.int64, device="cuda"))


@pytest.mark.parametrize("T,V,D", [(2304, 110000, 2048), (100, 200000, 72)])
def test_over_the_vocabulary(gpu_lib, T, V, D):
    w = positive(V, D, 1)
    w[0] = 0                             # the labels' row
    lse, dloss, labels = weights_of_2_to_minus_16(T)
    x = torch.zeros(T, D, dtype=BF16, device="cuda")
    dx, _ = vocab.cross_entropy_backward(x, w, labels, lse, dloss, dw=False)
    want = w.double().sum(0) * 2.0 ** -16
    assert bool(((dx.double() - want).abs() <= TOL * want).all())


@pytest.mark.parametrize("T,V,D", [(140000, 1280, 2560), (300000, 33, 72)])
def test_over_the_tokens(gpu_lib, T, V, D):
    x = positive(T, D, 2)
    lse, dloss, labels = weights_of_2_to_minus_16(T)
    w = torch.zeros(V, D, dtype=BF16, device="cuda")
    _, dw = vocab.cross_entropy_backward(x, w, labels, lse, dloss, dx=False)
    want = x.double().sum(0) * 2.0 ** -16
    assert bool(((dw[1:].double() - want).abs() <= TOL * want).all())
