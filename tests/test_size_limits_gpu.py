"""Calls at the ends of the 32-bit sizes: as many slots as an int counts, and
requests of as many keys (one page, named by every entry of the table)."""
import math

import pytest
import torch

from paper_2411_12364_gb300.paged import paged_attention, paged_check, paged_plan

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_plan_with_as_many_slots_as_an_int_counts(gpu_lib):
    n = 2 ** 31 - 1
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    q_start, kv, slots, _ = paged_plan(i32([3, 0]), i32([20, 7]), table, i32([5, 6, 7, 8]), i32([4]),
                                       16, n)
    assert q_start.tolist() == [0, 20, 27] and kv.tolist() == [23, 7]
    assert (slots[:27] >= -1).all() and slots[20].item() == 7 * 16
    for a in range(27, n, 2 ** 28):
        assert (slots[a:a + 2 ** 28] == -1).all()


@pytest.mark.parametrize("dtype,n,dim", [(BF16, 1, 64), (BF16, 40, 64), (F32, 1, 64)])
def test_requests_of_as_many_keys_as_an_int_counts(dtype, n, dim, gpu_lib):
    page = 256
    k = torch.zeros(2, 1, page, dim, dtype=dtype, device="cuda")
    v = torch.ones_like(k)
    table = torch.zeros(1, 2 ** 23 + 8, dtype=torch.int32, device="cuda")
    q = torch.randn(n, 1, dim, device="cuda").to(dtype)
    out, lse = paged_attention(q, k, v, table, i32([0, n]), i32([2 ** 31 - 1]), n, with_lse=True)
    # all scores are 0: the mean of ones, and the logarithm of the keys' number.
    # A share's sums of ones are exact below 2^24; joining at most 480 of them
    # rounds at most 100 times in a row, 2^-24 each, and the logarithm near 21
    # three times, 2^-19 each
    assert (out.float() - 1).abs().max().item() <= 2.0 ** -8
    assert (lse - math.log(2 ** 31 - 1024)).abs().max().item() <= 100 * 2.0 ** -24 + 3 * 2.0 ** -19
    assert paged_check() == 0
