"""Scores of -inf weigh nothing, and a row that has no other score is treated
like a row without keys, in each of the attention's kernels and across split
tiles."""
import math

import pytest
import torch

from paper_2411_12364_gb300.paged import paged_attention

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,dim", [(BF16, 64), (BF16, 128), (BF16, 192), (F32, 64)])
@pytest.mark.parametrize("n", [1, 60])
@pytest.mark.parametrize("kv", [70, 6000])
def test_scores_of_minus_infinity(dtype, dim, n, kv, gpu_lib):
    gen = torch.Generator(device="cuda").manual_seed(kv + dim)
    page, hk, hq = 16, 1, 4
    pages = -(-kv // page)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    # the first column alone makes the scores: 0 or -inf, by key
    for lowest in ("all", "some"):
        k = torch.zeros(pages, hk, page, dim, device="cuda", dtype=dtype)
        gone = torch.ones(pages * page, dtype=torch.bool, device="cuda")
        if lowest == "some":
            gone = torch.rand(pages * page, generator=gen, device="cuda") < 0.5
            gone[0] = False                   # every row sees key 0
        k[..., 0] = torch.where(gone, -math.inf, 0.0).view(pages, 1, page).to(dtype)
        v = torch.randn(pages, hk, page, dim, generator=gen, device="cuda").to(dtype)
        q = torch.zeros(n, hq, dim, device="cuda", dtype=dtype)
        q[..., 0] = 1.0
        out, lse = paged_attention(q, k, v, torch.arange(pages, dtype=torch.int32,
                                                         device="cuda").view(1, -1),
                                   ints([0, n]), ints([kv]), n, with_lse=True)
        if lowest == "all":
            assert (out == 0).all() and (lse == -math.inf).all()
            continue
        # equal weights of the keys that are left
        left = (~gone).double()
        flat = v.transpose(1, 2).reshape(-1, dim).double() * left[:, None]
        size = flat.abs()
        for i in range(n):
            sees = kv - n + i + 1
            count = left[:sees].sum()
            want, a = flat[:sees].sum(0) / count, size[:sees].sum(0) / count
            # fp32 sums, and at most two roundings to bf16
            tol = (2 * 2.0 ** -8 if dtype == BF16 else 0.0) * a + (kv + 16) * 2.0 ** -24 * a + 1e-30
            assert ((out[i].double() - want).abs() <= tol).all(), i
            assert ((lse[i].double() - count.log()).abs() <= 2.0 ** -18 + kv * 2.0 ** -24).all()
