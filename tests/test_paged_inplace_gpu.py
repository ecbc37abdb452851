"""Attention with its output in the queries' place gives the bits of the same
call with an output of its own."""
import pytest
import torch

from paper_2411_12364_gb300 import binding
from paper_2411_12364_gb300.paged import paged_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.bfloat16, 64),
                                       (torch.bfloat16, 192), (torch.float32, 128)])
@pytest.mark.parametrize("news", [[1, 1, 1, 0, 1], [5, 300, 1, 0, 77], [40] * 30],
                         ids=["single", "chunks", "many"])
def test_output_in_the_queries_place(dtype, dim, news, gpu_lib):
    gen = torch.Generator(device="cuda").manual_seed(dim)
    page, hq, hk = 16, 8, 2
    R, T = len(news), sum(news)
    kv = [n + 4000 * (r % 3) + 17 * r for r, n in enumerate(news)]
    width = max(-(-k // page) for k in kv) + 1

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    k, v = randn(R * width, hk, page, dim), randn(R * width, hk, page, dim)
    table = torch.randperm(R * width, generator=gen, device="cuda").to(torch.int32).view(R, width)
    start = torch.tensor([0] + torch.tensor(news).cumsum(0).tolist(), dtype=torch.int32,
                         device="cuda")
    lens = torch.tensor(kv, dtype=torch.int32, device="cuda")
    q = randn(T, hq, dim)
    want = paged_attention(q, k, v, table, start, lens, max(news), with_lse=True)
    for _ in range(5):
        x = q.clone()
        got = paged_attention(x, k, v, table, start, lens, max(news), out=x, with_lse=True)
        assert got[0].data_ptr() == x.data_ptr()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_overlapping_outputs_are_refused(gpu_lib):
    k = torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    ints = dict(dtype=torch.int32, device="cuda")
    start, lens, table = torch.tensor([0, 4], **ints), torch.tensor([40], **ints), \
        torch.arange(4, **ints).view(1, 4)
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.UltraMemError) as e:
        paged_attention(q[:4], k, k.clone(), table, start, lens, 4, out=q[1:])
    assert e.value.status == binding.EINVAL
