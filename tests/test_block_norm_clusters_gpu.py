"""The gradient of rows past 4096 entries runs in clusters of two blocks that
exchange their sums.  Its results do not depend on what else the GPU does: a
call beside other work, whose blocks start late and unevenly, gives the bits
of a call alone."""
import pytest
import torch

from paper_2411_12364_gb300.norms import block_norm_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("T,D,dtype", [(1, 8192, torch.bfloat16), (37, 5000, torch.float32),
                                       (600, 8192, torch.bfloat16), (90, 4097, torch.bfloat16)])
def test_wide_gradients_beside_other_work(T, D, dtype, kind, gpu_lib):
    gen = torch.Generator(device="cuda").manual_seed(T)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    p = dict(y=randn(T, D).to(dtype), u=randn(T, D).to(dtype), du=randn(T, D).to(dtype),
             dn=randn(T, D).to(dtype), w_post=randn(D), w_pre=randn(D), gate=randn(D))
    want = block_norm_backward(kind=kind, **p)
    torch.cuda.synchronize()
    busy, side = torch.cuda.Stream(), torch.cuda.Stream()
    x = torch.randn(1024, 1024, device="cuda", dtype=torch.bfloat16)
    side.wait_stream(torch.cuda.current_stream())
    busy.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(40):
        with torch.cuda.stream(busy):
            x @ x
        with torch.cuda.stream(side):
            got.append(block_norm_backward(kind=kind, **p))
    torch.cuda.synchronize()
    for g in got:
        for name, t in want.items():
            assert t is None or torch.equal(g[name], t), name
