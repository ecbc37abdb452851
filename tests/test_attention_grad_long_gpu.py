"""The gradient of attention where its lists of blocks count the longest together
(sequences of more than 1024 blocks), and wide heads over longer sequences."""
import math

import pytest
import torch

from paper_2411_12364_gb300 import paged
from tests.test_attention_grad_gpu import check, inputs, starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def one_head(q, k, v, out, lse, dout, lens, scale, half):
    """The formula in 64 bits for one head, in pieces of 2048 rows, and bounds as in
    the other tests of this gradient."""
    T, _, D = q.shape
    e = 2.0 ** -23
    q, k, v, out, dout = (x[:, 0].double() for x in (q, k, v, out, dout))
    want = [torch.zeros(T, D, dtype=torch.float64, device="cuda") for _ in range(3)]
    tol = [torch.zeros_like(x) for x in want]
    starts = starts_of(lens)
    for a, b in zip(starts, starts[1:]):
        n = b - a
        steps = (n + 10) * e
        for r in range(a, b, 2048):
            rows, keys = slice(r, min(b, r + 2048)), slice(a, min(b, r + 2048))
            Q, O, dO, K, V = q[rows], out[rows], dout[rows], k[keys], v[keys]
            L = lse[rows].double()
            at = torch.arange(a, keys.stop, device="cuda")
            seen = at[None, :] <= torch.arange(rows.start, rows.stop, device="cuda")[:, None]
            z = Q @ K.T * scale
            p = torch.where(seen, torch.exp(z - L), 0.0)
            ds = p * (dO @ V.T - (dO * O).sum(1, keepdim=True)) * scale
            z_err = (D + 4) * e * scale * (Q.abs() @ K.abs().T)
            p_rel = z_err + 2.0 ** -20 + 4 * e * (z.abs() + L.abs())
            dp_err = (D + 4) * e * (dO.abs() @ V.abs().T + (dO * O).abs().sum(1, keepdim=True))
            ds_err = ds.abs() * (p_rel + 4 * e) + p * scale * dp_err * (1 + p_rel)
            p_err = p * p_rel
            p_err, ds_err = p_err + half * (p + p_err), ds_err + half * (ds.abs() + ds_err)
            want[0][rows] = ds @ K
            want[1][keys] += ds.T @ Q
            want[2][keys] += p.T @ dO
            tol[0][rows] = ds_err @ K.abs() + steps * (ds.abs() @ K.abs())
            tol[1][keys] += ds_err.T @ Q.abs() + steps * (ds.T.abs() @ Q.abs())
            tol[2][keys] += p_err.T @ dO.abs() + steps * (p.T @ dO.abs())
    return want, [t + half * (w.abs() + t) + 1e-38 for w, t in zip(want, tol)]


@pytest.mark.parametrize("dtype,lens,D", [
    (BF16, [300, 132000, 5, 0, 131072, 700], 64),  # 1032 blocks of 128, 1024 and few
    (F32, [65537, 129, 66000], 8),                 # blocks of 64
])
def test_more_than_1024_blocks(gpu_lib, dtype, lens, D):
    T = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k, v, out, dout = (torch.randn(T, 1, D, generator=g, device="cuda").to(dtype)
                          for _ in range(5))
    # any lse will do: rows of about the sum that unit scores have
    at = torch.cat([torch.arange(n, device="cuda") for n in lens])
    lse = (torch.log1p(at.double()) + 0.5).float()[:, None].contiguous()
    start = torch.tensor(starts_of(lens), dtype=torch.int32, device="cuda")
    scale = 1 / math.sqrt(D)
    given = [torch.full_like(q, 9.0) for _ in range(3)]
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, start, dq=given[0], dk=given[1],
                                         dv=given[2])
    want, tol = one_head(q, k, v, out, lse, dout, lens, scale, torch.finfo(dtype).eps / 2)
    for name, a, b, t in zip(("dq", "dk", "dv"), got, want, tol):
        err = (a[:, 0].double() - b).abs()
        assert bool((err <= t).all()), (name, float((err / t).max()))
    again = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert paged.paged_check() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,H,heads,D", [([1500, 3, 700], 4, 2, 256), ([2100], 3, 1, 136),
                                            ([600] * 5, 2, 2, 200)])
def test_wide_heads(gpu_lib, dtype, lens, H, heads, D):
    q, k, v, out, lse, dout, start, scale = inputs(lens, H, heads, D, dtype)
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    check(got, q, k, v, out, lse, dout, lens, scale)
    assert paged.paged_check() == 0
