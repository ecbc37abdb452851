"""The gradient of the attention of whole sequences against the formula in 64
bits and against differences of the forward pass."""
import math

import pytest
import torch

from paper_2411_12364_gb300 import paged

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


def starts_of(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def forward(q, k, v, lens, scale):
    """out and lse of whole sequences in 64 bits."""
    T, H, D = q.shape
    group = H // k.shape[1]
    out = torch.zeros(T, H, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    starts = starts_of(lens)
    for a, b in zip(starts, starts[1:]):
        n = b - a
        for h in range(H):
            z = q[a:b, h].double() @ k[a:b, h // group].double().T * scale
            z = z.masked_fill(torch.ones(n, n, device="cuda").triu(1) > 0, -math.inf)
            out[a:b, h] = torch.softmax(z, -1) @ v[a:b, h // group].double()
            lse[a:b, h] = torch.logsumexp(z, -1)
    return out, lse


def gradient(q, k, v, out, lse, dout, lens, scale, half):
    """The formula in 64 bits, and a bound of the error of each result.

    A score is off by D additions of 2^-23 of the sum of magnitudes (the tensor
    cores may truncate), P by that and the error of e^ (2^-20) and of its
    exponent; dout.v and d likewise; P and dS enter the products rounded
    to the storage type (half a step: `half`), n additions each, and the
    result is rounded once."""
    T, H, D = q.shape
    group = H // k.shape[1]
    e = 2.0 ** -23
    want = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, k, v)]
    tol = [torch.zeros_like(x) for x in want]
    starts = starts_of(lens)
    for a, b in zip(starts, starts[1:]):
        n = b - a
        causal = torch.ones(n, n, device="cuda").tril() > 0
        for h in range(H):
            g = h // group
            Q, K, V, O, dO = (x[a:b, i].double() for x, i in
                              ((q, h), (k, g), (v, g), (out, h), (dout, h)))
            L = lse[a:b, h, None].double()
            seen = causal & (L > -math.inf)
            z = Q @ K.T * scale
            p = torch.where(seen, torch.exp(z - torch.where(L > -math.inf, L, 0.0)), 0.0)
            dp = dO @ V.T
            d = (dO * O).sum(1, keepdim=True)
            ds = p * (dp - d) * scale
            z_err = (D + 4) * e * scale * (Q.abs() @ K.abs().T)
            p_rel = z_err + 2.0 ** -20 + 4 * e * (z.abs() + torch.where(L > -math.inf, L, 0.0).abs())
            p_err = p * p_rel
            dp_err = (D + 4) * e * (dO.abs() @ V.abs().T + (dO * O).abs().sum(1, keepdim=True))
            ds_err = ds.abs() * (p_rel + 4 * e) + p * scale * dp_err * (1 + p_rel)
            p_err, ds_err = p_err + half * (p + p_err), ds_err + half * (ds.abs() + ds_err)
            want[0][a:b, h] = ds @ K
            want[1][a:b, g] += ds.T @ Q
            want[2][a:b, g] += p.T @ dO
            steps = (n * group + 10) * e
            tol[0][a:b, h] = ds_err @ K.abs() + steps * (ds.abs() @ K.abs())
            tol[1][a:b, g] += ds_err.T @ Q.abs() + steps * (ds.T.abs() @ Q.abs())
            tol[2][a:b, g] += p_err.T @ dO.abs() + steps * (p.T @ dO.abs())
    return want, [t + half * (w.abs() + t) + 1e-38 for w, t in zip(want, tol)]


def inputs(lens, H, heads, D, dtype, seed=0):
    T = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(seed + T + H + D)
    qkv = torch.randn(T, H + 2 * heads, D, generator=g, device="cuda").to(dtype)
    q, k, v = qkv[:, :H], qkv[:, H:H + heads], qkv[:, H + heads:]
    dout = torch.randn(T, H, D, generator=g, device="cuda").to(dtype)
    scale = 1 / math.sqrt(D)
    out, lse = forward(q, k, v, lens, scale)
    start = torch.tensor(starts_of(lens), dtype=torch.int32, device="cuda")
    return q, k, v, out.to(dtype), lse.float(), dout, start, scale


def check(got, q, k, v, out, lse, dout, lens, scale):
    half = torch.finfo(q.dtype).eps / 2
    want, tol = gradient(q, k, v, out, lse, dout, lens, scale, half)
    for name, a, b, t in zip(("dq", "dk", "dv"), got, want, tol):
        err = (a.double() - b).abs()
        assert bool((err <= t).all()), (name, float((err / t).max()))


LENS = [[1], [2, 1, 3], [64], [63, 0, 65], [128, 128], [127, 1, 129], [0, 0, 5, 0], [300],
        [31, 33, 257, 7]]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("H,heads,D", [(1, 1, 64), (4, 2, 128), (5, 1, 80), (2, 2, 8),
                                       (8, 4, 96), (3, 1, 256), (2, 1, 136)])
def test_gradient(gpu_lib, dtype, lens, H, heads, D):
    q, k, v, out, lse, dout, start, scale = inputs(lens, H, heads, D, dtype)
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    check(got, q, k, v, out, lse, dout, lens, scale)
    again = paged.paged_attention_backward(q, k, v, out, lse, dout, start, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(got, again))     # sums of a fixed order
    assert paged.paged_check() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,H,heads,D", [([1100, 70], 4, 1, 64), ([900, 3, 514], 8, 8, 128),
                                            ([5] * 300, 4, 2, 64), ([40, 600], 64, 1, 64)])
def test_longer_sequences(gpu_lib, dtype, lens, H, heads, D):
    q, k, v, out, lse, dout, start, scale = inputs(lens, H, heads, D, dtype)
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    check(got, q, k, v, out, lse, dout, lens, scale)


@pytest.mark.parametrize("dtype,lens,H,heads,D", [
    (F32, [1] * 5, 8, 1, 64), (F32, [120], 4, 1, 80), (F32, [33], 1, 1, 64),
    (F32, [512] * 4, 8, 2, 64), (F32, [1, 40, 7], 20, 4, 128), (F32, [100] * 16, 16, 2, 80),
    (BF16, [250], 8, 1, 136), (BF16, [200, 3], 2, 1, 256), (F32, [0, 70, 0, 0], 64, 1, 8),
    (BF16, [700], 8, 1, 128), (BF16, [129, 1, 1000], 16, 2, 64), (BF16, [5] * 3, 10, 2, 80)])
def test_blocks_shared_out(gpu_lib, dtype, lens, H, heads, D):
    """Batches in which several thread blocks share out a block of keys."""
    q, k, v, out, lse, dout, start, scale = inputs(lens, H, heads, D, dtype)
    T = q.shape[0]
    given = [torch.full((T + 2, *x.shape[1:]), 9.0, dtype=dtype, device="cuda") for x in (q, k, v)]
    dq, dk, dv = (x[1:T + 1] for x in given)
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, start, dq=dq, dk=dk, dv=dv)
    check(got, q, k, v, out, lse, dout, lens, scale)
    assert all(bool((x[0] == 9).all()) and bool((x[-1] == 9).all()) for x in given)
    again = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_no_sequence(gpu_lib, dtype, D):
    """Rows before, behind and beside a sequence: neither used nor written."""
    lens = [37, 130]
    q, k, v, out, lse, dout, _, scale = inputs(lens, 4, 2, D, dtype)
    T, pad = sum(lens), 60

    def padded(x):
        y = torch.full((T + pad, *x.shape[1:]), NAN, dtype=x.dtype, device="cuda")
        y[10:10 + T] = x
        return y

    q2, k2, v2, out2, lse2, dout2 = (padded(x) for x in (q, k, v, out, lse, dout))
    start = torch.tensor([10, 10 + lens[0], 10 + T], dtype=torch.int32, device="cuda")
    grads = [torch.full_like(x, 7.0) for x in (q2, k2, v2)]
    paged.paged_attention_backward(q2, k2, v2, out2, lse2, dout2, start, dq=grads[0], dk=grads[1],
                                   dv=grads[2])
    check([x[10:10 + T] for x in grads], q, k, v, out, lse, dout, lens, scale)
    for x in grads:
        assert bool((x[:10] == 7).all()) and bool((x[10 + T:] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_as_slices_of_one(gpu_lib, dtype):
    lens = [50, 90]
    q, k, v, out, lse, dout, start, scale = inputs(lens, 4, 2, 64, dtype)
    whole = torch.full((sum(lens), 8 + 1, 64), 3.0, dtype=dtype, device="cuda")
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, start, dq=whole[:, :4],
                                         dk=whole[:, 4:6], dv=whole[:, 6:8])
    check(got, q, k, v, out, lse, dout, lens, scale)
    assert bool((whole[:, 8] == 3).all())
    # an input on another boundary than 16 bytes
    wide = torch.zeros(sum(lens), 4 * 64 + 3, dtype=dtype, device="cuda")
    odd = wide[:, 1:257].unflatten(1, (4, 64))
    odd.copy_(dout)
    same = paged.paged_attention_backward(q, k, v, out, lse, odd, start)
    check(same, q, k, v, out, lse, dout, lens, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_saw_nothing(gpu_lib, dtype):
    """A request that the plan refused: its rows' lse is -inf."""
    lens = [70, 40, 20]
    q, k, v, out, lse, dout, start, scale = inputs(lens, 4, 2, 64, dtype)
    lse[70:110], out[70:110] = -math.inf, 0.0
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    check(got, q, k, v, out, lse, dout, lens, scale)
    for x in got:
        assert not bool(x[70:110].any())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_after_the_paged_forward(gpu_lib, dtype):
    """The run as a step makes it: plan, append, attention, gradient."""
    lens, H, heads, D, page = [150, 1, 77], 8, 2, 128, 16
    q, k, v, _, _, dout, _, scale = inputs(lens, H, heads, D, dtype)
    T, R = sum(lens), len(lens)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.full((R, 12), -1, **i32)
    pages = torch.randperm(24, device="cuda").to(torch.int32)
    q_start, kv_lens, slots, _ = paged.paged_plan(
        torch.zeros(R, **i32), torch.tensor(lens, **i32), table, pages, torch.tensor([24], **i32),
        page, T)
    caches = [torch.zeros(24, heads, page, D, dtype=dtype, device="cuda") for _ in range(2)]
    paged.paged_append(*caches, k, v, slots)
    out, lse = paged.paged_attention(q, *caches, table, q_start, kv_lens, max(lens), with_lse=True)
    got = paged.paged_attention_backward(q, k, v, out, lse, dout, q_start)
    check(got, q, k, v, out, lse, dout, lens, scale)


def test_gradient_against_differences(gpu_lib):
    """Central differences of sum(dout . out) in 64 bits against 32-bit storage."""
    lens = [9, 4]
    q, k, v, out, lse, dout, start, scale = inputs(lens, 4, 2, 16, F32)
    grads = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    h = 1e-4

    def total(*x):
        return float((forward(*x, lens, scale)[0] * dout.double()).sum())

    # h^2 times a third derivative (of order 10 here) and 32-bit errors of the
    # gradient: 2^-20 of its terms' magnitudes, which stay below 100
    tol = 10 * h * h + 100 * 2.0 ** -20
    for n, (t, c, e) in ((0, (5, 3, 2)), (0, (12, 0, 7)), (1, (0, 1, 15)), (1, (10, 0, 3)),
                         (2, (8, 1, 0)), (2, (3, 0, 9))):
        x = [y.double() for y in (q, k, v)]
        up = [y.clone() for y in x]
        down = [y.clone() for y in x]
        up[n][t, c, e] += h
        down[n][t, c, e] -= h
        assert abs((total(*up) - total(*down)) / (2 * h) - float(grads[n][t, c, e])) <= tol


def test_captured_beside_an_eager_call(gpu_lib):
    lens = [200, 33]
    q, k, v, out, lse, dout, start, scale = inputs(lens, 4, 2, 64, BF16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
    for seed in (1, 2):
        fresh = inputs(lens, 4, 2, 64, BF16, seed=seed)
        for a, b in zip((q, k, v, out, lse, dout), fresh):
            a.copy_(b)
        graph.replay()
        eager = paged.paged_attention_backward(q, k, v, out, lse, dout, start)
        torch.cuda.synchronize()
        check(got, q, k, v, out, lse, dout, lens, scale)
        assert all(torch.equal(a, b) for a, b in zip(got, eager))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_past_32_bits(gpu_lib, dtype):
    """Tokens so far apart that the last ones' offsets pass 2^32 entries."""
    lens, H, heads, D = [70, 60], 2, 1, 64
    q, k, v, out, lse, dout, start, scale = inputs(lens, H, heads, D, dtype)
    T, step = sum(lens), 2 ** 25 + 64        # 130 steps: 4.4e9 entries

    def apart(x):
        n = x.shape[1] * D
        flat = torch.empty((T - 1) * step + n, dtype=dtype, device="cuda")
        y = flat.as_strided((T, x.shape[1], D), (step, D, 1))
        y.copy_(x)
        return y

    got = paged.paged_attention_backward(apart(q), k, apart(v), out, lse, apart(dout), start,
                                         dq=apart(torch.zeros_like(q)))
    check(got, q, k, v, out, lse, dout, lens, scale)


def test_first_call_inside_a_capture(gpu_lib):
    """In a process of its own, where nothing was looked up before."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    body = """
import torch
from paper_2411_12364_gb300 import binding, paged, vocab
binding.load()
bf = dict(dtype=torch.bfloat16, device="cuda")
x, w = torch.randn(40, 64, **bf), torch.randn(300, 64, **bf)
ids = torch.arange(40, device="cuda")
q, k = torch.randn(40, 2, 64, **bf), torch.randn(40, 1, 64, **bf)
lse = torch.full((40, 2), 5.0, device="cuda")
start = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
stream = torch.cuda.Stream()
stream.wait_stream(torch.cuda.current_stream())
graph = torch.cuda.CUDAGraph()


def run():
    loss, row = vocab.cross_entropy(x, w, ids)
    dx, dw = vocab.cross_entropy_backward(x, w, ids, row, torch.ones_like(row))
    return (loss, dx, dw, vocab.embedding(w, ids), vocab.embedding_backward(ids, x, 300),
            *paged.paged_attention_backward(q, k, k, q, lse, q, start))


with torch.cuda.graph(graph, stream=stream):
    held = run()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(held, run()))
print("done")
"""
    out = subprocess.run([sys.executable, "-c", body], cwd=root, capture_output=True, text=True,
                         timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "done", out.stdout + out.stderr
