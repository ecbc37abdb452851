"""The decoder-block operators as one path (examples/decoder_block.py): a
prompt taken whole and the same tokens in chunks and single steps agree, the
block agrees with its parts in plain torch, and the memory half's gradient
with autograd through the same slots."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2411_12364_gb300 import workloads
from paper_2411_12364_gb300.norms import block_norm
from paper_2411_12364_gb300.paged import paged_check

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = torch.bfloat16
U16 = 2.0 ** -8     # rounding to bf16


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "decoder_block", os.path.join(ROOT, "examples", "decoder_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _block(example, heads=(4, 2), dim=32, tokens=64):
    cfg = workloads.small_config(d_in=128, d_out=128, n=32)
    return example.DecoderBlock(cfg, heads[0], heads[1], dim, tokens)


def _inputs(count, d, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.randn(count, d, generator=gen, device="cuda").to(BF16)
    return block_norm(torch.zeros_like(u), u, post=False)


def test_chunks_and_single_steps_give_the_whole_prompt(example, gpu_lib):
    """The attention's kernels differ between a prompt, a chunk and a token
    (same inputs, fp32 sums, weights rounded to bf16), so the attention
    outputs agree to two roundings of weights and output: 4 U16 of the row's
    typical entry, element-wise at 4 times that for the largest."""
    block = _block(example)
    h, hk, hd = block.heads, block.kv_heads, block.head_dim
    total = 60
    u, n = _inputs(total, 128)
    seen = []
    for parts in ([total], [33, 20, 1, 1, 5], [1] * total):
        cache = example.Cache(12, 1, 8, hk, hd)
        outs, at = [], 0
        for count in parts:
            q_start, kv_lens, slots, max_new = cache.plan([count])
            qkv = (n[at:at + count] @ block.w_qkv.T).view(-1, h + 2 * hk, hd)
            example.paged_append(cache.k, cache.v, qkv[:, h:h + hk], qkv[:, h + hk:], slots)
            outs.append(example.paged_attention(qkv[:, :h], cache.k, cache.v, cache.table, q_start,
                                                kv_lens, max_new))
            at += count
        assert cache.lens.item() == total and cache.free.item() == 12 - math.ceil(total / 16)
        seen.append(torch.cat(outs).float())
    for other in seen[1:]:
        err = (other - seen[0]).abs()
        rms = seen[0].square().mean().sqrt()
        assert err.square().mean().sqrt() <= 4 * U16 * rms
        assert err.max() <= 16 * U16 * seen[0].abs().max()
    assert paged_check() == 0


def test_block_agrees_with_its_parts_in_torch(example, gpu_lib):
    """Attention and both norms restated in 64 bits between the kernels' own
    roundings; the memory layer is the library's own call on the same n."""
    block = _block(example)
    h, hk, hd = block.heads, block.kv_heads, block.head_dim
    lens = [17, 1, 30]
    u, n = _inputs(sum(lens), 128, seed=1)
    cache = example.Cache(12, 3, 4, hk, hd)
    u2, n2 = block.serve(u, n, cache, cache.plan(lens))
    qkv = (n @ block.w_qkv.T).view(-1, h + 2 * hk, hd).double()
    outs, at = [], 0
    for count in lens:
        q, k, v = (qkv[at:at + count, a:b] for a, b in ((0, h), (h, h + hk), (h + hk, h + 2 * hk)))
        k, v = (x.repeat_interleave(h // hk, 1) for x in (k, v))
        s = torch.einsum("nhd,khd->hnk", q, k) / math.sqrt(hd)
        s = s.masked_fill(torch.ones(count, count, device="cuda").triu(1) > 0, -math.inf)
        outs.append(torch.einsum("hnk,khd->nhd", torch.softmax(s, -1), v))
        at += count
    a = torch.cat(outs).to(BF16).reshape(-1, h * hd) @ block.w_o.T

    def rms(x, w):
        return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w

    def close(y, u, p):
        u = (u.double() + p["gate"] * rms(y.double(), p["w_post"])).to(BF16)
        return u, rms(u.double(), p["w_pre"]).to(BF16)

    u1, n1 = close(a, u, block.norms[0])
    want_u, want_n = close(block.layer.forward(n1), u1, block.norms[1])
    # roundings of the attention's weights and outputs pass through the norms
    # and, where they move a near-tied slot, through the layer's selection
    for got, want in ((u2, want_u), (n2, want_n)):
        off = ((got.double() - want.double()).norm(dim=-1) / want.double().norm(dim=-1))
        assert off.median() <= 4 * U16
    assert block.layer.check() == 0 and paged_check() == 0


def test_memory_gradient_matches_autograd(example, gpu_lib):
    block = _block(example)
    T = 24
    u, n = _inputs(T, 128, seed=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    du, dn = (torch.randn(T, 128, generator=gen, device="cuda").to(BF16) for _ in range(2))
    got = block.memory_gradient(u, n, du, dn)
    idx, w = block.layer.retrieve(n)
    y = block.layer.lookup_reduce(idx, w).double().requires_grad_()
    p = {k: v.double().requires_grad_() for k, v in block.norms[1].items()}

    def rms(x, w):
        return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w

    stored, _ = block_norm(y.detach().to(BF16), u, **block.norms[1])
    s = stored.double().requires_grad_()
    rms(s, p["w_pre"]).backward(dn.double())
    gu = du.double() + s.grad
    (p["gate"] * rms(y, p["w_post"])).backward(gu)
    for name, want in (("dy", y.grad), ("dr", gu), ("dw_post", p["w_post"].grad),
                       ("dw_pre", p["w_pre"].grad), ("dgate", p["gate"].grad)):
        low = U16 if got[name].dtype == BF16 else 1e-5
        err = (got[name].double() - want).norm() / want.norm()
        assert err <= low, name
    # the lookup's gradient takes dy as it was stored
    dv, dw, dwp = block.layer.lookup_reduce_backward(idx, w, got["dy"])
    assert torch.equal(dw, got["dw"]) and torch.equal(dwp, got["dw_proj"])
    assert ((dv - got["dvalues"]).norm() <= 1e-5 * dv.norm())


def test_example_runs(example, gpu_lib, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["decoder_block.py", "--steps", "2"])
    example.main()
    text = capsys.readouterr().out
    assert "lengths [39, 132, 66, 3]" in text and "dvalues" in text


FIRST_CALL = """
import torch
from paper_2411_12364_gb300.norms import block_norm, block_norm_backward
from paper_2411_12364_gb300.paged import paged_append, paged_attention, paged_plan
i32 = dict(dtype=torch.int32, device="cuda")
k = torch.zeros(8, 2, 16, 64, device="cuda", dtype=torch.bfloat16)
v = torch.zeros_like(k)
new = torch.randn(40, 2, 64, device="cuda").bfloat16()
q = torch.randn(40, 4, 64, device="cuda").bfloat16()
x = torch.randn(40, 256, device="cuda").bfloat16()
lens, table = torch.zeros(1, **i32), torch.zeros(1, 4, **i32)
pages, free = torch.arange(8, **i32), torch.tensor([8], **i32)
count = torch.tensor([40], **i32)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    start, kv, slots, _ = paged_plan(lens, count, table, pages, free, 16, 40)
    paged_append(k, v, new, new, slots)
    many = paged_attention(q, k, v, table, start, kv, 40)
    few = paged_attention(q, k, v, table, start, kv, 1)
    single = paged_attention(q.float(), k.float(), v.float(), table, start, kv, 40)
    u, n = block_norm(x, x)
    grads = block_norm_backward(x, u, n, n)
g.replay()
torch.cuda.synchronize()
assert slots.tolist() == [int(table[0, t // 16]) * 16 + t % 16 for t in range(40)]
assert (many.float() - single).abs().max() < 0.05 and (few.float() - single).abs().max() < 0.05
assert torch.isfinite(grads["dy"].float()).all()
print("captured")
"""


def test_first_calls_may_be_captured(gpu_lib):
    """In a fresh process the very first call of each operator is inside a
    graph capture."""
    import subprocess
    import sys
    out = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=ROOT, capture_output=True,
                         text=True, timeout=300)
    assert out.returncode == 0 and "captured" in out.stdout, out.stderr[-2000:]
