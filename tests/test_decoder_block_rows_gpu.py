"""Every token of a decoder block's step against a 64-bit restatement, request
by request: the attention, both outputs of the norm that closes it and, with
the memory layer run on the kernels' own input (so that no near-tied slot can
change), both outputs of the norm that closes the layer."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2411_12364_gb300 import workloads
from paper_2411_12364_gb300.norms import block_norm
from paper_2411_12364_gb300.paged import paged_append, paged_attention, paged_check

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


def rms64(x, w):
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w.double()


def rows_within(got, want, bound, what, lens):
    """|got - want| <= bound for every entry, named by request and token."""
    over = ((got.double() - want).abs() - bound).amax(-1)
    at = 0
    for r, count in enumerate(lens):
        worst = over[at:at + count]
        assert (worst <= 0).all(), f"{what}: request {r}, token {worst.argmax().item()}"
        at += count


def close64(y, u, p):
    """The stream before it is stored, and a bound of the kernel's error: one
    rounding of the stored stream, fp32 arithmetic (2^-16 of the row's terms)."""
    add = p["gate"].double() * rms64(y.double(), p["w_post"])
    want = u.double() + add
    return want, U16 * want.abs() + 2.0 ** -16 * (u.double().abs() + add.abs().amax(-1, True))


def open64(u, p):
    """The next input from the stream as stored, and its bound."""
    want = rms64(u.double(), p["w_pre"])
    return want, U16 * want.abs() + 2.0 ** -16 * want.abs().amax(-1, True)


@pytest.mark.parametrize("lens,steps", [([17, 1, 30], 2), ([1, 1], 1), ([130, 0, 5, 64], 1)])
def test_every_token_of_a_step(example, lens, steps, gpu_lib):
    cfg = workloads.small_config(d_in=128, d_out=128, n=32)
    block = example.DecoderBlock(cfg, 4, 2, 32, 256)
    h, hk, hd = block.heads, block.kv_heads, block.head_dim
    gen = torch.Generator(device="cuda").manual_seed(4)
    cache = example.Cache(40, len(lens), 12, hk, hd)
    past = [[torch.zeros(0, hk, hd, dtype=torch.float64, device="cuda")] * 2 for _ in lens]
    for step in range(steps):
        new = lens if step == 0 else [1] * len(lens)
        u = torch.randn(sum(new), 128, generator=gen, device="cuda").to(BF16)
        u, n = block_norm(torch.zeros_like(u), u, post=False)
        q_start, kv_lens, slots, max_new = cache.plan(new)
        qkv = (n @ block.w_qkv.T).view(-1, h + 2 * hk, hd)
        paged_append(cache.k, cache.v, qkv[:, h:h + hk], qkv[:, h + hk:], slots)
        a = paged_attention(qkv[:, :h], cache.k, cache.v, cache.table, q_start, kv_lens, max_new)
        want, size, at = [], [], 0
        for r, count in enumerate(new):
            mine = qkv[at:at + count].double()
            past[r] = [torch.cat([x, mine[:, i:i + hk]]) for x, i in zip(past[r], (h, h + hk))]
            k, v = (x.repeat_interleave(h // hk, 1) for x in past[r])
            s = torch.einsum("nhd,khd->hnk", mine[:, :h], k) / math.sqrt(hd)
            later = torch.ones(count, len(k), device="cuda").triu(len(k) - count + 1) > 0
            p = torch.softmax(s.masked_fill(later, -math.inf), -1)
            want.append(torch.einsum("hnk,khd->nhd", p, v))
            size.append(torch.einsum("hnk,khd->nhd", p, v.abs()))
            at += count
        # weights and output are each rounded once to bf16
        rows_within(a.flatten(1), torch.cat(want).flatten(1),
                    2.1 * U16 * torch.cat(size).flatten(1) + 1e-6, "attention", new)
        y = a.view(-1, h * hd) @ block.w_o.T
        u1, n1 = block_norm(y, u, **block.norms[0])
        rows_within(u1, *close64(y, u, block.norms[0]), "u after attention", new)
        rows_within(n1, *open64(u1, block.norms[0]), "n after attention", new)
        m = block.layer.forward(n1)
        u2, n2 = block_norm(m, u1, **block.norms[1])
        rows_within(u2, *close64(m, u1, block.norms[1]), "u after the layer", new)
        rows_within(n2, *open64(u2, block.norms[1]), "n after the layer", new)
        # the example's step is these calls
        got_u, got_n = block.serve(u, n, cache, (q_start, kv_lens, slots, max_new))
        assert torch.equal(got_u, u2) and torch.equal(got_n, n2)
    assert block.layer.check() == 0 and paged_check() == 0
