"""A decoder block around the memory layer, served and trained.

Serving: requests of different lengths share a paged key/value cache.  A step
plans pages and slots for the requests' new tokens on the GPU, and each block
then appends keys and values, attends, closes the attention with the fused
norm (post-norm, gate, residual, the next pre-norm), runs the memory layer and
closes that the same way:

    n -> attention -> u, n = block_norm(.) -> memory layer -> u, n = block_norm(.)

Training: the gradient of the second half (block_norm around the memory
layer's lookup) down to the value table, the slot weights, the projectors, the
gains and the gate; and a whole step of the first half between its ends, from
token ids to the loss and back: embedding, attention of packed sequences,
cross entropy against the same table, and the gradients of all of them.

    python examples/decoder_block.py [--steps N]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2411_12364_gb300 import workloads  # noqa: E402
from paper_2411_12364_gb300.binding import UltraMemLayer  # noqa: E402
from paper_2411_12364_gb300.norms import block_norm, block_norm_backward  # noqa: E402
from paper_2411_12364_gb300.paged import (paged_append, paged_attention,  # noqa: E402
                                          paged_attention_backward, paged_check, paged_plan)
from paper_2411_12364_gb300.vocab import (cross_entropy, cross_entropy_backward,  # noqa: E402
                                          embedding, embedding_backward)

BF16 = torch.bfloat16


class Cache:
    """Pages of one block's keys and values, and the pages' bookkeeping."""

    def __init__(self, n_pages, requests, width, kv_heads, head_dim, page_size=16, dtype=BF16):
        self.page_size = page_size
        shape = (n_pages, kv_heads, page_size, head_dim)
        self.k = torch.zeros(shape, dtype=dtype, device="cuda")
        self.v = torch.zeros(shape, dtype=dtype, device="cuda")
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
        self.free_pages = torch.arange(n_pages, dtype=torch.int32, device="cuda")
        # the free list's length before and after a step change places
        self.free = torch.tensor([n_pages], dtype=torch.int32, device="cuda")
        self.left = torch.zeros_like(self.free)
        self.lens = torch.zeros(requests, dtype=torch.int32, device="cuda")

    def plan(self, new_lens):
        """Slots for new_lens (host numbers) more tokens of each request."""
        new = torch.tensor(new_lens, dtype=torch.int32, device="cuda")
        q_start, kv_lens, slots, _ = paged_plan(self.lens, new, self.table, self.free_pages,
                                                self.free, self.page_size, sum(new_lens),
                                                free_left=self.left)
        self.free, self.left = self.left, self.free
        # a refused request keeps its length (its kv_len is 0)
        self.lens = torch.maximum(kv_lens, self.lens)
        return q_start, kv_lens, slots, max(new_lens)


class DecoderBlock:
    """Attention and one UltraMem layer with pre- and post-norms."""

    def __init__(self, cfg, q_heads, kv_heads, head_dim, max_tokens, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, std=1.0):
            return torch.randn(*shape, generator=gen, device="cuda") * std

        d = cfg["d_in"]
        self.heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.w_qkv = randn((q_heads + 2 * kv_heads) * head_dim, d, std=d ** -0.5).to(BF16)
        self.w_o = randn(d, q_heads * head_dim, std=(q_heads * head_dim) ** -0.5).to(BF16)
        weights = workloads.make_weights(cfg, device="cuda")
        self.layer = UltraMemLayer(cfg, weights, max_tokens)
        # post-norm gain, gate and next pre-norm gain after attention and after the layer
        self.norms = [dict(w_post=1 + 0.1 * randn(d), gate=0.5 + 0.1 * randn(d),
                           w_pre=1 + 0.1 * randn(d)) for _ in range(2)]

    def serve(self, u, n, cache, step):
        """One step's tokens through the block: the stream u and the normed
        input n [tokens, d] -> the same after the block."""
        q_start, kv_lens, slots, max_new = step
        h, hk, hd = self.heads, self.kv_heads, self.head_dim
        qkv = (n @ self.w_qkv.T).view(-1, h + 2 * hk, hd)
        paged_append(cache.k, cache.v, qkv[:, h:h + hk], qkv[:, h + hk:], slots)
        a = paged_attention(qkv[:, :h], cache.k, cache.v, cache.table, q_start, kv_lens, max_new)
        u, n = block_norm(a.view(-1, h * hd) @ self.w_o.T, u, **self.norms[0])
        return block_norm(self.layer.forward(n), u, **self.norms[1])

    def memory_gradient(self, u, n, du, dn):
        """Gradients of the memory half at its inputs u, n, for the gradients
        of its outputs: of the norms' parameters, the table, the slots'
        weights, the projectors and the residual stream."""
        idx, w = self.layer.retrieve(n)
        y = self.layer.lookup_reduce(idx, w)
        u_out, _ = block_norm(y, u, **self.norms[1])
        g = block_norm_backward(y, u_out, du, dn, **self.norms[1])
        dvalues, dw, dw_proj = self.layer.lookup_reduce_backward(idx, w, g["dy"])
        return dict(g, dvalues=dvalues, dw=dw, dw_proj=dw_proj)


class AttentionStep:
    """One attention block between the ends of a language model, whose table
    embeds the ids and scores the vocabulary."""

    def __init__(self, vocab, dim, q_heads, kv_heads, head_dim, dtype=BF16, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, std=1.0):
            return torch.randn(*shape, generator=gen, device="cuda") * std

        self.heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.scale = dim ** 0.5
        self.table = randn(vocab, dim, std=dim ** -0.5).to(dtype)
        self.w_qkv = randn((q_heads + 2 * kv_heads) * head_dim, dim, std=dim ** -0.5).to(dtype)
        self.w_o = randn(dim, q_heads * head_dim, std=(q_heads * head_dim) ** -0.5).to(dtype)
        self.w_in = 1 + 0.1 * randn(dim)              # the gain before attention
        self.norm = dict(w_post=1 + 0.1 * randn(dim), gate=0.5 + 0.1 * randn(dim),
                         w_pre=1 + 0.1 * randn(dim))

    def step(self, ids, labels, lens):
        """The tokens' losses and the gradient of their mean over the labelled
        ones, for sequences of lens tokens (host numbers) packed in ids."""
        h, hk, hd = self.heads, self.kv_heads, self.head_dim
        x = embedding(self.table, ids, scale=self.scale)
        none = torch.zeros_like(x)                    # no block before the first norm
        _, n = block_norm(none, x, w_pre=self.w_in, post=False)
        qkv = (n @ self.w_qkv.T).view(-1, h + 2 * hk, hd)
        q, k, v = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        pages = [-(-length // 16) for length in lens]
        cache = Cache(sum(pages), len(lens), max(pages), hk, hd, dtype=x.dtype)
        q_start, kv_lens, slots, max_new = cache.plan(lens)
        paged_append(cache.k, cache.v, k, v, slots)
        a, lse_rows = paged_attention(q, cache.k, cache.v, cache.table, q_start, kv_lens, max_new,
                                      with_lse=True)
        y = a.view(-1, h * hd) @ self.w_o.T
        u, out = block_norm(y, x, **self.norm)
        loss, lse = cross_entropy(out, self.table, labels)

        counts = (labels >= 0) & (labels < self.table.shape[0])
        dloss = counts.float() / counts.sum().clamp(min=1)
        dout, dtable = cross_entropy_backward(out, self.table, labels, lse, dloss)
        g = block_norm_backward(y, u, None, dout, **self.norm)
        da = (g["dy"] @ self.w_o).view(-1, h, hd)
        dqkv = torch.empty_like(qkv)
        paged_attention_backward(q, k, v, a, lse_rows, da, q_start, dq=dqkv[:, :h],
                                 dk=dqkv[:, h:h + hk], dv=dqkv[:, h + hk:])
        flat = dqkv.view(dqkv.shape[0], -1)
        g_in = block_norm_backward(none, x, g["dr"], flat @ self.w_qkv, w_pre=self.w_in, post=False)
        embedding_backward(ids, g_in["dr"], self.table.shape[0], scale=self.scale, dtable=dtable,
                           accumulate=True)
        return loss, dict(table=dtable, w_qkv=flat.T @ n, w_o=g["dy"].T @ a.view(-1, h * hd),
                          w_in=g_in["dw_pre"], w_post=g["dw_post"], gate=g["dgate"],
                          w_pre=g["dw_pre"])


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=4, help="decode steps after the prompts")
    args = ap.parse_args()
    cfg = workloads.layer_config("decode_1m")
    prompts = [37, 130, 64, 1]
    block = DecoderBlock(cfg, q_heads=8, kv_heads=2, head_dim=128, max_tokens=sum(prompts))
    cache = Cache(n_pages=64, requests=len(prompts), width=16, kv_heads=2, head_dim=128)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def tokens(count):
        u = torch.randn(count, cfg["d_in"], generator=gen, device="cuda").to(BF16)
        # the first pre-norm of the stack: no block before it
        return block_norm(torch.zeros_like(u), u, post=False)

    for new_lens in [prompts] + [[1] * len(prompts)] * args.steps:
        u, n = tokens(sum(new_lens))
        u, n = block.serve(u, n, cache, cache.plan(new_lens))
        print(f"{sum(new_lens):4d} tokens, lengths {cache.lens.tolist()}, free pages "
              f"{cache.free.item()}, |u| {u.float().norm().item() / math.sqrt(u.numel()):.3f}")
    du, dn = torch.randn_like(u), torch.randn_like(n)
    grads = block.memory_gradient(u, n, du, dn)
    print("gradients:", ", ".join(f"{k} {tuple(v.shape)}" for k, v in grads.items()
                                  if v is not None))
    model = AttentionStep(vocab=5000, dim=512, q_heads=8, kv_heads=2, head_dim=64)
    ids = torch.randint(0, 5000, (sum(prompts),), generator=gen, device="cuda")
    loss, grads = model.step(ids, ids.roll(-1), prompts)
    print(f"loss {loss.mean().item():.3f}, gradients:",
          ", ".join(f"{k} {tuple(v.shape)}" for k, v in grads.items()))
    assert block.layer.check() == 0 and paged_check() == 0
    block.layer.close()


if __name__ == "__main__":
    main()
