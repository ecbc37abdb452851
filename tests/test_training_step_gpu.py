"""A training step through the embedding, the norms, attention of packed
sequences and the cross entropy (examples/decoder_block.py, AttentionStep):
its loss and all its gradients against autograd in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2411_12364_gb300.paged import paged_check

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "decoder_block", os.path.join(ROOT, "examples", "decoder_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(model, ids, labels, lens):
    """The step in 64 bits at the stored parameters, by autograd."""
    names = dict(table=model.table, w_qkv=model.w_qkv, w_o=model.w_o, w_in=model.w_in, **model.norm)
    p = {k: v.double().requires_grad_() for k, v in names.items()}

    def rms(x, w):
        return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w

    h, hk, hd = model.heads, model.kv_heads, model.head_dim
    V = model.table.shape[0]
    known = (ids >= 0) & (ids < V)
    x = torch.where(known[:, None], p["table"][ids.clamp(0, V - 1)] * model.scale, 0.0)
    qkv = (rms(x, p["w_in"]) @ p["w_qkv"].T).view(-1, h + 2 * hk, hd)
    rows, at = [], 0
    for n in lens:
        q, k, v = (t.transpose(0, 1) for t in qkv[at:at + n].split([h, hk, hk], 1))
        k, v = (t.repeat_interleave(h // hk, 0) for t in (k, v))
        z = q @ k.transpose(1, 2) / math.sqrt(hd)
        z = z.masked_fill(torch.ones(n, n, device="cuda").triu(1) > 0, -math.inf)
        rows.append((torch.softmax(z, -1) @ v).transpose(0, 1).reshape(n, -1))
        at += n
    u = x + p["gate"] * rms(torch.cat(rows) @ p["w_o"].T, p["w_post"])
    z = rms(u, p["w_pre"]) @ p["table"].T
    counts = (labels >= 0) & (labels < V)
    lse = torch.logsumexp(z, 1)
    loss = torch.where(counts, lse - z.gather(1, labels.clamp(0, V - 1)[:, None])[:, 0], 0.0)
    (loss.sum() / counts.sum().clamp(min=1)).backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,heads,hd", [([40, 1, 77], (4, 2), 64), ([130, 5], (2, 1), 128),
                                           ([3], (3, 3), 16)])
def test_step(example, gpu_lib, dtype, lens, heads, hd):
    """From the ids to a gradient and back lie at most 24 results that are
    rounded to the storage type (or products of fp32 storage whose sums lose
    that much); each is off by at most half a step of its size, and each map
    on the way changes a relative error, taken over a whole tensor, by a factor of
    order 1 (2 is allowed for)."""
    V, dim = 300, 128
    model = example.AttentionStep(V, dim, *heads, hd, dtype=dtype, seed=len(lens))
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, V, (sum(lens),), generator=gen, device="cuda")
    labels = ids.roll(-1)
    labels[::7] = -100                   # tokens without a target
    if len(ids) > 5:
        ids[4] = -1                      # and one without an id
    loss, grads = model.step(ids, labels, lens)
    want_loss, want = reference(model, ids, labels, lens)
    tol = 2 * 24 * (torch.finfo(dtype).eps / 2)
    tol = max(tol, 2 * 24 * 2.0 ** -20)  # fp32: exponentials and sums of hundreds of terms
    assert float((loss.double() - want_loss).abs().max()) <= tol * (1 + float(want_loss.abs().max()))
    assert set(grads) == set(want)
    for name, g in grads.items():
        err = float((g.double() - want[name]).norm() / want[name].norm())
        assert err <= tol, (name, err)
    assert paged_check() == 0


def test_captured_step(example, gpu_lib):
    """The run of calls in one graph, replayed on other ids, beside eager calls."""
    lens, V = [33, 70], 200
    model = example.AttentionStep(V, 64, 2, 1, 64)
    gen = torch.Generator(device="cuda").manual_seed(5)
    ids = torch.randint(0, V, (sum(lens),), generator=gen, device="cuda")
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    table = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
    from paper_2411_12364_gb300 import norms, paged, vocab
    starts = torch.tensor([0, 33, 103], dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(n, device="cuda") for n in lens])
    seq = torch.repeat_interleave(torch.arange(2, device="cuda"), new.long())
    slots = (table[seq, pos // 16] * 16 + pos % 16).to(torch.int32)
    caches = [torch.zeros(10, 1, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dloss = torch.full((sum(lens),), 1.0 / sum(lens), device="cuda")

    def run():
        x = vocab.embedding(model.table, ids, scale=8.0)
        _, n = norms.block_norm(torch.zeros_like(x), x, w_pre=model.w_in, post=False)
        qkv = (n @ model.w_qkv.T).view(-1, 4, 64)
        paged.paged_append(*caches, qkv[:, 2:3], qkv[:, 3:], slots)
        out, lse = paged.paged_attention(qkv[:, :2], *caches, table, starts, new, 70, with_lse=True)
        y = out.view(-1, 128) @ model.w_o.T
        loss, row = vocab.cross_entropy(y, model.table, ids)
        dy, dtable = vocab.cross_entropy_backward(y, model.table, ids, row, dloss)
        dqkv = paged.paged_attention_backward(qkv[:, :2], qkv[:, 2:3], qkv[:, 3:], out, lse,
                                              (dy @ model.w_o).view(-1, 2, 64), starts)
        vocab.embedding_backward(ids, dy, V, dtable=dtable, accumulate=True)
        return (loss, dtable, *dqkv)

    run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        held = run()
    for _ in range(2):
        ids.copy_(torch.randint(0, V, (sum(lens),), generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        eager = run()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
    assert paged_check() == 0


def test_calls_at_once_on_two_streams(gpu_lib):
    """Calls that overlap on the GPU, each with its own workspace, give what they
    give one after another."""
    from paper_2411_12364_gb300 import paged, vocab
    gen = torch.Generator(device="cuda").manual_seed(9)

    def randn(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    sets = []
    for dtype, T, V, D in ((torch.bfloat16, 700, 3000, 256), (torch.float32, 200, 900, 100)):
        x, w = randn(T, D, dtype=dtype), randn(V, D, dtype=dtype) * 0.1
        ids = torch.randint(0, V, (T,), generator=gen, device="cuda")
        q, k = randn(T, 4, 64, dtype=dtype), randn(T, 2, 64, dtype=dtype)
        lse = torch.full((T, 4), 9.0, device="cuda")
        start = torch.tensor([0, T // 3, T], dtype=torch.int32, device="cuda")
        sets.append((x, w, ids, q, k, lse, start))

    def run(x, w, ids, q, k, lse, start):
        loss, row = vocab.cross_entropy(x, w, ids)
        dx, dw = vocab.cross_entropy_backward(x, w, ids, row, torch.ones_like(row))
        return (loss, dx, dw, vocab.embedding_backward(ids, x, w.shape[0]),
                *paged.paged_attention_backward(q, k, k, q, lse, q, start))

    alone = [run(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(run(*sets[i]))
    torch.cuda.synchronize()
    for i, want in enumerate(alone):
        for have in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(have, want))
    assert paged_check() == 0
