"""Cases of the operators that a decoder's training step needs at its ends and
in its attention: the embedding of token ids and its gradient, the softmax cross
entropy over a vocabulary (from hidden states and the output weights, without
keeping the logits) and its gradient, and the gradient of the attention of whole
sequences.

``run`` computes one pass, either in a plain form (elementary torch operations
in 32 bits) or, with ``own`` set, through the package's entry points.  Lengths
of sequences follow from the case alone; values, ids and labels from the
seed."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
IGNORED = -100            # the label of a token without a target


# ---- the cases -------------------------------------------------------------

def listed():
    return [
        # the ids of one decode step
        dict(name="embed_decode_64", op="embed", tokens=64, vocab=32000, dim=1024, dtype="bf16"),
        # the ids of a prefill chunk, from a large vocabulary
        dict(name="embed_prefill_16k", op="embed", tokens=16384, vocab=128000, dim=2048,
             dtype="bf16"),
        # a short batch in 32-bit storage, odd sizes
        dict(name="embed_grad_5003", op="embed_grad", tokens=5003, vocab=50021, dim=1000,
             dtype="f32"),
        # a training batch of 16384 tokens: few ids make up most of it
        dict(name="embed_grad_16k", op="embed_grad", tokens=16384, vocab=32000, dim=2048,
             dtype="bf16"),
        # scoring the last tokens of a step: few rows against the whole vocabulary
        dict(name="ce_64", op="ce", tokens=64, vocab=32000, dim=1024, logit_scale=1.0,
             dtype="bf16"),
        # the loss of a training batch
        dict(name="ce_16k", op="ce", tokens=16384, vocab=32000, dim=2048, logit_scale=1.0,
             dtype="bf16"),
        # a small batch in 32-bit storage, odd sizes, scaled logits
        dict(name="ce_grad_333", op="ce_grad", tokens=333, vocab=5003, dim=509, logit_scale=0.5,
             dtype="f32"),
        # a long vocabulary before a short batch
        dict(name="ce_grad_4k", op="ce_grad", tokens=4096, vocab=128000, dim=1024,
             logit_scale=1.0, dtype="bf16"),
        # the gradient of the loss of a training batch
        dict(name="ce_grad_16k", op="ce_grad", tokens=16384, vocab=32000, dim=2048,
             logit_scale=1.0, dtype="bf16"),
        # a few short sequences in 32-bit storage
        dict(name="attn_grad_short", op="attn_grad", seqs=5, len_lo=1, len_hi=300, q_heads=4,
             kv_heads=4, dim=80, dtype="f32"),
        # documents of ragged length packed into one batch
        dict(name="attn_grad_ragged", op="attn_grad", seqs=24, len_lo=1, len_hi=2048, q_heads=16,
             kv_heads=2, dim=64, dtype="bf16"),
        # a training batch of 4 sequences of 4096 tokens
        dict(name="attn_grad_4x4096", op="attn_grad", seqs=4, len_lo=4096, len_hi=4096,
             q_heads=16, kv_heads=4, dim=128, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dim(rng, lo, hi):
    d = _log(rng, lo, hi)
    return (d + 63) // 64 * 64 if rng.random() < 0.7 else d


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "ce", "ce_grad", "ce_grad", "attn_grad", "attn_grad"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op in ("embed", "embed_grad"):
        dim = _dim(rng, 64, 4096)
        entries = 1 << (25 if dtype == "bf16" else 24)
        return dict(op=op, tokens=_log(rng, 1, min(32768, entries // dim)),
                    vocab=_log(rng, 100, min(131072, 2 * entries // dim)), dim=dim, dtype=dtype)
    if op in ("ce", "ce_grad"):
        dim = _dim(rng, 64, 4096)
        most = (16384 * 32000 * 2048 >> (0 if dtype == "bf16" else 4)) // dim
        tokens = _log(rng, 1, 16384)
        vocab = _log(rng, 100, max(200, min(131072, most // tokens)))
        return dict(op=op, tokens=min(tokens, most // vocab), vocab=vocab, dim=dim,
                    logit_scale=rng.choice([1.0, 1.0, round(rng.uniform(0.1, 2.0), 3)]),
                    dtype=dtype)
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 5, 8])
    seqs, len_hi = _log(rng, 1, 64), _log(rng, 1, 4096)
    most = 1 << (30 if dtype == "bf16" else 26)
    while seqs * q_heads * len_hi * len_hi > most:
        seqs, len_hi = max(1, seqs // 2), max(1, len_hi * 4 // 5)
    return dict(op=op, seqs=seqs, len_lo=rng.choice([1, len_hi]), len_hi=len_hi, q_heads=q_heads,
                kv_heads=kv_heads, dim=rng.choice([64, 64, 128, 128, 80]), dtype=dtype)


def _lengths(case):
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    lens = [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(case["seqs"])]
    lens[0] = case["len_hi"]
    return lens


def work(case):
    op = case["op"]
    es = 2 if case["dtype"] == "bf16" else 4
    if op == "attn_grad":
        lens = _lengths(case)
        tokens, pairs = sum(lens), sum(n * (n + 1) // 2 for n in lens)
        hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
        # in: q, out, dout, k, v, the log-sum-exps; out: dq, dk, dv
        return {"bytes": tokens * d * es * (4 * hq + 4 * hk) + 4 * tokens * hq,
                "flops": 10 * hq * d * pairs}
    t, v, d = case["tokens"], case["vocab"], case["dim"]
    if op == "embed":
        return {"bytes": 2 * t * d * es + 8 * t, "flops": t * d}
    if op == "embed_grad":
        return {"bytes": (t + v) * d * es + 8 * t, "flops": t * d}
    if op == "ce":
        return {"bytes": (t + v) * d * es + 16 * t, "flops": 2 * t * v * d}
    return {"bytes": 2 * (t + v) * d * es + 16 * t, "flops": 6 * t * v * d}


# ---- the inputs ------------------------------------------------------------

def _tokens(n, vocab, gen):
    """Ids as text has them: the frequency falls as the inverse of the rank, and
    the ranks are spread over the vocabulary."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = 2.7 * torch.expm1(u * math.log1p(vocab / 2.7))     # density 1 / (rank + 2.7)
    return torch.randperm(vocab, generator=gen, device="cuda")[rank.long().clamp(max=vocab - 1)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    s, op, dt = dict(case), case["op"], DTYPES[case["dtype"]]
    if op == "attn_grad":
        lens = _lengths(case)
        t, hq, hk, d = sum(lens), case["q_heads"], case["kv_heads"], case["dim"]
        # queries, keys and values are slices of one projection's output
        qkv = randn(t, hq + 2 * hk, d).to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        s["dout"] = randn(t, hq, d).to(dt)
        starts = [0]
        for n in lens:
            starts.append(starts[-1] + n)
        s["starts"] = starts
        s["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["scale"] = 1.0 / math.sqrt(d)
        s["out"] = torch.empty(t, hq, d, dtype=dt, device="cuda")
        s["lse"] = torch.empty(t, hq, dtype=torch.float32, device="cuda")
        for a, b in zip(starts, starts[1:]):      # the forward pass that a step has done
            score = _scores(s, a, b)
            lse = torch.logsumexp(score, -1)      # [kv heads, group, rows]
            p = torch.exp(score - lse[..., None])
            out = torch.matmul(p, s["v"][a:b].float().transpose(0, 1)[:, None])
            s["out"][a:b] = out.permute(2, 0, 1, 3).reshape(b - a, hq, d).to(dt)
            s["lse"][a:b] = lse.permute(2, 0, 1).reshape(b - a, hq)
        return s
    t, v, d = case["tokens"], case["vocab"], case["dim"]
    if op == "embed":
        s["table"] = randn(v, d).mul_(0.02).to(dt)
        s["ids"] = _tokens(t, v, gen)
        s["scale"] = math.sqrt(d)
    elif op == "embed_grad":
        s["dout"] = randn(t, d).to(dt)
        s["ids"] = _tokens(t, v, gen)
        s["scale"] = math.sqrt(d)
    else:
        s["x"] = randn(t, d).to(dt)                               # normed hidden states
        s["w"] = randn(v, d).mul_(2.0 / math.sqrt(d)).to(dt)      # logits of deviation 2
        labels = _tokens(t, v, gen)
        padding = torch.rand(t, generator=gen, device="cuda") < 0.06
        s["labels"] = torch.where(padding, IGNORED, labels)
        if op == "ce_grad":
            s["lse"] = _cross_entropy(s)["lse"]
            # the mean over the tokens that count, with a weight of each
            weight = 0.5 + torch.rand(t, generator=gen, device="cuda")
            s["dloss"] = weight / max(1, int((~padding).sum()))
    return s


# ---- the plain forms -------------------------------------------------------

def _embed(s):
    ids = s["ids"]
    known = (ids >= 0) & (ids < s["vocab"])
    rows = s["table"][ids.clamp(0, s["vocab"] - 1)].float() * s["scale"]
    return {"out": torch.where(known[:, None], rows, 0.0).to(s["table"].dtype)}


def _embed_grad(s):
    total = torch.zeros(s["vocab"], s["dim"], device="cuda")
    total.index_add_(0, s["ids"], s["dout"].float())
    return {"dtable": total.mul_(s["scale"]).to(s["dout"].dtype)}


def _pieces(s):
    """Ranges of the vocabulary of at most 2^28 logits."""
    step = max(1, min(s["vocab"], (1 << 28) // s["tokens"]))
    return [(v, min(s["vocab"], v + step)) for v in range(0, s["vocab"], step)]


def _cross_entropy(s):
    x, labels = s["x"].float(), s["labels"]
    counts = (labels >= 0) & (labels < s["vocab"])
    top = torch.full((s["tokens"],), -math.inf, device="cuda")
    total = torch.zeros(s["tokens"], device="cuda")
    target = torch.zeros(s["tokens"], device="cuda")
    for lo, hi in _pieces(s):
        z = torch.matmul(x, s["w"][lo:hi].float().t()).mul_(s["logit_scale"])
        new = torch.maximum(top, z.amax(1))
        here = (labels >= lo) & (labels < hi)
        at = (labels - lo).clamp(0, hi - lo - 1)
        target += torch.where(here, z.gather(1, at[:, None])[:, 0], 0.0)
        total = total * torch.exp(top - new) + z.sub_(new[:, None]).exp_().sum(1)
        top = new
    lse = top + total.log()
    return {"loss": torch.where(counts, lse - target, 0.0), "lse": lse}


def _cross_entropy_grad(s):
    x, labels, dt = s["x"].float(), s["labels"], s["x"].dtype
    counts = (labels >= 0) & (labels < s["vocab"])
    g = torch.where(counts, s["dloss"], 0.0) * s["logit_scale"]
    dx = torch.zeros_like(x)
    dw = torch.empty_like(s["w"])
    rows = torch.arange(s["tokens"], device="cuda")
    for lo, hi in _pieces(s):
        w = s["w"][lo:hi].float()
        p = torch.matmul(x, w.t()).mul_(s["logit_scale"]).sub_(s["lse"][:, None]).exp_()
        here = (labels >= lo) & (labels < hi)
        p[rows, (labels - lo).clamp(0, hi - lo - 1)] -= here.float()
        p.mul_(g[:, None])
        dx += torch.matmul(p, w)
        dw[lo:hi] = torch.matmul(p.t(), x).to(dt)
    return {"dx": dx.to(dt), "dw": dw}


def _scores(s, a, b):
    """[kv heads, group, rows, keys] of the sequence of tokens a to b."""
    n, hk, d = b - a, s["kv_heads"], s["dim"]
    q = s["q"][a:b].float().reshape(n, hk, -1, d).permute(1, 2, 0, 3)
    k = s["k"][a:b].float().transpose(0, 1)[:, None]
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    at = torch.arange(n, device="cuda")
    return score.masked_fill_(at[None, :] > at[:, None], -math.inf)


def _attention_grad(s):
    hq, hk, d, dt = s["q_heads"], s["kv_heads"], s["dim"], s["q"].dtype
    t = s["starts"][-1]
    dq = torch.empty(t, hq, d, dtype=dt, device="cuda")
    dk = torch.empty(t, hk, d, dtype=dt, device="cuda")
    dv = torch.empty(t, hk, d, dtype=dt, device="cuda")
    for a, b in zip(s["starts"], s["starts"][1:]):
        n = b - a

        def heads(x):
            return x[a:b].float().reshape(n, hk, -1, d).permute(1, 2, 0, 3)

        q, dout, out = heads(s["q"]), heads(s["dout"]), heads(s["out"])
        k, v = heads(s["k"]), heads(s["v"])                       # [kv heads, 1, n, d]
        lse = s["lse"][a:b].reshape(n, hk, -1).permute(1, 2, 0)[..., None]
        p = _scores(s, a, b).sub_(lse).exp_()
        dv[a:b] = torch.matmul(p.transpose(2, 3), dout).sum(1).transpose(0, 1).to(dt)
        dp = torch.matmul(dout, v.transpose(2, 3))
        ds = p.mul_(dp.sub_((dout * out).sum(-1, keepdim=True))).mul_(s["scale"])
        dq[a:b] = torch.matmul(ds, k).permute(2, 0, 1, 3).reshape(n, hq, d).to(dt)
        dk[a:b] = torch.matmul(ds.transpose(2, 3), q).sum(1).transpose(0, 1).to(dt)
    return {"dq": dq, "dk": dk, "dv": dv}


# ---- one pass --------------------------------------------------------------

def run(s):
    op = s["op"]
    if not own:
        return {"embed": _embed, "embed_grad": _embed_grad, "ce": _cross_entropy,
                "ce_grad": _cross_entropy_grad, "attn_grad": _attention_grad}[op](s)
    if op == "embed":
        from paper_2411_12364_gb300.vocab import embedding
        return {"out": embedding(s["table"], s["ids"], scale=s["scale"])}
    if op == "embed_grad":
        from paper_2411_12364_gb300.vocab import embedding_backward
        return {"dtable": embedding_backward(s["ids"], s["dout"], s["vocab"], scale=s["scale"])}
    if op == "ce":
        from paper_2411_12364_gb300.vocab import cross_entropy
        loss, lse = cross_entropy(s["x"], s["w"], s["labels"], logit_scale=s["logit_scale"])
        return {"loss": loss, "lse": lse}
    if op == "ce_grad":
        from paper_2411_12364_gb300.vocab import cross_entropy_backward
        dx, dw = cross_entropy_backward(s["x"], s["w"], s["labels"], s["lse"], s["dloss"],
                                        logit_scale=s["logit_scale"])
        return {"dx": dx, "dw": dw}
    from paper_2411_12364_gb300.paged import paged_attention_backward
    dq, dk, dv = paged_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"],
                                          s["q_start"], scale=s["scale"])
    return {"dq": dq, "dk": dk, "dv": dv}


# ---- the definitions in 64 bits --------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        one = s["table"].double() * s["scale"]
        return {"out": one.index_select(0, s["ids"])}
    if op == "embed_grad":
        table = torch.zeros(s["vocab"], s["dim"], dtype=torch.float64, device="cuda")
        order = torch.argsort(s["ids"], stable=True)
        ids, counts = torch.unique_consecutive(s["ids"][order], return_counts=True)
        at = 0
        for i, n in zip(ids.tolist(), counts.tolist()):
            table[i] = s["dout"][order[at:at + n]].double().sum(0) * s["scale"]
            at += n
        return {"dtable": table}
    if op in ("ce", "ce_grad"):
        w = s["w"].double()
        valid = s["labels"] != IGNORED
        step = max(1, (1 << 27) // s["vocab"])        # rows at a time
        got = {"loss": [], "lse": []} if op == "ce" else {"dx": []}
        dw = torch.zeros_like(w) if op == "ce_grad" else None
        for r in range(0, s["tokens"], step):
            x = s["x"][r:r + step].double()
            ok, label = valid[r:r + step], s["labels"][r:r + step]
            z = (x @ w.T) * s["logit_scale"]
            if op == "ce":
                lse = torch.logsumexp(z, 1)
                pick = torch.take_along_dim(z, label.clamp(min=0)[:, None], 1).squeeze(1)
                got["lse"].append(lse)
                got["loss"].append((lse - pick) * ok)
                continue
            g = torch.exp(z - s["lse"][r:r + step, None].double())
            g -= torch.zeros_like(g).scatter_(1, label.clamp(min=0)[:, None], 1.0)
            g *= (s["logit_scale"] * s["dloss"][r:r + step].double() * ok)[:, None]
            got["dx"].append(g @ w)
            dw += g.T @ x
        got = {k: torch.cat(v) for k, v in got.items()}
        return got if dw is None else dict(got, dw=dw)
    group = s["q_heads"] // s["kv_heads"]
    q, k, v, out, dout, lse = (s[n].double() for n in ("q", "k", "v", "out", "dout", "lse"))
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a, b in zip(s["starts"], s["starts"][1:]):
        for h in range(s["q_heads"]):
            e = h // group
            z = torch.einsum("id,jd->ij", q[a:b, h], k[a:b, e]) * s["scale"]
            p = torch.tril(torch.exp(z - lse[a:b, h, None]))
            moved = torch.einsum("id,jd->ij", dout[a:b, h], v[a:b, e])
            mean = (dout[a:b, h] * out[a:b, h]).sum(1, keepdim=True)
            ds = p * (moved - mean)
            dq[a:b, h] = s["scale"] * (ds @ k[a:b, e])
            dk[a:b, e] += s["scale"] * (ds.T @ q[a:b, h])
            dv[a:b, e] += p.T @ dout[a:b, h]
    return {"dq": dq, "dk": dk, "dv": dv}
