"""Cases of the decoder-block operators: the paged key/value cache (page plan,
append, attention of new tokens over the pages) and the fused norms around a
block, forward and backward.

``run`` computes one pass, either in a plain form (elementary torch operations
in 32 bits) or, with ``own`` set, through the package's entry points.  Lengths
of the requests follow from the case alone; values and page orders from the
seed."""
import math
import random

import torch

own = False

EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases -------------------------------------------------------------

def listed():
    return [
        # one decode step of 64 requests: every request gets one token
        dict(name="plan_decode_64", op="plan", seqs=64, ctx_lo=511, ctx_hi=8191, new_lo=1,
             new_hi=1, page=16, short=False),
        # a batch that mixes decodes and short prompts, some idle requests among
        # them, with fewer free pages than they ask for
        dict(name="plan_mixed_2048", op="plan", seqs=2048, ctx_lo=0, ctx_hi=4095, new_lo=0,
             new_hi=32, page=16, short=True),
        # the keys and values of one decode step
        dict(name="append_decode_64", op="append", seqs=64, ctx_lo=511, ctx_hi=2047, new_lo=1,
             new_hi=1, q_heads=16, kv_heads=4, dim=128, page=16, dtype="bf16"),
        # those of a prefill chunk: 4 sequences of 4096 tokens
        dict(name="append_prefill_16k", op="append", seqs=4, ctx_lo=0, ctx_hi=0, new_lo=4096,
             new_hi=4096, q_heads=16, kv_heads=4, dim=128, page=64, dtype="bf16"),
        # a decode step of 64 requests with ragged contexts
        dict(name="attn_decode_64", op="attn", seqs=64, ctx_lo=511, ctx_hi=8191, new_lo=1,
             new_hi=1, q_heads=16, kv_heads=4, dim=128, page=16, dtype="bf16"),
        # one request deep into a long context: few rows, a long axis
        dict(name="attn_decode_long", op="attn", seqs=1, ctx_lo=131071, ctx_hi=131071, new_lo=1,
             new_hi=1, q_heads=16, kv_heads=4, dim=128, page=64, dtype="bf16"),
        # whole prompts: 4 sequences of 4096 tokens, nothing cached before them
        dict(name="attn_prefill_4x4096", op="attn", seqs=4, ctx_lo=0, ctx_hi=0, new_lo=4096,
             new_hi=4096, q_heads=16, kv_heads=4, dim=128, page=64, dtype="bf16"),
        # chunked prefill beside decodes: ragged chunks over ragged contexts
        dict(name="attn_chunks_ragged", op="attn", seqs=8, ctx_lo=1000, ctx_hi=30000, new_lo=1,
             new_hi=1024, q_heads=16, kv_heads=2, dim=64, page=16, dtype="bf16"),
        # between two blocks of a decode step
        dict(name="norm_decode_64", op="norm", tokens=64, dim=1024, kind="rms", gate="channel",
             dtype="bf16"),
        # between two blocks of a prefill chunk, with a gate of its own per entry
        dict(name="norm_prefill_16k", op="norm", tokens=16384, dim=2048, kind="rms", gate="full",
             dtype="bf16"),
        # gradients of a short training batch in 32-bit storage, one gate a token
        dict(name="grad_1000x1000", op="grad", tokens=1000, dim=1000, kind="layer", gate="token",
             dtype="f32"),
        # gradients of a training batch of 16384 tokens
        dict(name="grad_16k", op="grad", tokens=16384, dim=2048, kind="rms", gate="channel",
             dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attn", "attn", "norm", "grad"])
    if op == "plan":
        new_hi = _log(rng, 1, 512)
        seqs = _log(rng, 1, min(4096, 65536 // new_hi))
        return dict(op=op, seqs=seqs, ctx_lo=0, ctx_hi=_log(rng, 1, 16384),
                    new_lo=rng.choice([0, 1]), new_hi=new_hi, page=rng.choice([16, 32, 64, 128]),
                    short=rng.random() < 0.3)
    if op in ("norm", "grad"):
        dim = _log(rng, 64, 8192)
        if rng.random() < 0.7:
            dim = (dim + 63) // 64 * 64
        if dim == 3072:
            dim = 3008
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        entries = 16384 * 2048 // (1 if dtype == "bf16" else 2)
        return dict(op=op, tokens=_log(rng, 1, min(16384, entries // dim)), dim=dim,
                    kind=rng.choice(["rms", "layer"]),
                    gate=rng.choice(["none", "channel", "token", "full"]), dtype=dtype)
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = dict(q_heads=kv_heads * rng.choice([1, 2, 4, 5, 8]), kv_heads=kv_heads,
                 dim=rng.choice([64, 64, 128, 128, 80]), page=rng.choice([16, 32, 64, 128]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "append":
        new_hi = rng.choice([1, _log(rng, 2, 4096)])
        return dict(op=op, seqs=_log(rng, 1, max(1, min(256, 16384 // new_hi))), ctx_lo=0,
                    ctx_hi=_log(rng, 1, 2048), new_lo=1, new_hi=new_hi, dtype=dtype, **heads)
    rows = 8192 if dtype == "bf16" else 512   # most rows (tokens of a request x query heads)
    new_hi = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, rows // heads["q_heads"]))
    seqs = _log(rng, 1, 64)
    ctx_hi = _log(rng, 1, 65536)
    while seqs * heads["q_heads"] * new_hi * (ctx_hi + new_hi) > 1 << 30 or \
            seqs * kv_heads * (ctx_hi + new_hi) > 1 << 21:
        seqs, ctx_hi = max(1, seqs // 2), max(1, ctx_hi * 2 // 3)
        if seqs == 1:
            new_hi = max(1, new_hi * 2 // 3)
    return dict(op=op, seqs=seqs, ctx_lo=ctx_hi // 8, ctx_hi=ctx_hi, new_lo=1, new_hi=new_hi,
                dtype=dtype, **heads)


def _lengths(case):
    """(context, new tokens) of each request, from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    ctx = [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    new[0] = max(1, case["new_hi"])
    return ctx, new


def _ceil(a, b):
    return (a + b - 1) // b


def work(case):
    op = case["op"]
    es = 2 if case.get("dtype") == "bf16" else 4
    if op in ("norm", "grad"):
        t, d = case["tokens"], case["dim"]
        n = {"none": 0, "channel": 0, "token": t, "full": t * d}[case["gate"]]
        if op == "norm":
            return {"bytes": es * (4 * t * d + n), "flops": 12 * t * d}
        return {"bytes": es * (6 * t * d + 2 * n) + 16 * d, "flops": 30 * t * d}
    ctx, new = _lengths(case)
    tokens, page = sum(new), case["page"]
    if op == "plan":
        pages = sum(_ceil(c + n, page) - _ceil(c, page) for c, n in zip(ctx, new))
        return {"bytes": 16 * case["seqs"] + 4 * tokens + 8 * pages, "flops": 0}
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    if op == "append":
        return {"bytes": 4 * tokens * hk * d * es + 4 * tokens, "flops": 0}
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))
    cached = sum(c + n for c, n in zip(ctx, new))
    pages = sum(_ceil(c + n, page) for c, n in zip(ctx, new))
    return {"bytes": 2 * tokens * hq * d * es + 2 * cached * hk * d * es + 4 * pages
            + 4 * tokens * hq, "flops": 4 * hq * d * pairs}


# ---- the inputs ------------------------------------------------------------

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    s = dict(case)
    if case["op"] in ("norm", "grad"):
        t, d, dt = case["tokens"], case["dim"], DTYPES[case["dtype"]]
        s["y"] = randn(t, d).mul_(1.5).to(dt)          # a block's output
        s["r"] = randn(t, d).mul_(4.0).to(dt)          # the residual stream
        s["w_post"], s["w_pre"] = 1 + 0.1 * randn(d), 1 + 0.1 * randn(d)
        layer = case["kind"] == "layer"
        s["b_post"] = 0.1 * randn(d) if layer else None
        s["b_pre"] = 0.1 * randn(d) if layer else None
        s["gate"] = {"none": lambda: None, "channel": lambda: 0.5 + 0.1 * randn(d),
                     "token": lambda: torch.sigmoid(randn(t, 1)).to(dt),
                     "full": lambda: torch.sigmoid(randn(t, d)).to(dt)}[case["gate"]]()
        s["res_scale"], s["out_scale"] = 0.9, 0.5
        if case["op"] == "grad":
            s["u"] = s.pop("r")
            s["du"], s["dn"] = randn(t, d).to(dt), randn(t, d).to(dt)
        return s

    ctx, new = _lengths(case)
    page = case["page"]
    tokens = sum(new)
    old_pages = [_ceil(c, page) for c in ctx]
    all_pages = [_ceil(c + n, page) for c, n in zip(ctx, new)]
    width = max(all_pages) + 1
    n_pages = sum(all_pages) + 7
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    s["ctx"], s["new"] = _ints(ctx), _ints(new)
    s["tokens"], s["max_new"] = tokens, max(new)
    if case["op"] == "plan":
        # pages of the contexts are in the table, the others on the free list
        held = sum(old_pages)
        want = n_pages - 7 - held
        free = want // 2 if case["short"] else want + 7
        s["table"] = _table(order, old_pages, width)
        s["free_pages"] = order[held:].contiguous()
        s["free"] = _ints([free])
        return s
    dt = DTYPES[case["dtype"]]
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    s["k_cache"] = torch.empty(n_pages, hk, page, d, dtype=dt, device="cuda").normal_(generator=gen)
    s["v_cache"] = torch.empty(n_pages, hk, page, d, dtype=dt, device="cuda").normal_(generator=gen)
    s["table"] = _table(order, all_pages, width)
    # queries, keys and values are slices of one projection's output
    qkv = randn(tokens, hq + 2 * hk, d).to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    s["q_start"] = _ints([0] + torch.tensor(new).cumsum(0).tolist())
    s["kv_lens"] = s["ctx"] + s["new"]
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), s["new"].long())
    pos = s["ctx"][seq] + torch.arange(tokens, device="cuda") - s["q_start"][seq]
    s["slots"] = (s["table"][seq, pos // page] * page + pos % page).to(torch.int32)
    s["scale"] = 1.0 / math.sqrt(d)
    return s


def _table(order, pages, width):
    """The block table: request r's pages in order, -1 past them."""
    n = _ints(pages)[:, None]
    col = torch.arange(width, device="cuda")[None, :]
    at = (torch.cumsum(n, 0) - n) + col
    return torch.where(col < n, order[at.clamp(max=order.numel() - 1)], -1).to(torch.int32)


# ---- the plain forms -------------------------------------------------------

def _plan(s):
    page, ctx, new, table = s["page"], s["ctx"].long(), s["new"].long(), s["table"]
    free = s["free"].long()
    old, full = (ctx + page - 1) // page, (ctx + new + page - 1) // page
    fits = full <= table.shape[1]
    need = torch.where(fits, full - old, 0)
    upto = torch.cumsum(need, 0)
    granted = fits & ((need == 0) | (upto <= free))
    taken = torch.where(granted, upto, 0).amax()
    q_start = torch.cumsum(torch.cat([new.new_zeros(1), new]), 0)
    # page k of the call's new ones comes from the end of the free list
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    fresh = granted[:, None] & (col >= old[:, None]) & (col < full[:, None])
    at = free - 1 - ((upto - need - old)[:, None] + col)
    pages = s["free_pages"][at.clamp(0, s["free_pages"].numel() - 1)]
    table.copy_(torch.where(fresh, pages, table))
    seq = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new,
                                  output_size=s["tokens"])
    pos = ctx[seq] + torch.arange(s["tokens"], device="cuda") - q_start[seq]
    at = (pos // page).clamp(max=table.shape[1] - 1)
    slots = torch.where(granted[seq], table[seq, at] * page + pos % page, -1)
    return {"table": table, "q_start": q_start.to(torch.int32),
            "kv_lens": torch.where(granted, ctx + new, 0).to(torch.int32),
            "slots": slots.to(torch.int32), "free": (free - taken).to(torch.int32)}


def _append(s):
    page, off = s["slots"] // s["page"], s["slots"] % s["page"]
    s["k_cache"][page, :, off] = s["k"]
    s["v_cache"][page, :, off] = s["v"]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend(s):
    """Every request padded to the longest: [requests, kv heads, rows, keys]."""
    hk, d, n = s["kv_heads"], s["dim"], s["max_new"]
    group = s["q_heads"] // hk
    new, kv = s["new"].long(), s["kv_lens"].long()
    width = s["table"].shape[1] - 1
    keys = width * s["page"]
    pages = s["table"][:, :width].clamp(min=0).long()
    k = s["k_cache"][pages].float().transpose(2, 3).reshape(-1, keys, hk, d)
    v = s["v_cache"][pages].float().transpose(2, 3).reshape(-1, keys, hk, d)
    i = torch.arange(n, device="cuda")
    at = (s["q_start"][:-1].long()[:, None] + i).clamp(max=s["tokens"] - 1)
    q = s["q"][at].float().reshape(-1, n, hk, group, d).permute(0, 2, 1, 3, 4)
    q = q.reshape(-1, hk, n * group, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(s["scale"])
    pos = (kv - new)[:, None] + i                                       # [requests, n]
    hidden = torch.arange(keys, device="cuda") > pos[:, :, None]        # [requests, n, keys]
    score.view(-1, hk, n, group, keys).masked_fill_(hidden[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v.permute(0, 2, 1, 3)).div_(total)
    lse = (top + total.log()).reshape(-1, hk, n, group)
    seq = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new,
                                  output_size=s["tokens"])
    row = torch.arange(s["tokens"], device="cuda") - s["q_start"][seq]
    out = out.view(-1, hk, n, group, d)[seq, :, row].reshape(-1, s["q_heads"], d)
    return {"out": out.to(s["q"].dtype), "lse": lse[seq, :, row].reshape(-1, s["q_heads"])}


def _hat(x, kind):
    """The normalised rows and the reciprocal deviation."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * rstd, rstd


def _norm(s):
    dt = s["y"].dtype
    z = _hat(s["y"].float(), s["kind"])[0] * s["w_post"]
    if s["b_post"] is not None:
        z = z + s["b_post"]
    if s["gate"] is not None:
        z = z * s["gate"].float()
    u = s["res_scale"] * s["r"].float() + s["out_scale"] * z
    n = _hat(u, s["kind"])[0] * s["w_pre"]
    if s["b_pre"] is not None:
        n = n + s["b_pre"]
    return {"u": u.to(dt), "n": n.to(dt)}


def _norm_back(g, hat, rstd, w, kind):
    wg = g * w
    dx = wg - hat * (wg * hat).mean(-1, keepdim=True)
    if kind == "layer":
        dx = dx - wg.mean(-1, keepdim=True)
    return dx * rstd


def _grad(s):
    dt, kind = s["y"].dtype, s["kind"]
    dn, gate = s["dn"].float(), 1.0 if s["gate"] is None else s["gate"].float()
    u_hat, u_rstd = _hat(s["u"].float(), kind)
    y_hat, y_rstd = _hat(s["y"].float(), kind)
    gu = s["du"].float() + _norm_back(dn, u_hat, u_rstd, s["w_pre"], kind)
    gz = s["out_scale"] * gate * gu
    got = {"dy": _norm_back(gz, y_hat, y_rstd, s["w_post"], kind).to(dt),
           "dr": (s["res_scale"] * gu).to(dt), "dw_post": (gz * y_hat).sum(0),
           "dw_pre": (dn * u_hat).sum(0)}
    if s["b_post"] is not None:
        got["db_post"], got["db_pre"] = gz.sum(0), dn.sum(0)
    if s["gate"] is not None:
        z = y_hat * s["w_post"] + (0.0 if s["b_post"] is None else s["b_post"])
        dgate = s["out_scale"] * z * gu
        if s["gate"].dim() == 1:
            got["dgate"] = dgate.sum(0)
        elif s["gate"].shape[1] == 1:
            got["dgate"] = dgate.sum(1, keepdim=True).to(dt)
        else:
            got["dgate"] = dgate.to(dt)
    return got


# ---- one pass --------------------------------------------------------------

def run(s):
    op = s["op"]
    if not own:
        return {"plan": _plan, "append": _append, "attn": _attend, "norm": _norm,
                "grad": _grad}[op](s)
    if op == "plan":
        from paper_2411_12364_gb300.paged import paged_plan
        q_start, kv_lens, slots, free = paged_plan(
            s["ctx"], s["new"], s["table"], s["free_pages"], s["free"], s["page"], s["tokens"])
        return {"table": s["table"], "q_start": q_start, "kv_lens": kv_lens, "slots": slots,
                "free": free}
    if op == "append":
        from paper_2411_12364_gb300.paged import paged_append
        paged_append(s["k_cache"], s["v_cache"], s["k"], s["v"], s["slots"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if op == "attn":
        from paper_2411_12364_gb300.paged import paged_attention
        out, lse = paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["q_start"],
                                   s["kv_lens"], s["max_new"], scale=s["scale"], with_lse=True)
        return {"out": out, "lse": lse}
    if op == "norm":
        from paper_2411_12364_gb300.norms import block_norm
        u, n = block_norm(s["y"], s["r"], w_post=s["w_post"], b_post=s["b_post"], gate=s["gate"],
                          w_pre=s["w_pre"], b_pre=s["b_pre"], kind=s["kind"], eps=EPS,
                          res_scale=s["res_scale"], out_scale=s["out_scale"])
        return {"u": u, "n": n}
    from paper_2411_12364_gb300.norms import block_norm_backward
    got = block_norm_backward(s["y"], s["u"], s["du"], s["dn"], w_post=s["w_post"],
                              b_post=s["b_post"], gate=s["gate"], w_pre=s["w_pre"],
                              b_pre=s["b_pre"], kind=s["kind"], eps=EPS,
                              res_scale=s["res_scale"], out_scale=s["out_scale"])
    return {k: v for k, v in got.items() if v is not None}


# ---- the definitions in 64 bits --------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "plan":
        return None
    if op == "append":
        got = {}
        for name in ("k", "v"):
            cache = s[name + "_cache"].double()
            flat = cache.transpose(1, 2).reshape(-1, *cache.shape[1::2])   # [slots, heads, dim]
            flat.index_copy_(0, s["slots"].long(), s[name].double())
            got[name + "_cache"] = flat.view(cache.shape[0], cache.shape[2], cache.shape[1],
                                             cache.shape[3]).transpose(1, 2).contiguous()
        return got
    if op == "attn":
        hq, hk, d = s["q_heads"], s["kv_heads"], s["dim"]
        out = torch.empty(s["tokens"], hq, d, dtype=torch.float64, device="cuda")
        lse = torch.empty(s["tokens"], hq, dtype=torch.float64, device="cuda")
        start, kv = s["q_start"].tolist(), s["kv_lens"].tolist()
        for r, length in enumerate(kv):
            pages = s["table"][r, :_ceil(length, s["page"])].long()
            k, v = (s[c][pages].transpose(0, 1).reshape(hk, -1, d)[:, :length].double()
                    for c in ("k_cache", "v_cache"))
            n = start[r + 1] - start[r]
            for h in range(hq):
                for i0 in range(0, n, 512):
                    i1 = min(n, i0 + 512)
                    score = s["q"][start[r] + i0:start[r] + i1, h].double() @ k[h * hk // hq].T
                    seen = torch.ones(i1 - i0, length, device="cuda").tril(length - n + i0) > 0
                    score = torch.where(seen, score * s["scale"], -math.inf)
                    out[start[r] + i0:start[r] + i1, h] = torch.softmax(score, -1) @ v[h * hk // hq]
                    lse[start[r] + i0:start[r] + i1, h] = torch.logsumexp(score, -1)
        return {"out": out, "lse": lse}
    f = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in s.items()}

    def norm(x, w, b):
        if s["kind"] == "layer":
            return torch.nn.functional.layer_norm(x, x.shape[-1:], w, b, EPS)
        return x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w

    def add(z):
        return f["out_scale"] * (z if f["gate"] is None else f["gate"] * z)

    if op == "norm":
        u = f["res_scale"] * f["r"] + add(norm(f["y"], f["w_post"], f["b_post"]))
        return {"u": u, "n": norm(u, f["w_pre"], f["b_pre"])}
    leaves = {k: f[k].requires_grad_() for k in ("y", "u", "w_post", "b_post", "w_pre", "b_pre",
                                                 "gate") if f[k] is not None}
    n = norm(f["u"], f["w_pre"], f["b_pre"])
    n.backward(f["dn"])
    gu = f["du"] + f["u"].grad
    add(norm(f["y"], f["w_post"], f["b_post"])).backward(gu)
    got = {"dy": f["y"].grad, "dr": f["res_scale"] * gu}
    got.update({"d" + k: v.grad for k, v in leaves.items() if k not in ("y", "u")})
    return {k: v.detach() for k, v in got.items()}
