"""The paged key/value cache on the GPU: the page plan against a loop over
requests, the append against indexing, and the attention against a 64-bit
softmax over the gathered pages, at the lengths, head groups, widths, page
sizes and strides where the kernels change path."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2411_12364_gb300 import binding
from paper_2411_12364_gb300.paged import paged_append, paged_attention, paged_plan

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24    # rounding of one fp32 operation
EPS16 = 2.0 ** -8     # rounding to bf16 (8 bits of significand)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- plan ------------------------------------------------------------------

def plan_reference(ctx, new, table, free_pages, free, page, n_tokens):
    """Request by request, as a scheduler would."""
    table = table.copy()
    q_start, kv, slots = [0], [], []
    upto = taken = asked = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        c, n = max(0, c), max(0, n)
        old, full = -(-c // page), -(-(c + n) // page)
        fits = full <= table.shape[1]
        need = full - old if fits else 0
        upto += need
        ok = fits and (need == 0 or upto <= free) and q_start[-1] + n <= n_tokens
        if ok:
            for k in range(need):
                table[r, old + k] = free_pages[free - 1 - (upto - need + k)]
            taken = upto if need else taken
            asked = upto
        kv.append(c + n if ok else 0)
        for p in range(c, c + n):
            slots.append(int(table[r, p // page]) * page + p % page if ok else -1)
        q_start.append(q_start[-1] + n)
    slots = (slots + [-1] * n_tokens)[:n_tokens]
    return table, q_start, kv, slots, free - taken, free - asked


def _check_plan(ctx, new, width, page, free, n_free, n_tokens=None, seed=0):
    rng = np.random.default_rng(seed)
    R = len(ctx)
    table = rng.integers(0, 50, (R, width)).astype(np.int32)
    pages = rng.permutation(n_free).astype(np.int32) + 50
    n_tokens = sum(max(0, n) for n in new) if n_tokens is None else n_tokens
    want = plan_reference(ctx, new, table, pages, free, page, n_tokens)
    dev = torch.from_numpy(table).cuda()
    args = (_i32(ctx), _i32(new), dev, torch.from_numpy(pages).cuda(), _i32([free]), page, n_tokens)
    for _ in range(2):   # the call may be repeated
        left = _i32([-7])
        q_start, kv, slots, balance = paged_plan(*args, free_left=left)
        assert np.array_equal(dev.cpu().numpy(), want[0])
        assert q_start.tolist() == want[1]
        assert kv.tolist() == want[2]
        assert slots.tolist() == want[3]
        assert left.item() == want[4] and balance.item() == want[5]
        assert paged_plan(*args)[3].item() == want[5]


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("R", [1, 7, 256, 257, 1025, 2500])
def test_plan_matches_a_loop(page, R, gpu_lib):
    rng = np.random.default_rng(R + page)
    ctx = rng.integers(0, 700, R).tolist()
    new = rng.integers(0, 40, R).tolist()
    ctx[0] = page            # a context that ends at a page's end
    need = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(ctx, new))
    _check_plan(ctx, new, 760 // page + 2, page, need + 3, need + 3)


def test_plan_refuses_what_does_not_fit(gpu_lib):
    # too few free pages from the second request on; the last needs none
    _check_plan([0, 30, 5, 40], [40, 40, 100, 3], 9, 16, 4, 8)
    # a row that is too narrow takes no page from the others
    _check_plan([0, 0, 0], [64, 17, 16], 2, 16, 3, 3)
    # no free page, no table at all
    _check_plan([16, 0, 15], [1, 0, 1], 2, 16, 0, 1)
    # tokens past the capacity
    _check_plan([3, 0, 9], [10, 10, 2], 4, 16, 9, 9, n_tokens=15)
    # more capacity than tokens
    _check_plan([3, 0, 9], [10, 10, 2], 4, 16, 9, 9, n_tokens=40)


def test_plan_counts_no_more_pages_than_the_list_has(gpu_lib):
    args = (_i32([0, 0]), _i32([40, 40]))
    pages = _i32([7, 8, 9, 4])
    out = []
    for free in (4, 5, 1 << 30):
        table, left = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), _i32([0])
        q_start, kv, slots, balance = paged_plan(*args, table, pages, _i32([free]), 16, 80, left)
        out.append([x.tolist() for x in (table, left, q_start, kv, slots, balance)])
    assert out[0][0] == [[4, 9, 8, -1], [-1] * 4] and out[0][1] == [1] and out[0][3] == [40, 0]
    assert out[1] == out[0] and out[2] == out[0]


def test_plan_of_idle_negative_and_long_requests(gpu_lib):
    _check_plan([0, 5, 0], [0, 0, 0], 3, 16, 2, 2, n_tokens=0)
    _check_plan([-3, 7, 4], [5, -2, 1], 3, 16, 4, 4)
    _check_plan([100000], [5000], 105000 // 16 + 1, 16, 400, 400)
    left = _i32([9])
    empty = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    q_start, kv, slots, _ = paged_plan(_i32([]), _i32([]), empty, _i32([1, 2]), _i32([2]), 16, 3,
                                       free_left=left)
    assert q_start.tolist() == [0] and kv.numel() == 0
    assert slots.tolist() == [-1] * 3 and left.item() == 2


# ---- append ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,dim,page", [(4, 128, 16), (1, 8, 32), (3, 80, 64), (8, 64, 256)])
@pytest.mark.parametrize("layout", ["packed", "qkv", "misaligned", "transposed"])
def test_append_writes_each_slot_once(dtype, heads, dim, page, layout, gpu_lib):
    gen = torch.Generator().manual_seed(3)
    T, pages = 77, 7 + 200 // page
    kc = torch.randn(pages, heads, page, dim, generator=gen).to(dtype).cuda()
    vc = torch.randn(pages, heads, page, dim, generator=gen).to(dtype).cuda()
    slots = torch.randperm(pages * page, generator=gen)[:T].to(torch.int32)
    slots[5], slots[11] = -1, pages * page    # refused, and outside the cache
    qkv = torch.randn(T, 3 * heads * dim + 1, generator=gen).to(dtype).cuda()
    if layout == "packed":
        k, v = (qkv[:, i * heads * dim:(i + 1) * heads * dim].reshape(T, heads, dim)
                for i in (0, 1))
    elif layout == "qkv":
        flat = qkv[:, :-1].contiguous().view(T, 3 * heads, dim)
        k, v = flat[:, heads:2 * heads], flat[:, 2 * heads:]
    elif layout == "misaligned":
        k, v = (qkv[:, 1 + i * heads * dim:1 + (i + 1) * heads * dim].unflatten(1, (heads, dim))
                for i in (0, 1))
    else:
        k, v = (qkv[:, i * heads * dim:(i + 1) * heads * dim].reshape(T, dim, heads)
                .transpose(1, 2) for i in (0, 1))
    want_k, want_v = kc.cpu().clone(), vc.cpu().clone()
    for t in range(T):
        s = int(slots[t])
        if 0 <= s < pages * page:
            want_k[s // page, :, s % page] = k[t].cpu()
            want_v[s // page, :, s % page] = v[t].cpu()
    paged_append(kc, vc, k, v, slots.cuda())
    assert torch.equal(kc.cpu(), want_k) and torch.equal(vc.cpu(), want_v)


# ---- attention -------------------------------------------------------------

class Case:
    """Caches, tables and queries of requests (kv length, new tokens); the
    pages' places past a request's length hold NaN, and so do unused pages."""

    def __init__(self, reqs, hq, hk, dim, page, dtype, seed=0, peak=1.0, qkv=True, spare=3):
        gen = torch.Generator().manual_seed(seed)
        n_pages = [max(0, -(-kv // page)) for kv, _ in reqs]
        total = sum(n_pages) + spare
        self.page, self.dtype, self.reqs, self.hq, self.hk, self.dim = page, dtype, reqs, hq, hk, dim
        order = torch.randperm(total, generator=gen)
        width = max(n_pages) + 1
        table = torch.full((len(reqs), width), -1, dtype=torch.int32)
        nan = float("nan")
        self.k = torch.full((total, hk, page, dim), nan).to(dtype)
        self.v = torch.full((total, hk, page, dim), nan).to(dtype)
        self.keys, self.values = [], []
        at = 0
        for r, (kv, _) in enumerate(reqs):
            kk = torch.randn(hk, kv, dim, generator=gen).to(dtype)
            vv = torch.randn(hk, kv, dim, generator=gen).to(dtype)
            for i in range(n_pages[r]):
                p = int(order[at])
                at += 1
                table[r, i] = p
                n = min(page, kv - i * page)
                self.k[p, :, :n] = kk[:, i * page:i * page + n]
                self.v[p, :, :n] = vv[:, i * page:i * page + n]
            self.keys.append(kk)
            self.values.append(vv)
        self.k, self.v, self.table = self.k.cuda(), self.v.cuda(), table.cuda()
        self.start = [0]
        for _, n in reqs:
            self.start.append(self.start[-1] + n)
        T = self.start[-1]
        q = (peak * torch.randn(T, hq + (2 * hk if qkv else 0), dim, generator=gen)).to(dtype).cuda()
        self.q = q[:, :hq]
        self.max_new = max(n for _, n in reqs)

    def run(self, **kw):
        return paged_attention(self.q, self.k, self.v, self.table, _i32(self.start),
                               _i32([kv for kv, _ in self.reqs]), kw.pop("max_new", self.max_new),
                               with_lse=True, **kw)

    def check(self, out, lse, scale=None):
        """Bounds from the arithmetic, per entry.  B bounds a score's sum of
        products, A is the weighted sum of |v|: a score is off by at most
        (D + 4) eps32 B, which moves every weight by twice that; the weights'
        sum and the output's add up at most kv + 16 roundings, exp2 and the
        final division 2^-20; bf16 adds a rounding of each weight and of the
        output."""
        scale = 1 / math.sqrt(self.dim) if scale is None else scale
        group = self.hq // self.hk
        out, lse = out.cpu().double(), lse.cpu().double()
        assert out.shape == (self.start[-1], self.hq, self.dim)
        for r, (kv, n) in enumerate(self.reqs):
            q = self.q[self.start[r]:self.start[r + 1]].cpu().double()
            k = self.keys[r].double().repeat_interleave(group, 0)
            v = self.values[r].double().repeat_interleave(group, 0)
            s = torch.einsum("nhd,hkd->nhk", q, k) * scale
            seen = torch.arange(kv)[None, :] <= (kv - n + torch.arange(n))[:, None]
            s = s.masked_fill(~seen[:, None, :], -math.inf)
            bound = (torch.einsum("nhd,hkd->nhk", q.abs(), k.abs()) * scale
                     * seen[:, None, :]).amax(-1, keepdim=True) if kv else torch.zeros(n, self.hq, 1)
            got, got_l = out[self.start[r]:self.start[r + 1]], lse[self.start[r]:self.start[r + 1]]
            empty = ~seen.any(-1) if kv else torch.ones(n, dtype=torch.bool)
            assert (got[empty] == 0).all() and (got_l[empty] == -math.inf).all()
            live = ~empty
            if not live.any():
                continue
            p = torch.softmax(s[live], -1)
            want = torch.einsum("nhk,hkd->nhd", p, v)
            a = torch.einsum("nhk,hkd->nhd", p, v.abs())
            moved = 2 * (self.dim + 4) * EPS32 * bound[live] + (kv + 16) * EPS32 + 2.0 ** -20
            tol = a * moved + 1e-30
            if self.dtype == torch.bfloat16:
                tol = tol + EPS16 * (a + want.abs() + tol)
            err = (got[live] - want).abs()
            assert (err <= tol).all(), f"request {r}: {(err / tol).max():.2f} of the bound"
            want_l = torch.logsumexp(s[live], -1)
            tol_l = moved[..., 0] + 2.0 ** -20 * want_l.abs()
            err_l = (got_l[live] - want_l).abs()
            assert (err_l <= tol_l).all(), f"lse of request {r}: {(err_l / tol_l).max():.2f}"


BF16, F32 = torch.bfloat16, torch.float32

DECODE = [(1, 1), (15, 1), (16, 1), (17, 1), (64, 1), (65, 1), (700, 1), (1301, 1), (127, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,dim,page", [(16, 4, 128, 16), (8, 8, 64, 32), (5, 1, 80, 64),
                                            (32, 2, 128, 128), (6, 2, 40, 256), (2, 1, 8, 16),
                                            (40, 1, 128, 16), (4, 1, 192, 32), (9, 3, 256, 64)])
def test_decode_matches_64_bits(dtype, hq, hk, dim, page, gpu_lib):
    c = Case(DECODE, hq, hk, dim, page, dtype)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,dim,page", [(8, 2, 128, 16), (4, 4, 64, 64), (6, 2, 80, 32),
                                            (10, 2, 128, 128), (2, 2, 72, 256), (64, 1, 64, 16),
                                            (7, 1, 128, 64), (2, 1, 200, 16)])
def test_chunks_match_64_bits(dtype, hq, hk, dim, page, gpu_lib):
    reqs = [(300, 37), (1, 1), (129, 129), (128, 128), (640, 1), (257, 200), (500, 3), (64, 64),
            (131, 130)]
    c = Case(reqs, hq, hk, dim, page, dtype, seed=1)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("reqs", [
    [(0, 3), (5, 5), (0, 1)],             # rows without a key
    [(3, 7), (200, 300), (40, 9)],        # first rows of a request see nothing
    [(50, 0), (60, 2), (70, 0), (1, 0)],  # requests without rows
    [(1, 1)],
], ids=["empty", "short", "idle", "one"])
def test_rows_without_keys(dtype, reqs, gpu_lib):
    c = Case(reqs, 8, 2, 128, 16, dtype, seed=2)
    c.check(*c.run())
    c.check(*c.run(max_new=400))          # the kernel that a longer chunk takes


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv,n,page", [(20000, 1, 16), (20011, 2, 64), (9001, 150, 128)])
def test_long_axis_is_split_and_joined(dtype, kv, n, page, gpu_lib):
    c = Case([(kv, n)], 4, 1, 128, page, dtype, seed=4, peak=2.0)
    out, lse = c.run()
    c.check(out, lse)
    again = c.run()                       # the join's order is fixed
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype,dim", [(BF16, 64), (BF16, 128), (BF16, 192), (F32, 128), (F32, 256)])
@pytest.mark.parametrize("reqs", [[(20011, 29)], [(15000, 150), (40, 3)],
                                  [(3000 + 77 * i, 20 + 9 * i) for i in range(12)]],
                         ids=["one", "two", "several"])
def test_tall_tiles_in_many_or_few_shares(dtype, dim, reqs, gpu_lib):
    """17 and more rows a tile: many partials each, and few."""
    c = Case(reqs, 10, 2, dim, 32, dtype, seed=14, peak=2.0)
    out, lse = c.run()
    c.check(out, lse)
    again = c.run()                       # the join's order is fixed
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    c.check(*c.run(max_new=2))            # less than there is


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_requests_and_peaked_scores(dtype, gpu_lib):
    rng = np.random.default_rng(5)
    reqs = [(int(kv), 1) for kv in rng.integers(1, 300, 600)]
    c = Case(reqs, 8, 2, 64, 16, dtype, seed=5, peak=12.0)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,n", [(8, 4), (8, 5), (16, 4), (16, 8), (16, 9), (2, 16), (2, 17),
                                  (64, 1), (32, 2)])
def test_few_rows_a_request(dtype, hq, n, gpu_lib):
    """Around the row counts where another kernel takes over."""
    c = Case([(333, n), (n, n), (70, max(1, n - 1))], hq, 2, 128, 32, dtype, seed=6)
    c.check(*c.run())


def test_rising_scores_move_the_maximum(gpu_lib):
    """Keys that grow along the axis: every block raises the maximum."""
    for dtype in (BF16, F32):
        for reqs in ([(1500, 1)], [(1500, 300)]):
            c = Case(reqs, 4, 1, 128, 16, dtype, seed=7)
            ramp = torch.linspace(0.1, 4.0, 1500)[None, :, None]
            c.keys[0] = (c.keys[0].float().abs() * ramp).to(dtype)
            pages = c.table[0, :-1].long().cpu()
            flat = torch.zeros(1, len(pages) * 16, 128, dtype=dtype)
            flat[:, :1500] = c.keys[0]
            c.k[pages.cuda()] = flat.view(1, -1, 16, 128).transpose(0, 1).cuda()
            c.q = c.q.abs()
            c.check(*c.run())


def test_scale_dense_queries_and_given_output(gpu_lib):
    c = Case([(100, 20), (90, 1)], 4, 2, 64, 16, BF16, seed=8, qkv=False)
    out = torch.full((21, 4, 64), 7.0, dtype=BF16, device="cuda")
    got, lse = c.run(scale=0.5, out=out)
    assert got.data_ptr() == out.data_ptr()
    c.check(got, lse, scale=0.5)
    # tokens that belong to no request keep what out held
    c.q = torch.cat([c.q, c.q[:4]])
    out = torch.full((25, 4, 64), 7.0, dtype=BF16, device="cuda")
    c.run(out=out)
    assert (out[21:] == 7.0).all()


def test_misaligned_queries(gpu_lib):
    for n in (1, 60):
        c = Case([(100, n)], 4, 2, 64, 16, BF16, seed=9)
        wide = torch.zeros(n, 4 * 64 + 3, dtype=BF16, device="cuda")
        wide[:, 3:] = c.q.reshape(n, -1)
        c.q = wide[:, 3:].unflatten(1, (4, 64))
        c.check(*c.run())


def test_bad_table_entries_read_as_zeros(gpu_lib):
    """Entries outside the cache inside a request's length: keys and values
    of zero, no access."""
    for n in (1, 40):
        c = Case([(64, n)], 4, 2, 64, 16, BF16, seed=10)
        for i, bad in ((1, -1), (2, 10 ** 6)):
            c.table[0, i] = bad
            c.keys[0][:, 16 * i:16 * i + 16] = 0
            c.values[0][:, 16 * i:16 * i + 16] = 0
        c.check(*c.run())


def test_attention_on_another_stream_and_in_a_graph(gpu_lib):
    c = Case([(333, 1), (90, 1)], 8, 2, 128, 16, BF16, seed=11)
    want = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = c.run()
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    start, kv = _i32(c.start), _i32([k for k, _ in c.reqs])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = paged_attention(c.q, c.k, c.v, c.table, start, kv, 1)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0])


def test_plan_append_attend_over_steps(gpu_lib):
    """Two prompts of different lengths, then decode steps: the cache that the
    plan and the append build gives the attention over all tokens so far."""
    torch.manual_seed(0)
    hq, hk, dim, page, width = 8, 2, 64, 16, 12
    kc = torch.full((40, hk, page, dim), float("nan"), device="cuda", dtype=BF16)
    vc = kc.clone()
    table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    free_pages = torch.randperm(40, device="cuda").to(torch.int32)
    free, ctx = _i32([40]), _i32([0, 0, 0])
    hist = [[], [], []]
    for new in ([33, 80, 1], [1, 1, 1], [1, 0, 16], [1, 1, 1]):
        T = sum(new)
        qkv = torch.randn(T, hq + 2 * hk, dim, device="cuda").to(BF16)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        left = _i32([0])
        q_start, kv_lens, slots, _ = paged_plan(ctx, _i32(new), table, free_pages, free, page, T,
                                                free_left=left)
        free = left
        paged_append(kc, vc, k, v, slots)
        out = paged_attention(q, kc, vc, table, q_start, kv_lens, max(new))
        at = 0
        for r, n in enumerate(new):
            hist[r] += [(k[at + i].double(), v[at + i].double()) for i in range(n)]
            for i in range(n):
                seen = hist[r][:len(hist[r]) - n + i + 1]
                ks = torch.stack([x for x, _ in seen]).repeat_interleave(hq // hk, 1)
                vs = torch.stack([x for _, x in seen]).repeat_interleave(hq // hk, 1)
                p = torch.softmax(torch.einsum("hd,khd->hk", q[at + i].double(), ks)
                                  / math.sqrt(dim), -1)
                want = torch.einsum("hk,khd->hd", p, vs)
                a = torch.einsum("hk,khd->hd", p, vs.abs())
                assert ((out[at + i].double() - want).abs() <= 2.2 * EPS16 * a + 1e-4 * a).all()
            at += n
        ctx = kv_lens
    assert free.item() == 40 - sum(-(-len(h) // page) for h in hist)


# ---- refusals ----------------------------------------------------------------

def test_refusals_of_the_python_calls(gpu_lib):
    c = Case([(33, 1)], 4, 2, 64, 16, BF16)
    start, kv = _i32([0, 1]), _i32([33])
    with pytest.raises(ValueError):
        paged_attention(c.q.float(), c.k, c.v, c.table, start, kv, 1)
    with pytest.raises(ValueError):
        paged_attention(c.q, c.k, c.v.float(), c.table, start, kv, 1)
    with pytest.raises(ValueError):
        paged_attention(c.q, c.k, c.v, c.table.long(), start, kv, 1)
    with pytest.raises(ValueError):
        paged_attention(c.q, c.k, c.v, c.table, start[:1], kv, 1)
    with pytest.raises(ValueError):
        paged_attention(c.q, c.k.transpose(1, 2), c.v.transpose(1, 2), c.table, start, kv, 1)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(max_new=-1)):
        with pytest.raises(binding.UltraMemError) as e:
            c.run(**kw)
        assert e.value.status == binding.EINVAL
    with pytest.raises(binding.UltraMemError):      # 3 query heads on 2
        paged_attention(c.q[:, :3], c.k, c.v, c.table, start, kv, 1)
    with pytest.raises(ValueError):
        paged_append(c.k, c.v, c.q[:, :2], c.q[:, :2].float(), _i32([0]))
    with pytest.raises(ValueError):
        paged_append(c.k, c.v, c.q[:, :2], c.q[:, :2], _i32([0, 1]))
    with pytest.raises(ValueError):
        paged_plan(kv, kv, c.table, _i32([1]), _i32([1, 2]), 16, 1)
    with pytest.raises(binding.UltraMemError):
        paged_plan(kv, _i32([1]), c.table, _i32([1]), _i32([1]), 24, 1)


def test_offsets_past_32_bits(gpu_lib):
    """Pages whose entries lie past 2^31 elements into the cache, for each
    kernel that reads or writes it."""
    hk, page, dim = 8, 256, 64
    n_pages = (1 << 31) // (hk * page * dim) + 40
    for dtype, n in ((BF16, 1), (BF16, 50), (F32, 1), (F32, 30)):
        kc = torch.empty(n_pages, hk, page, dim, dtype=dtype, device="cuda")
        vc = torch.empty_like(kc)
        used = [n_pages - 1, 3, n_pages - 20]
        for p in used:
            kc[p] = float("nan")
            vc[p] = float("nan")
        kv = 600
        gen = torch.Generator(device="cuda").manual_seed(12)
        k, v = (torch.randn(kv, hk, dim, generator=gen, device="cuda").to(dtype) for _ in range(2))
        table = _i32([used])
        pos = torch.arange(kv, device="cuda")
        slots = (table[0, pos // page] * page + pos % page).to(torch.int32)
        paged_append(kc, vc, k, v, slots)
        q = torch.randn(n, 2 * hk, dim, generator=gen, device="cuda").to(dtype)
        out = paged_attention(q, kc, vc, table, _i32([0, n]), _i32([kv]), n).double()
        kk, vv = (x.double().repeat_interleave(2, 1) for x in (k, v))
        s = torch.einsum("nhd,khd->hnk", q.double(), kk) / math.sqrt(dim)
        s = s.masked_fill(pos[None, :] > kv - n + torch.arange(n, device="cuda")[:, None], -math.inf)
        p = torch.softmax(s, -1)
        want = torch.einsum("hnk,khd->nhd", p, vv)
        a = torch.einsum("hnk,khd->nhd", p, vv.abs())
        low = 2 * EPS16 if dtype == BF16 else 0.0
        assert ((out - want).abs() <= (low + 1e-4) * a).all()
        del kc, vc


def test_workspace_is_not_read_before_it_is_written(gpu_lib):
    """Any contents of the workspace give the same result."""
    lib = binding.load()
    for dtype, reqs in ((BF16, [(3000, 1), (70, 1)]), (BF16, [(3000, 90), (70, 5)]),
                        (F32, [(3000, 1)]), (F32, [(900, 70)])):
        c = Case(reqs, 8, 2, 128, 16, dtype, seed=13)
        want, want_lse = c.run()
        cache = binding.KVCache(c.k.data_ptr(), c.v.data_ptr(), *c.k.shape,
                                binding.BF16 if dtype == BF16 else binding.F32)
        need = lib.ultramem_paged_attention_workspace(cache.dtype, 8, 2, 128, c.max_new)
        start, kv = _i32(c.start), _i32([k for k, _ in reqs])
        for fill in (0, 255, 1):
            ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
            out, lse = torch.empty_like(want), torch.empty_like(want_lse)
            q = c.q
            st = lib.ultramem_paged_attention(
                ctypes.byref(cache), q.data_ptr(), q.stride(0), 8, start.data_ptr(), kv.data_ptr(),
                c.table.data_ptr(), c.table.shape[1], len(reqs), c.start[-1], c.max_new,
                1 / math.sqrt(128), out.data_ptr(), lse.data_ptr(), ws.data_ptr(), need,
                torch.cuda.current_stream().cuda_stream)
            assert st == binding.OK
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert lib.ultramem_paged_check(None) == binding.OK


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv", [60, 64, 120, 128, 130, 250, 510, 760, 768, 770, 800])
def test_tables_around_the_length_that_is_never_split(dtype, kv, gpu_lib):
    """Row capacities on both sides of the lengths whose tiles stay whole."""
    for n in (1, min(kv, 40)):
        c = Case([(kv, n), (17, n if n <= 17 else 17)], 8, 1, 64, 16, dtype, seed=14)
        c.check(*c.run())
        c = Case([(kv, n)], 4, 1, 128, 32, dtype, seed=15)
        c.check(*c.run())
