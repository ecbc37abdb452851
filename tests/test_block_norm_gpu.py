"""The fused norms around a block and their gradient on the GPU, against
64-bit formulas, torch's 64-bit autograd and finite differences."""
import itertools

import pytest
import torch

from paper_2411_12364_gb300 import binding
from paper_2411_12364_gb300.norms import block_norm, block_norm_backward

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5
# A row's sums pass at most 80 additions in a chain (32 in a thread, 5 between
# lanes, 32 between warps), each off by 2^-24 of the sum of magnitudes; a
# statistic, and what it multiplies, is off by a small multiple of that.
SUM = 80 * 2.0 ** -24
EPS16 = 2.0 ** -8     # rounding to bf16 (8 bits of significand)
DIMS = [1, 7, 31, 64, 100, 256, 257, 264, 512, 520, 1000, 1024, 1032, 2048, 2051, 4096, 5000, 8192]


def make(T, D, dtype, kind, gate, seed=0, gains=True):
    gen = torch.Generator().manual_seed(seed)

    def randn(*s):
        return torch.randn(*s, generator=gen)

    p = dict(y=(1.5 * randn(T, D) + 0.3).to(dtype), r=(3 * randn(T, D) - 0.5).to(dtype),
             du=randn(T, D).to(dtype), dn=randn(T, D).to(dtype))
    w = dict(w_post=1 + 0.2 * randn(D), w_pre=1 + 0.2 * randn(D)) if gains else {}
    if kind == "layer" and gains:
        w.update(b_post=0.2 * randn(D), b_pre=0.2 * randn(D))
    if gate is not None:
        w["gate"] = {"channel": lambda: 0.5 + 0.2 * randn(D),
                     "token": lambda: randn(T, 1).to(dtype),
                     "full": lambda: randn(T, D).to(dtype)}[gate]()
    return p, w


def cuda(d):
    return {k: v.cuda() for k, v in d.items()}


def norm64(x, w, b, kind):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    h = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    return h * (1.0 if w is None else w) + (0.0 if b is None else b)


def stream64(p, w, kind, res, out, post=True):
    """u before it is stored."""
    z = norm64(p["y"], w.get("w_post"), w.get("b_post"), kind) if post else p["y"]
    return res * p["r"] + out * (w["gate"] if "gate" in w else 1.0) * z, z


def double(d):
    return {k: v.double() for k, v in d.items()}


def within(got, want, tol, what):
    err = (got.double().cpu() - want).abs()
    assert (err <= tol).all(), f"{what}: {(err / tol).max():.2f} of the bound"


def check_forward(T, D, dtype, kind, gate, post=True, pre=True, gains=True, **views):
    p, w = make(T, D, dtype, kind, gate, gains=gains)
    dp, dw = cuda(p), cuda(w)
    for k, f in views.items():
        dp[k] = f(dp[k])
    u, n = block_norm(dp["y"], dp["r"], kind=kind, eps=EPS, res_scale=0.9, out_scale=0.5,
                      post=post, pre=pre, **dw)
    p64, w64 = double(p), double(w)
    want, z = stream64(p64, w64, kind, 0.9, 0.5, post)
    add = (want - 0.9 * p64["r"]).abs()
    size = add.amax(-1, keepdim=True) + 0.9 * p64["r"].abs() + 0.5 * w64.get(
        "gate", torch.ones(1)).abs().amax(-1, keepdim=True)
    tol = 8 * SUM * size + 1e-30
    if dtype == BF16:
        tol = tol + EPS16 * (want.abs() + tol)
    within(u, want, tol, "u")
    if not pre:
        assert n is None
        return
    us = u.double().cpu()                      # the second norm reads the stored stream
    want = norm64(us, w64.get("w_pre"), w64.get("b_pre"), kind)
    # a rounding of mean or square sum acts on the whole row; a row of one
    # entry (or of equal ones) has only eps under the root
    centred = us - us.mean(-1, keepdim=True) if kind == "layer" else us
    rstd = 1 / torch.sqrt(centred.square().mean(-1, keepdim=True) + EPS)
    tol = 8 * SUM * (want.abs().amax(-1, keepdim=True) + 1
                     + rstd * us.abs().mean(-1, keepdim=True)) + 1e-30
    if dtype == BF16:
        tol = tol + EPS16 * (want.abs() + tol)
    within(n, want, tol, "n")


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_forward_matches_64_bits(D, dtype, kind, gpu_lib):
    for T, gate in ((5, "channel"), (1, None), (3, "token"), (9, "full")):
        check_forward(T, D, dtype, kind, gate)


@pytest.mark.parametrize("T", [1, 2, 63, 700, 5000])
@pytest.mark.parametrize("D", [64, 200, 1024, 2048])
def test_forward_over_many_tokens(T, D, gpu_lib):
    check_forward(T, D, BF16, "rms", "full")
    check_forward(T, D, F32, "layer", "channel")


@pytest.mark.parametrize("post,pre,gains", [(False, True, True), (True, False, True),
                                            (False, False, True), (True, True, False)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_forward_without_a_norm_or_gains(post, pre, gains, kind, gpu_lib):
    for gate in (None, "channel", "token", "full"):
        check_forward(6, 320, BF16, kind, gate, post, pre, gains)


def test_forward_reads_strided_and_misaligned_rows(gpu_lib):
    def strided(t):
        wide = torch.zeros(t.shape[0], t.shape[1] + 40, dtype=t.dtype, device="cuda")
        wide[:, 8:8 + t.shape[1]] = t
        return wide[:, 8:8 + t.shape[1]]

    def misaligned(t):
        wide = torch.zeros(t.shape[0], t.shape[1] + 3, dtype=t.dtype, device="cuda")
        wide[:, 1:1 + t.shape[1]] = t
        return wide[:, 1:1 + t.shape[1]]

    def transposed(t):
        return t.t().contiguous().t()

    for dtype in (BF16, F32):
        for f in (strided, misaligned, transposed):
            check_forward(33, 512, dtype, "layer", "full", y=f, r=f)


def test_forward_in_place(gpu_lib):
    for D in (512, 2048, 333):
        p, w = make(300, D, BF16, "rms", "channel")
        dp, dw = cuda(p), cuda(w)
        u, n = block_norm(dp["y"], dp["r"], **dw)
        y, r = dp["y"].clone(), dp["r"].clone()
        u2, n2 = block_norm(y, r, u=r, n=y, **dw)
        assert u2.data_ptr() == r.data_ptr() and n2.data_ptr() == y.data_ptr()
        assert torch.equal(u, u2) and torch.equal(n, n2)


def test_rows_of_zeros_equal_and_non_finite_entries(gpu_lib):
    """A row of zeros or of one value is normalised by eps alone; a NaN or an
    infinity stays in its row."""
    for dtype, D in itertools.product((BF16, F32), (64, 1024, 2048)):
        y = torch.randn(5, D).to(dtype)
        y[0] = 0
        y[1] = 2.0
        y[2, D // 2] = float("nan")
        y[3, 1] = float("inf")
        r = torch.randn(5, D).to(dtype)
        r[0] = 0
        u, n = block_norm(y.cuda(), r.cuda(), kind="layer")
        u, n = u.float().cpu(), n.float().cpu()
        assert (u[0] == 0).all() and (n[0] == 0).all()
        assert torch.equal(u[1], r[1].float())
        assert u[2].isnan().all() and u[3].isnan().any()
        assert torch.isfinite(u[4]).all() and torch.isfinite(n[4]).all()
        want = norm64(y.double(), None, None, "layer") + r.double()
        within(u[4], want[4], 0.05 * torch.ones(D, dtype=torch.float64), "a finite row")


def check_backward(T, D, dtype, kind, gate, post=True, pre=True, with_du=True, gains=True,
                   **views):
    p, w = make(T, D, dtype, kind, gate, seed=1, gains=gains)
    p["u"] = p.pop("r")
    dp, dw = cuda(p), cuda(w)
    for k, f in views.items():
        dp[k] = f(dp[k])
    got = block_norm_backward(dp["y"], dp["u"], dp["du"] if with_du else None,
                              dp["dn"] if pre else None, kind=kind, eps=EPS, res_scale=0.9,
                              out_scale=0.5, post=post, pre=pre, **dw)
    p64, w64 = double(p), double(w)
    for t in (p64["y"], p64["u"], *w64.values()):
        t.requires_grad_()
    gu = p64["du"].clone() if with_du else torch.zeros(T, D, dtype=torch.float64)
    if pre:
        norm64(p64["u"], w64.get("w_pre"), w64.get("b_pre"), kind).backward(p64["dn"])
        gu = gu + p64["u"].grad
    z = norm64(p64["y"], w64.get("w_post"), w64.get("b_post"), kind) if post else p64["y"]
    (0.5 * (w64["gate"] * z if gate else z)).backward(gu)

    def hat(x):
        c = x.detach() - x.detach().mean(-1, keepdim=True) if kind == "layer" else x.detach()
        rstd = 1 / torch.sqrt(c.square().mean(-1, keepdim=True) + EPS)
        return (c * rstd).abs() + rstd * x.detach().abs().mean(-1, keepdim=True) * SUM, rstd

    # magnitudes of what a sum over a row or over the tokens adds up
    uh, ru = hat(p64["u"])
    yh, ry = hat(p64["y"])
    wd = (w64["w_pre"].detach() if "w_pre" in w64 else 1.0) * p64["dn"].abs()
    mix = 1 + rows(uh)
    size = p64["du"].abs() * with_du
    if pre:
        size = size + ru * (wd + wd.mean(-1, keepdim=True) + uh * (wd * uh).mean(-1, keepdim=True)
                            ) * mix
    e_gu = 16 * SUM * size                            # of d u
    g64 = (w64["gate"].detach().abs() if gate else torch.ones(1, dtype=torch.float64)) * 0.5
    gz, e_gz = g64 * size, g64 * e_gu
    low = EPS16 if dtype == BF16 else 2.0 ** -24
    within(got["dr"], 0.9 * gu, 0.9 * e_gu + low * (gu.abs() + e_gu) + 1e-30, "dr")
    if post:
        wp = w64["w_post"].detach().abs() if "w_post" in w64 else 1.0
        s = gz * wp
        e_dy = 16 * SUM * ry * (s + s.mean(-1, keepdim=True)
                                + yh * (s * yh).mean(-1, keepdim=True)) * (1 + rows(yh)) * 2
    else:
        e_dy = 2 * e_gz
    want = p64["y"].grad
    within(got["dy"], want, e_dy + low * (want.abs() + e_dy) + 1e-30, "dy")

    def columns(name, terms, want):
        tol = 40 * SUM * terms.sum(0) + 1e-30        # at most 900 terms here, in chunks
        within(got[name], want, tol, name)

    if pre and gains:
        columns("dw_pre", p64["dn"].abs() * (uh + 1), w64["w_pre"].grad)
        if kind == "layer":
            columns("db_pre", p64["dn"].abs(), w64["b_pre"].grad)
    if post and gains:
        columns("dw_post", gz * (yh + 1) * mix, w64["w_post"].grad)
        if kind == "layer":
            columns("db_post", gz * mix, w64["b_post"].grad)
    zs = (z.detach().abs() + 1) * size * 0.5 * mix
    if gate == "channel":
        columns("dgate", zs, w64["gate"].grad)
    elif gate is not None:
        want = w64["gate"].grad
        terms = zs.sum(-1, keepdim=True) if gate == "token" else zs
        tol = 40 * SUM * terms
        within(got["dgate"], want, tol + low * (want.abs() + tol) + 1e-30, "dgate")
    else:
        assert got["dgate"] is None
    if not gains:
        assert got["dw_post"] is None and got["dw_pre"] is None and got["db_pre"] is None


def rows(x):
    return x.amax(-1, keepdim=True)


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_backward_matches_64_bit_autograd(D, dtype, kind, gpu_lib):
    for T, gate in ((5, "channel"), (1, None), (3, "token"), (9, "full")):
        check_backward(T, D, dtype, kind, gate)


# the first and last widths of each number of threads a row, odd and even
EDGES = [255, 513, 1025, 1026, 1535, 1536, 1537, 1544, 2049, 3000, 3064, 3080, 4095, 4097, 4104,
         6143, 6144, 6145, 6152, 8191]


@pytest.mark.parametrize("D", EDGES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_widths_around_the_threads_of_a_row(D, dtype, kind, gpu_lib):
    for T, gate in ((4, "channel"), (3, "token"), (311, "full")):
        check_forward(T, D, dtype, kind, gate)
        check_backward(T, D, dtype, kind, gate)


@pytest.mark.parametrize("T,D", [(2, 64), (900, 200), (700, 1024), (613, 2048)])
def test_backward_sums_over_many_tokens(T, D, gpu_lib):
    for dtype, kind, gate in ((BF16, "rms", "channel"), (F32, "layer", "channel"),
                              (F32, "rms", "full")):
        check_backward(T, D, dtype, kind, gate)


@pytest.mark.parametrize("kw", [dict(post=False), dict(pre=False), dict(with_du=False),
                                dict(post=False, with_du=False), dict(gains=False)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_backward_without_a_norm_gradient_or_gains(kw, kind, gpu_lib):
    for gate in (None, "channel", "token", "full"):
        check_backward(11, 320, F32, kind, gate, **kw)
        check_backward(11, 333, BF16, kind, gate, **kw)


def test_backward_reads_strided_rows_and_repeats_bitwise(gpu_lib):
    def strided(t):
        wide = torch.zeros(t.shape[0], t.shape[1] + 24, dtype=t.dtype, device="cuda")
        wide[:, 8:8 + t.shape[1]] = t
        return wide[:, 8:8 + t.shape[1]]

    for dtype in (BF16, F32):
        check_backward(33, 512, dtype, "layer", "full", y=strided, u=strided, du=strided,
                       dn=strided)
    p, w = make(3000, 1024, BF16, "layer", "channel")
    p["u"] = p.pop("r")
    args = dict(cuda(p), **cuda(w))
    a = block_norm_backward(kind="layer", **args)
    b = block_norm_backward(kind="layer", **args)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_backward_of_no_tokens_gives_zero_sums(gpu_lib):
    p, w = make(0, 64, F32, "layer", "channel")
    p["u"] = p.pop("r")
    got = block_norm_backward(kind="layer", **dict(cuda(p), **cuda(w)))
    for k in ("dw_post", "db_post", "dw_pre", "db_pre", "dgate"):
        assert (got[k] == 0).all()
    u, n = block_norm(p["y"].cuda(), p["u"].cuda())
    assert u.shape == n.shape == (0, 64)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate", ["channel", "token", "full"])
def test_gradient_matches_differences_of_the_forward(kind, gate, gpu_lib):
    """<gradient, direction> against the central difference of
    L = <du, u> + <dn, n> along random directions of every input (fp32,
    step 2^-6: the third derivative of a norm of unit rows leaves about
    step^2, the forward's rounding 2^-18 of L's terms over the step)."""
    T, D = 6, 128
    p, w = make(T, D, F32, kind, gate, seed=2)
    p, w = cuda(p), cuda(w)

    def loss(y, r, w):
        u, n = block_norm(y, r, kind=kind, eps=EPS, res_scale=0.9, out_scale=0.5, **w)
        return (p["du"].double() * u.double()).sum() + (p["dn"].double() * n.double()).sum()

    u, _ = block_norm(p["y"], p["r"], kind=kind, eps=EPS, res_scale=0.9, out_scale=0.5, **w)
    got = block_norm_backward(p["y"], u, p["du"], p["dn"], kind=kind, eps=EPS, res_scale=0.9,
                              out_scale=0.5, **w)
    h = 2.0 ** -6
    gen = torch.Generator().manual_seed(3)
    for name in ["y", "r", *w]:
        x = p[name] if name in p else w[name]
        d = torch.randn(x.shape, generator=gen).cuda()
        ends = []
        for s in (h, -h):
            moved = dict(w, **{name: x + s * d}) if name in w else w
            ends.append(loss(p["y"] + s * d if name == "y" else p["y"],
                             p["r"] + s * d if name == "r" else p["r"], moved))
        slope = ((ends[0] - ends[1]) / (2 * h)).item()
        grad = (got["d" + name].double() * d.double()).sum().item()
        scale = (got["d" + name].double().norm() * d.double().norm()).item()
        assert abs(slope - grad) <= 2e-3 * scale, name


def test_refusals(gpu_lib):
    p, w = make(4, 64, BF16, "rms", "channel")
    p, w = cuda(p), cuda(w)
    y, r = p["y"], p["r"]
    for bad in (dict(kind="batch"), dict(gate=torch.ones(3, device="cuda")),
                dict(gate=torch.ones(64, device="cuda", dtype=BF16)),
                dict(w_post=torch.ones(64, device="cuda", dtype=BF16)),
                dict(w_pre=torch.ones(65, device="cuda")), dict(w_pre=torch.ones(64))):
        with pytest.raises(ValueError):
            block_norm(y, r, **bad)
    with pytest.raises(ValueError):
        block_norm(y, r.float())
    with pytest.raises(ValueError):
        block_norm(y, r[:3])
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(res_scale=float("inf")),
                dict(b_post=w["w_post"])):
        with pytest.raises(binding.UltraMemError) as e:
            block_norm(y, r, **bad)
        assert e.value.status == binding.EINVAL
    with pytest.raises(binding.UltraMemError):
        block_norm(torch.zeros(1, 8200, device="cuda"), torch.zeros(1, 8200, device="cuda"))
    with pytest.raises(binding.UltraMemError):
        block_norm_backward(y, r, p["du"], None)      # the second norm needs dn
    with pytest.raises(binding.UltraMemError):
        block_norm_backward(y, r, None, None, pre=False)
