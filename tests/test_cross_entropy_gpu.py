"""The softmax cross entropy over a vocabulary and its gradient against plain
forms in 64 bits."""
import pytest
import torch

from paper_2411_12364_gb300 import paged, vocab

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def inputs(T, V, D, dtype, seed=0, spread=2.0):
    g = gen(seed + T + 7 * V + 31 * D)
    x = torch.randn(T, D, generator=g, device="cuda").to(dtype)
    w = (torch.randn(V, D, generator=g, device="cuda") * spread / D ** 0.5).to(dtype)
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    labels = torch.where(torch.rand(T, generator=g, device="cuda") < 0.15, -100, labels)
    dloss = torch.rand(T, generator=g, device="cuda") + 0.5
    return x, w, labels, dloss


def counts(labels, V):
    return (labels >= 0) & (labels < V)


def z_error(x, w, s):
    """Bound of a logit's error [T, V]: D additions, each off by at most 2^-23 of
    the sum of magnitudes (the tensor cores may truncate), the product with
    the scale; values in three bf16 terms keep 24 bits and drop products
    of 2^-24."""
    D = x.shape[1]
    return (D + 10) * 2.0 ** -23 * abs(s) * (x.double().abs() @ w.double().abs().T)


def check_forward(x, w, labels, s, got):
    T, V = x.shape[0], w.shape[0]
    z = (x.double() @ w.double().T) * s
    lse = torch.logsumexp(z, 1)
    err = z_error(x, w, s)
    top = err.amax(1)
    # the logits' error, that of e^ and of a sum of V values in pieces (its
    # relative error), and roundings of the result and of what it is made of
    tol = top + 2.0 ** -20 + (256 + V / 64) * 2.0 ** -24 + \
        8 * 2.0 ** -24 * (z.abs().amax(1) + lse.abs())
    loss, got_lse = got
    assert bool(((got_lse.double() - lse).abs() <= tol).all())
    ok = counts(labels, V)
    want = torch.where(ok, lse - z.gather(1, labels.clamp(0, V - 1)[:, None])[:, 0], 0.0)
    assert bool(((loss.double() - want).abs() <= 2 * tol).all())
    assert not bool(loss[~ok].any())


def check_backward(x, w, labels, lse, dloss, s, got):
    T, V = x.shape[0], w.shape[0]
    half = torch.finfo(x.dtype).eps / 2
    xd, wd = x.double(), w.double()
    ok = counts(labels, V)
    xd = torch.where(ok[:, None], xd, 0.0)
    z = (xd @ wd.T) * s
    p = torch.exp(z - lse.double()[:, None])
    onehot = torch.zeros_like(p)
    onehot[ok, labels[ok]] = 1.0
    d = torch.where(ok, dloss.double(), 0.0)[:, None] * s
    g = torch.where(ok[:, None], (p - onehot) * d, 0.0)
    # G: the logit's error and that of e^ (2^-20 and the rounding of exponents
    # of this size) scale p; then roundings in 32 bits and one to the type
    rel = z_error(xd, w, s) + 2.0 ** -20 + 4 * 2.0 ** -24 * (z.abs() + lse.double().abs()[:, None])
    ge = torch.where(ok[:, None], (p * rel + 2.0 ** -22 * (p + onehot)) * d.abs(), 0.0)
    ge = ge + half * (g.abs() + ge)
    dx, dw = got
    for want, err, size, n in ((g @ wd, ge @ wd.abs(), g.abs() @ wd.abs(), V),
                               (g.T @ xd, ge.T @ xd.abs(), g.T.abs() @ xd.abs(), T)):
        have, dx = dx, dw
        tol = err + (n + 10) * 2.0 ** -23 * size
        tol = tol + half * (want.abs() + tol) + 1e-38
        assert bool(((have.double() - want).abs() <= tol).all()), \
            float(((have.double() - want).abs() / tol).max())


SIZES = [(1, 1, 1), (1, 100, 8), (3, 2, 64), (64, 333, 40), (65, 257, 129), (100, 1000, 96),
         (128, 256, 64), (129, 255, 72), (257, 513, 200), (300, 77, 512), (17, 5003, 333),
         (1000, 130, 64), (513, 2050, 320)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_both_directions(gpu_lib, dtype, T, V, D):
    x, w, labels, dloss = inputs(T, V, D, dtype)
    for s, kind in ((1.0, torch.int64), (-0.37, torch.int32)):
        got = vocab.cross_entropy(x, w, labels.to(kind), logit_scale=s)
        check_forward(x, w, labels, s, got)
        grads = vocab.cross_entropy_backward(x, w, labels.to(kind), got[1], dloss, logit_scale=s)
        check_backward(x, w, labels, got[1], dloss, s, grads)
        again = vocab.cross_entropy_backward(x, w, labels, got[1], dloss, logit_scale=s)
        assert all(torch.equal(a, b) for a, b in zip(grads, again))   # a fixed order
        only = vocab.cross_entropy_backward(x, w, labels, got[1], dloss, logit_scale=s, dw=False)
        assert only[1] is None and torch.equal(only[0], grads[0])
        only = vocab.cross_entropy_backward(x, w, labels, got[1], dloss, logit_scale=s, dx=None)
        assert only[0] is None and torch.equal(only[1], grads[1])
    assert paged.paged_check() == 0


@pytest.mark.parametrize("T,V,D,dtype", [(9000, 40, 64, BF16), (2, 70000, 72, BF16),
                                         (40, 30011, 33, F32), (7000, 9, 8, F32)])
def test_long_sums(gpu_lib, T, V, D, dtype):
    """Few rows against many: the long sums are split."""
    x, w, labels, dloss = inputs(T, V, D, dtype)
    got = vocab.cross_entropy(x, w, labels)
    check_forward(x, w, labels, 1.0, got)
    check_backward(x, w, labels, got[1], dloss, 1.0,
                   vocab.cross_entropy_backward(x, w, labels, got[1], dloss))


def test_vocabulary_in_pieces(gpu_lib):
    """More logits than a piece of the workspace holds."""
    T, V, D = 8192, 40000, 64
    x, w, labels, dloss = inputs(T, V, D, BF16)
    loss, lse = vocab.cross_entropy(x, w, labels)
    z = x.float() @ w.float().T
    lse_want = torch.logsumexp(z.double(), 1)
    tol = z_error(x, w, 1.0).amax(1) + 2.0 ** -20 + (256 + V / 64) * 2.0 ** -24 + 2.0 ** -20
    assert bool(((lse.double() - lse_want).abs() <= 2 * tol).all())
    got = vocab.cross_entropy_backward(x, w, labels, lse, dloss)
    check_backward(x, w, labels, lse, dloss, 1.0, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_apart(gpu_lib, dtype):
    for start, width in ((0, 64), (1, 65), (8, 50)):
        x, w, labels, dloss = inputs(70, 140, 100, dtype)
        x, w = x[:, start:start + width], w[:, start:start + width]
        loss, lse = vocab.cross_entropy(x, w, labels)
        check_forward(x, w, labels, 1.0, (loss, lse))
        dx = torch.full((72, width), 9.0, dtype=dtype, device="cuda")
        dw = torch.full((142, width), 9.0, dtype=dtype, device="cuda")
        got = vocab.cross_entropy_backward(x, w, labels, lse, dloss, dx=dx[:70], dw=dw[1:141])
        check_backward(x, w, labels, lse, dloss, 1.0, got)
        assert bool((dx[70:] == 9).all()) and bool((dw[0] == 9).all()) and bool((dw[141] == 9).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tokens_that_do_not_count(gpu_lib, dtype):
    T, V, D = 90, 300, 72
    x, w, labels, dloss = inputs(T, V, D, dtype)
    labels[:] = torch.arange(T, device="cuda")
    labels[5], labels[40], labels[89] = -100, V, 2 ** 40
    clean = x.clone()
    x[5], x[40, 3], x[89] = NAN, INF, -INF
    dloss[5], dloss[40] = NAN, INF
    loss, lse = vocab.cross_entropy(x, w, labels)
    out = [5, 40, 89]
    assert not bool(loss[out].any())
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[out] = False
    check_forward(x[keep], w, labels[keep], 1.0, (loss[keep], lse[keep]))
    dx, dw = vocab.cross_entropy_backward(x, w, labels, lse, dloss)
    assert not bool(dx[out].any())
    lse2, dloss2 = lse.clone(), dloss.clone()
    lse2[out], dloss2[out] = 0.0, 0.0
    check_backward(clean, w, labels, lse2, dloss2, 1.0, (dx, dw))
    none = torch.full_like(labels, -1)
    loss, lse = vocab.cross_entropy(clean, w, none)
    assert not bool(loss.any())
    dx, dw = vocab.cross_entropy_backward(x, w, none, lse, dloss)
    assert not bool(dx.any()) and not bool(dw.any())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_logits(gpu_lib, dtype):
    """Logits of hundreds: only differences enter the exponentials."""
    x, w, labels, dloss = inputs(40, 500, 64, dtype, spread=150.0)
    loss, lse = vocab.cross_entropy(x, w, labels)
    check_forward(x, w, labels, 1.0, (loss, lse))
    check_backward(x, w, labels, lse, dloss, 1.0,
                   vocab.cross_entropy_backward(x, w, labels, lse, dloss))
    loss, lse = vocab.cross_entropy(x, w, labels, logit_scale=0.0)
    check_forward(x, w, labels, 0.0, (loss, lse))


def test_no_tokens(gpu_lib):
    x, w = torch.zeros(0, 16, dtype=BF16, device="cuda"), torch.ones(9, 16, dtype=BF16, device="cuda")
    labels, f = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    loss, lse = vocab.cross_entropy(x, w, labels)
    assert loss.shape == lse.shape == (0,)
    dx, dw = vocab.cross_entropy_backward(x, w, labels, f, f)
    assert dx.shape == (0, 16) and not bool(dw.any())


def test_gradient_against_differences(gpu_lib):
    """Central differences of the summed loss in 32-bit storage."""
    T, V, D = 6, 20, 8
    x, w, labels, dloss = inputs(T, V, D, F32, seed=3)
    labels[0] = 4

    def total(a, b):
        return float((vocab.cross_entropy(a, b, labels)[0].double() * dloss.double()).sum())

    dx, dw = vocab.cross_entropy_backward(x, w, labels, vocab.cross_entropy(x, w, labels)[1], dloss)
    h = 2.0 ** -6
    # h^2/6 of a third derivative (at most |w|^3 or |x|^3 a token, times dloss)
    # and the losses' own errors over 2h: 2^-19 each of a loss below 16
    tol = h * h / 6 * 2 * T * 1.5 * max(float(w.abs().max()), float(x.abs().max())) ** 3 + \
        T * 1.5 * 2.0 ** -19 / h
    for t, c in ((0, 0), (3, 5)):
        up, down = x.clone(), x.clone()
        up[t, c] += h
        down[t, c] -= h
        assert abs((total(up, w) - total(down, w)) / (2 * h) - float(dx[t, c])) <= tol
    for v, c in ((4, 1), (19, 7)):
        up, down = w.clone(), w.clone()
        up[v, c] += h
        down[v, c] -= h
        assert abs((total(x, up) - total(x, down)) / (2 * h) - float(dw[v, c])) <= tol


def test_captured_on_another_stream(gpu_lib):
    x, w, labels, dloss = inputs(130, 700, 128, BF16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        loss, lse = vocab.cross_entropy(x, w, labels)
        dx, dw = vocab.cross_entropy_backward(x, w, labels, lse, dloss)
    for seed in (1, 2):
        for a, b in zip((x, w, labels, dloss), inputs(130, 700, 128, BF16, seed=seed)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        check_forward(x, w, labels, 1.0, (loss, lse))
        check_backward(x, w, labels, lse, dloss, 1.0, (dx, dw))


def test_values_that_bf16_does_not_hold(gpu_lib):
    """The largest fp32 values among the weights: their terms stay finite."""
    x, w, labels, dloss = inputs(9, 40, 16, F32)
    x[:, 3] = 0
    x[0, 3] = 1e-30
    w[7, 3], w[8, 3] = -torch.finfo(F32).max, torch.finfo(F32).max
    labels[:] = torch.arange(9, device="cuda")
    x[0] *= 1e-8                         # its logits stay in range
    loss, lse = vocab.cross_entropy(x, w, labels)
    z = x.double() @ w.double().T
    keep = z.abs().amax(1) < 1e30
    assert bool(keep[1:].all())
    check_forward(x[1:], w, labels[1:], 1.0, (loss[1:], lse[1:]))


def test_offsets_past_32_bits(gpu_lib):
    """More than 2^32 entries in the weights and in their gradient."""
    V, D = 2 ** 20 + 77, 4096
    g = gen(11)
    w = torch.zeros(V, D, dtype=BF16, device="cuda")
    rows = torch.tensor([0, 5, V // 2, V - 1], device="cuda")
    w[rows] = torch.randn(4, D, generator=g, device="cuda").to(BF16) * 0.03
    x = torch.randn(3, D, generator=g, device="cuda").to(BF16)
    labels = torch.tensor([V - 1, 5, V // 2], device="cuda")
    loss, lse = vocab.cross_entropy(x, w, labels)
    z = x.double() @ w[rows].double().T
    want = torch.log((V - 4) + torch.exp(z).sum(1))
    pick = z[torch.arange(3), torch.tensor([3, 1, 2])]
    # all other logits are exactly 0; the rest as in check_forward
    tol = z_error(x, w[rows], 1.0).amax(1) + 2.0 ** -20 + (256 + V / 64) * 2.0 ** -24
    assert bool(((lse.double() - want).abs() <= tol).all())
    assert bool(((loss.double() - (want - pick)).abs() <= 2 * tol).all())
    dloss = torch.ones(3, device="cuda")
    dx, dw = vocab.cross_entropy_backward(x, w, labels, lse, dloss)
    # G and the results are rounded to bf16 (2^-8 each); the logits' errors, below
    # 2^-10, scale p: together below 2^-6 of the sums of magnitudes
    p = torch.exp(z - lse.double()[:, None])
    p[torch.arange(3), torch.tensor([3, 1, 2])] -= 1
    for i, r in enumerate(rows.tolist()):
        want = p[:, i] @ x.double()
        size = p[:, i].abs() @ x.double().abs()
        assert bool(((dw[r].double() - want).abs() <= 2.0 ** -6 * size + 1e-30).all())
    quiet = dw[1:5].double()             # rows of weight e^-lse alone
    even = torch.exp(-lse.double()) @ x.double()
    assert bool(((quiet - even).abs() <= 2.0 ** -6 * (torch.exp(-lse.double()) @ x.double().abs())).all())
    want = p @ w[rows].double()
    assert bool(((dx.double() - want).abs() <=
                 2.0 ** -6 * (p.abs() @ w[rows].double().abs()) + 1e-30).all())
