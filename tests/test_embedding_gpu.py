"""The embedding of token ids and its gradient against plain sums in 64 bits."""
import pytest
import torch

from paper_2411_12364_gb300 import vocab

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 7, 8), (5, 3, 13), (33, 100, 64), (300, 17, 257),
                                   (64, 1000, 1024), (2000, 50, 40), (9, 5, 4104)])
@pytest.mark.parametrize("ids_type", [torch.int32, torch.int64])
def test_embedding(gpu_lib, dtype, T, V, D, ids_type):
    g = gen(T + V + D)
    table = randn(g, V, D, dtype=dtype)
    ids = torch.randint(-2, V + 2, (T,), generator=g, device="cuda")   # some are outside
    scale = 1.7
    got = vocab.embedding(table, ids.to(ids_type), scale=scale)
    known = (ids >= 0) & (ids < V)
    # one product in 32 bits and one rounding: the result is a single value
    want = table[ids.clamp(0, V - 1)].float() * torch.tensor(scale, dtype=F32, device="cuda")
    assert torch.equal(got, torch.where(known[:, None], want, 0.0).to(dtype))


def test_embedding_rows_apart_and_given_output(gpu_lib):
    g = gen(1)
    for start in (0, 1, 8):          # 16-byte and other boundaries
        table = randn(g, 30, 100, dtype=BF16)[:, start:start + 64]
        ids = torch.arange(29, -1, -1, device="cuda")
        out = torch.full((31, 64), 7.0, dtype=BF16, device="cuda")
        got = vocab.embedding(table, ids, out=out[:30])
        assert got.data_ptr() == out.data_ptr()
        assert torch.equal(out[:30], table[ids]) and bool((out[30] == 7).all())
    wide = torch.iinfo(torch.int64).max
    ids = torch.tensor([0, 2 ** 32, -2 ** 32, wide, -wide - 1, 1], device="cuda")
    got = vocab.embedding(table, ids)
    assert torch.equal(got[[0, 5]], table[:2]) and not bool(got[1:5].any())


def test_embedding_offsets_past_32_bits(gpu_lib):
    V, D = 2 ** 20 + 3, 4096         # 2^32 entries and some
    table = torch.zeros(V, D, dtype=BF16, device="cuda")
    table[-1] = torch.arange(D, device="cuda").to(BF16)
    table[0] = 3
    got = vocab.embedding(table, torch.tensor([V - 1, 0, V - 2], device="cuda"))
    assert torch.equal(got, table[[V - 1, 0, V - 2]])
    del table
    dout = torch.ones(2, D, dtype=BF16, device="cuda")
    grad = vocab.embedding_backward(torch.tensor([V - 1, V - 1], device="cuda"), dout, V)
    assert bool((grad[-1] == 2).all()) and float(grad[-3:-1].abs().sum()) == 0
    assert float(grad.abs().amax()) == 2 and int((grad != 0).sum()) == D


def reference(ids, dout, V, scale):
    """The gradient in 64 bits, and the sum of magnitudes and the number of terms."""
    known = (ids >= 0) & (ids < V)
    D = dout.shape[1]
    total = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    size = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    count = torch.zeros(V, 1, dtype=torch.float64, device="cuda")
    i, x = ids[known], dout[known].double()
    total.index_add_(0, i, x * scale)
    size.index_add_(0, i, (x * scale).abs())
    count.index_add_(0, i, torch.ones(i.numel(), 1, dtype=torch.float64, device="cuda"))
    return total, size, count


def bound(total, size, count, dtype):
    """n terms: n - 1 additions, the product with the scale and the scale itself
    (each 2^-24 of at most the sum of magnitudes), one rounding to the type."""
    half = torch.finfo(dtype).eps / 2
    return (count + 2) * 2.0 ** -24 * size * (1 + half) + half * total.abs() + 1e-40


CASES = [(1, 1, 1), (1, 9, 8), (31, 5, 13), (32, 4, 64), (33, 1, 72), (100, 300, 257),
         (1000, 37, 1000), (4097, 64, 136), (3000, 70000, 24), (16384, 3, 40), (16385, 300, 33),
         (50000, 1000, 16), (40000, 1, 8), (70000, 200000, 8)]


@pytest.mark.parametrize("T,V,D", CASES)
@pytest.mark.parametrize("dtype,table_dtype", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
def test_gradient(gpu_lib, T, V, D, dtype, table_dtype):
    g = gen(T + 3 * V + D)
    ids = torch.randint(-1, V + 1, (T,), generator=g, device="cuda")
    ids = torch.where(torch.rand(T, generator=g, device="cuda") < 0.3, V // 2, ids)   # a frequent one
    dout = randn(g, T, D, dtype=dtype)
    scale = 0.75
    want, size, count = reference(ids, dout, V, scale)
    old = randn(g, V, D, dtype=table_dtype)
    for accumulate in (False, True):
        table = old.clone()
        got = vocab.embedding_backward(ids, dout, V, scale=scale, dtable=table,
                                       accumulate=accumulate)
        assert got is table
        if accumulate:
            err = (got.double() - (want + old.double())).abs()
            allowed = bound(want + old.double(), size + old.double().abs(), count + 1, table_dtype)
            still = (count == 0).squeeze(1)
            assert torch.equal(got[still], old[still])
        else:
            err, allowed = (got.double() - want).abs(), bound(want, size, count, table_dtype)
        assert bool((err <= allowed).all()), float((err / allowed).max())
        # the sums have a fixed order
        again = vocab.embedding_backward(ids.to(torch.int32), dout, V, scale=scale,
                                         dtable=old.clone(), accumulate=accumulate)
        assert torch.equal(got, again)


@pytest.mark.parametrize("T,V,D", [(512, 3, 1024), (512, 1, 8), (513, 40, 16), (512, 70001, 24),
                                   (257, 609, 100), (60, 607, 8200), (500, 2, 1), (7, 1300, 2056)])
@pytest.mark.parametrize("dtype,table_dtype", [(BF16, BF16), (F32, BF16), (BF16, F32)])
def test_short_batches(gpu_lib, T, V, D, dtype, table_dtype):
    """About the size up to which one launch does it all."""
    g = gen(T + V + 7 * D)
    ids = torch.randint(-1, V + 1, (T,), generator=g, device="cuda")
    ids = torch.where(torch.rand(T, generator=g, device="cuda") < 0.3, V - 1, ids)
    dout = randn(g, T, D, dtype=dtype)
    want, size, count = reference(ids, dout, V, -1.5)
    flat = torch.full((V + 2, D), 5.0, dtype=table_dtype, device="cuda")
    got = vocab.embedding_backward(ids, dout, V, scale=-1.5, dtable=flat[1:V + 1])
    assert bool(((got.double() - want).abs() <= bound(want, size, count, table_dtype)).all())
    assert bool((flat[0] == 5).all()) and bool((flat[-1] == 5).all())
    again = vocab.embedding_backward(ids.int(), dout, V, scale=-1.5,
                                     dtable=torch.empty_like(got))
    assert torch.equal(got, again)
    old = randn(g, V, D, dtype=table_dtype)
    got = vocab.embedding_backward(ids, dout, V, scale=-1.5, dtable=old.clone(), accumulate=True)
    allowed = bound(want + old.double(), size + old.double().abs(), count + 1, table_dtype)
    assert bool(((got.double() - want - old.double()).abs() <= allowed).all())
    still = (count == 0).squeeze(1)
    assert torch.equal(got[still], old[still])


def test_sorted_gradient_offsets_past_32_bits(gpu_lib):
    V, D, T = 2 ** 20 + 3, 4096, 600
    dout = torch.ones(T, D, dtype=BF16, device="cuda")
    ids = torch.full((T,), V - 1, device="cuda")
    ids[::2] = V - 2
    grad = vocab.embedding_backward(ids, dout, V)
    assert bool((grad[-2:] == 300).all()) and int((grad != 0).sum()) == 2 * D


def test_gradient_of_rows_apart_and_of_nothing(gpu_lib):
    g = gen(5)
    for start in (0, 3):
        dout = randn(g, 200, 90, dtype=BF16)[:, start:start + 80]
        ids = torch.randint(0, 40, (200,), generator=g, device="cuda")
        got = vocab.embedding_backward(ids, dout, 41)
        want, size, count = reference(ids, dout, 41, 1.0)
        assert bool(((got.double() - want).abs() <= bound(want, size, count, BF16)).all())
        assert not bool(got[40].any())
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    empty = torch.zeros(0, 24, dtype=F32, device="cuda")
    table = torch.ones(5, 24, device="cuda")
    vocab.embedding_backward(none, empty, 5, dtable=table, accumulate=True)
    assert bool((table == 1).all())
    vocab.embedding_backward(none, empty, 5, dtable=table)
    assert not bool(table.any())
    outside = torch.full((60,), -1, device="cuda")
    got = vocab.embedding_backward(outside, torch.full((60, 24), float("nan"), device="cuda"), 5)
    assert not bool(got.any())       # what outside ids bring does not count
    assert vocab.embedding(table, none).shape == (0, 24)


def test_gradient_beside_what_it_must_not_write(gpu_lib):
    g = gen(6)
    for offset in (0, 1, 3):         # dtable's ends within 16-byte pieces
        flat = torch.full((7 * 13 + 40,), 5.0, dtype=BF16, device="cuda")
        table = flat[offset:offset + 7 * 13].view(7, 13)
        ids = torch.tensor([2, 2, 6], device="cuda")
        dout = randn(g, 3, 13, dtype=BF16)
        vocab.embedding_backward(ids, dout, 7, dtable=table)
        assert bool((flat[:offset] == 5).all()) and bool((flat[offset + 7 * 13:] == 5).all())
        assert torch.equal(table[6], dout[2]) and not bool(table[[0, 1, 3, 4, 5]].any())


def test_gradient_against_differences(gpu_lib):
    """Through the forward: a linear map, so differences are exact up to rounding."""
    g = gen(7)
    table, ids = randn(g, 11, 16), torch.tensor([3, 0, 3, -1, 10], device="cuda")
    dout = randn(g, 5, 16)
    grad = vocab.embedding_backward(ids, dout, 11, scale=2.0)
    for v, c in ((3, 0), (0, 5), (10, 15), (7, 2)):
        up = table.clone()
        up[v, c] += 1.0
        change = vocab.embedding(up, ids, scale=2.0).double() - \
            vocab.embedding(table, ids, scale=2.0).double()
        # the step survives the table's rounding up to 2^-24 of |table| + 1
        allowed = 2.0 ** -20 * float(dout.abs().sum())
        assert abs(float((change * dout.double()).sum()) - float(grad[v, c])) <= allowed


def test_captured_on_another_stream(gpu_lib):
    g = gen(8)
    ids = torch.randint(0, 50, (600,), generator=g, device="cuda")
    dout, table = randn(g, 600, 64, dtype=BF16), randn(g, 50, 64, dtype=BF16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = vocab.embedding(table, ids)
        grad = vocab.embedding_backward(ids, dout, 50)
    for seed in (9, 10):             # replayed on other values
        ids.copy_(torch.randint(0, 50, (600,), generator=gen(seed), device="cuda"))
        dout.copy_(randn(gen(seed), 600, 64))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, table[ids])
        assert torch.equal(grad, vocab.embedding_backward(ids, dout, 50))
