"""The cross entropy and its gradient over a vocabulary in several pieces, made small
enough for a comparison of every result with 64 bits."""
import pytest
import torch

from paper_2411_12364_gb300 import binding, paged, vocab
from tests.test_cross_entropy_gpu import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def pieces(gpu_lib):
    def set_bytes(n):
        assert gpu_lib.ultramem_debug_cross_entropy_piece(n) == binding.OK
        vocab._workspace.cache_clear()
    yield set_bytes
    set_bytes(0)


# pieces of 256 rows at least; (T, V, D, bytes of a piece)
CASES = [
    (300, 700, 64, 1 << 16),      # three, one split: the last adds the others' sums and writes dx
    (300, 513, 200, 1 << 16),     # the last of one row
    (40, 24584, 64, 1 << 18),     # K of dx in splits; the last piece of 8 rows has fewer k blocks
    (1000, 1300, 72, 1 << 20),    # two splits of dx, several of dw
    (9000, 700, 8, 1 << 22),      # dw summed over many tokens in splits, piece by piece
    (17, 5003, 333, 1 << 18),     # odd sizes, copied operands
    (130, 1500, 65, 1 << 16),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("s", [1.0, -0.37])
@pytest.mark.parametrize("T,V,D,piece", CASES)
def test_pieces(pieces, dtype, T, V, D, piece, s):
    x, w, labels, dloss = inputs(T, V, D, dtype)
    edges = torch.tensor([0, 255, 256, V - 1, 511, 512], device="cuda").clamp(max=V - 1)
    labels[:6] = edges                   # at the pieces' first and last rows
    whole = vocab._workspace(x.get_device(), "ultramem_cross_entropy_backward_workspace",
                             binding.BF16 if dtype == BF16 else binding.F32, T, V, D)
    pieces(piece)
    got = vocab.cross_entropy(x, w, labels, logit_scale=s)
    check_forward(x, w, labels, s, got)
    grads = vocab.cross_entropy_backward(x, w, labels, got[1], dloss, logit_scale=s)
    check_backward(x, w, labels, got[1], dloss, s, grads)
    again = vocab.cross_entropy_backward(x, w, labels, got[1], dloss, logit_scale=s)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    for skip in (dict(dw=False), dict(dx=False)):
        only = vocab.cross_entropy_backward(x, w, labels, got[1], dloss, logit_scale=s, **skip)
        assert all(b is None or torch.equal(a, b) for a, b in zip(grads, only))
    assert paged.paged_check() == 0
    assert whole != vocab._workspace(x.get_device(), "ultramem_cross_entropy_backward_workspace",
                                     binding.BF16 if dtype == BF16 else binding.F32, T, V, D)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pieces_beside_what_they_must_not_write(pieces, dtype):
    T, V, D = 70, 600, 72
    x, w, labels, dloss = inputs(T, V, D, dtype)
    pieces(1 << 16)
    loss, lse = vocab.cross_entropy(x, w, labels)
    dx, dw = (torch.full((n + 2, D), 9.0, dtype=dtype, device="cuda") for n in (T, V))
    got = vocab.cross_entropy_backward(x, w, labels, lse, dloss, dx=dx[1:T + 1], dw=dw[1:V + 1])
    check_backward(x, w, labels, lse, dloss, 1.0, got)
    for t in (dx, dw):
        assert bool((t[0] == 9).all()) and bool((t[-1] == 9).all())


def test_a_piece_of_no_bytes(gpu_lib):
    assert gpu_lib.ultramem_debug_cross_entropy_piece(-1) == binding.EINVAL
