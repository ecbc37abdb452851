"""Argument checks of the embedding, the cross entropy and the attention's
gradient: what they refuse, they refuse before anything is launched (no device
needed)."""
import ctypes as C

import pytest

from paper_2411_12364_gb300 import binding as b

FAKE = 1 << 20    # never dereferenced
INF, NAN = float("inf"), float("nan")


def refused(call, good, bad):
    for at, value in bad:
        args = list(good)
        args[at] = value
        assert call(*args) == b.EINVAL, (at, value)


def test_embedding():
    lib = b.load()
    good = [FAKE, 64, b.BF16, 100, 64, 2 * FAKE, 8, 5, 1.0, 3 * FAKE, None]
    refused(lib.ultramem_embedding, good, [
        (0, None), (0, FAKE + 1), (1, 63), (2, 2), (3, 0), (3, -1), (3, (1 << 30) + 1), (4, 0),
        (4, 65537), (5, None), (5, 2 * FAKE + 4), (6, 2), (6, 16), (7, -1), (8, NAN), (8, INF),
        (9, None), (9, 3 * FAKE + 1),
        (9, FAKE + 128), (9, FAKE + 99 * 128), (9, FAKE - 4 * 128 - 2), (9, 2 * FAKE + 38)])
    nothing = [None, 64, b.BF16, 100, 64, None, 8, 0, 1.0, None, None]
    assert lib.ultramem_embedding(*nothing) == b.OK


def test_embedding_backward():
    lib = b.load()
    need = lib.ultramem_embedding_backward_workspace(5, 64)
    assert need > 0
    for bad in ((-1, 64), (5, 0), (5, 65537)):
        assert lib.ultramem_embedding_backward_workspace(*bad) == 0
    ids, dout, table, ws = FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE
    good = [ids, 8, 5, dout, 64, b.BF16, 100, 64, 1.0, table, b.F32, 0, ws, need, None]
    refused(lib.ultramem_embedding_backward, good, [
        (0, None), (0, ids + 4), (1, 3), (2, -1), (3, None), (3, dout + 1), (4, 63), (5, -1),
        (6, 0), (6, (1 << 30) + 1), (7, 0), (8, NAN), (9, None), (9, table + 2), (10, 5), (11, 2),
        (11, -1), (12, None), (12, ws + 8), (13, need - 1),
        (9, dout), (9, dout + 4 * 128 + 124), (9, ids + 36), (9, ids - 100 * 256 + 4),
        (12, table), (12, table + 100 * 256 - 16), (12, dout + 4 * 128 + 112), (12, ids + 32)])
    nothing = [None, 8, 0, None, 64, b.BF16, 100, 64, 1.0, table, b.F32, 1, None, 0, None]
    assert lib.ultramem_embedding_backward(*nothing) == b.OK


def ce(**over):
    a = b.CrossEntropyArgs(FAKE, 2 * FAKE, 3 * FAKE, 64, 64, 5, 100, 64, b.BF16, 8, 1.0)
    for k, v in over.items():
        setattr(a, k, v)
    return C.byref(a)


BAD_CE = [dict(x=None), dict(w=None), dict(labels=None), dict(x=FAKE + 1), dict(w=2 * FAKE + 1),
          dict(labels=3 * FAKE + 4), dict(ld_x=63), dict(ld_w=63), dict(n_tokens=-1), dict(vocab=0),
          dict(vocab=(1 << 30) + 1), dict(dim=0), dict(dim=65537), dict(dtype=2),
          dict(labels_bytes=2), dict(logit_scale=NAN), dict(logit_scale=INF),
          dict(logit_scale=3e38), dict(n_tokens=2 ** 31 - 1, vocab=1 << 30)]


def test_cross_entropy():
    lib = b.load()
    need = lib.ultramem_cross_entropy_workspace(b.BF16, 5, 100, 64)
    back = lib.ultramem_cross_entropy_backward_workspace(b.BF16, 5, 100, 64)
    assert need > 0 and back > 0
    for f in (lib.ultramem_cross_entropy_workspace, lib.ultramem_cross_entropy_backward_workspace):
        for bad in ((2, 5, 100, 64), (1, -1, 100, 64), (1, 5, 0, 64), (1, 5, 100, 0),
                    (1, 5, 100, 65537), (1, 5, (1 << 30) + 1, 64), (1, 2 ** 31 - 1, 1 << 30, 64)):
            assert f(*bad) == 0, bad
    loss, lse, ws = 4 * FAKE, 5 * FAKE, 6 * FAKE
    good = [ce(), loss, lse, ws, need, None]
    refused(lib.ultramem_cross_entropy, good, [(0, ce(**k)) for k in BAD_CE] + [
        (0, None), (1, None), (1, loss + 2), (2, None), (2, lse + 1), (2, loss + 16), (3, None),
        (3, ws + 8), (4, need - 1), (1, FAKE), (1, 2 * FAKE + 99 * 128), (2, 3 * FAKE + 36),
        (3, FAKE), (3, 2 * FAKE), (3, 3 * FAKE), (3, loss), (3, lse + 16)])
    lib.ultramem_cross_entropy.restype = C.c_int32
    assert lib.ultramem_cross_entropy(ce(n_tokens=0), None, None, None, 0, None) == b.OK
    dloss, dx, dw, big = 5 * FAKE, 7 * FAKE, 8 * FAKE, 9 * FAKE
    good = [ce(), 4 * FAKE, dloss, dx, dw, big, back, None]
    refused(lib.ultramem_cross_entropy_backward, good, [(0, ce(**k)) for k in BAD_CE] + [
        (0, None), (1, None), (1, 4 * FAKE + 2), (2, None), (2, dloss + 1), (3, dx + 1),
        (4, dw + 1), (5, None), (5, big + 4), (6, back - 1), (3, dw), (3, dw + 99 * 128),
        (3, FAKE), (4, 2 * FAKE), (4, FAKE + 4 * 128), (3, 4 * FAKE + 16), (4, dloss),
        (3, 3 * FAKE + 32), (5, dx), (5, dw + 99 * 128 + 112), (5, FAKE), (5, dloss)])
    for dx_, dw_ in ((None, None),):        # nothing asked for
        assert lib.ultramem_cross_entropy_backward(ce(), None, None, dx_, dw_, None, 0,
                                                   None) == b.OK
    assert lib.ultramem_cross_entropy_backward(ce(n_tokens=0), None, None, None, None, None, 0,
                                               None) == b.OK


AT = dict(q=1 << 30, out=2 << 30, dout=3 << 30, k=4 << 30, v=5 << 30, dq=6 << 30, dk=7 << 30,
          dv=8 << 30, lse=9 << 30, q_start=10 << 30)
ROW = {n: 256 if n in ("q", "out", "dout", "dq") else 128 for n in AT if n not in ("lse", "q_start")}
T = 12


def attention(**over):
    a = b.AttentionGrad(**AT, **{n + "_stride": r for n, r in ROW.items()}, n_tokens=T, n_seqs=3,
                        q_heads=4, kv_heads=2, head_dim=64, dtype=b.BF16, scale=0.125)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def test_attention_gradient():
    lib = b.load()
    need = lib.ultramem_paged_attention_backward_workspace(b.BF16, T, 3, 4, 2, 64)
    assert need > 0
    for bad in ((2, T, 3, 4, 2, 64), (1, -1, 3, 4, 2, 64), (1, T, -1, 4, 2, 64), (1, T, 3, 0, 2, 64),
                (1, T, 3, 5, 2, 64), (1, T, 3, 4, 0, 64), (1, T, 3, 4, 2, 60), (1, T, 3, 4, 2, 264),
                (1, T, 3, 130, 2, 64), (1, 2 ** 31 - 1, 2 ** 31 - 1, 64, 64, 64)):
        assert lib.ultramem_paged_attention_backward_workspace(*bad) == 0, bad
    ws = 11 << 30

    def call(a, at=ws, n=need):
        return lib.ultramem_paged_attention_backward(C.byref(a), at, n, None)

    for n in AT:
        assert call(attention(**{n: None})) == b.EINVAL, n
        assert call(attention(**{n: AT[n] + 1})) == b.EINVAL, n
    for n, row in ROW.items():
        assert call(attention(**{n + "_stride": row - 1})) == b.EINVAL, n
    for bad in (dict(n_tokens=-1), dict(n_seqs=-1), dict(q_heads=3), dict(q_heads=0),
                dict(q_heads=130), dict(kv_heads=0), dict(head_dim=60), dict(head_dim=0),
                dict(head_dim=264), dict(dtype=3), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=NAN), dict(scale=INF), dict(scale=3e38)):
        assert call(attention(**bad)) == b.EINVAL, bad
    assert call(attention(), None) == b.EINVAL and call(attention(), ws + 8) == b.EINVAL
    assert call(attention(), ws, need - 1) == b.EINVAL
    assert lib.ultramem_paged_attention_backward(None, ws, need, None) == b.EINVAL
    for none in (dict(n_tokens=0), dict(n_seqs=0)):
        assert call(attention(**none)) == b.OK
    # memory that an output shares with another tensor, and the workspace with any
    size = {n: T * r * 2 for n, r in ROW.items()}
    size.update(lse=T * 4 * 4, q_start=16)
    for o in ("dq", "dk", "dv"):
        for n in AT:
            if n != o:
                for at in (AT[n], AT[n] + size[n] - 2, AT[n] - size[o] + 2):
                    assert call(attention(**{o: at})) == b.EINVAL, (o, n)
    for n in AT:
        assert call(attention(), AT[n] + (size[n] - 2) // 16 * 16) == b.EINVAL, n
        assert call(attention(), AT[n] - need // 16 * 16 + 16) == b.EINVAL, n


@pytest.mark.parametrize("call", [test_embedding, test_cross_entropy])
def test_refusals_are_the_same_twice(call):
    call()
