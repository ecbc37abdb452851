"""The Python functions of the embedding, the cross entropy and the attention's
gradient: tensors of the current device, shapes, types and sizes, with stand-in
tensors and a stand-in library."""
import pytest
import torch

from paper_2411_12364_gb300 import paged, vocab
from tests.test_current_device_cpu import call, lib, on  # noqa: F401

BF16, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
BIG = 2 ** 31


@pytest.fixture
def calls(lib):  # noqa: F811
    for f in (vocab._workspace, paged._grad_workspace):
        f.cache_clear()
    yield lib
    for f in (vocab._workspace, paged._grad_workspace):
        f.cache_clear()


def embedding_args():
    return dict(table=((9, 64),), ids=((3,), I64), out=((3, 64),))


def embedding_grad_args():
    return dict(ids=((3,), I32), dout=((3, 64),), dtable=((9, 64), F32))


def ce_args():
    return dict(x=((3, 64),), w=((9, 64),), labels=((3,), I64))


def ce_grad_args():
    return dict(ce_args(), lse=((3,), F32), dloss=((3,), F32), dx=((3, 64),), dw=((9, 64),))


def attention_args():
    rows, keys = ((3, 4, 64),), ((3, 2, 64),)
    return dict(q=rows, k=keys, v=keys, out=rows, lse=((3, 4), F32), dout=rows, q_start=((3,), I32),
                dq=rows, dk=keys, dv=keys)


CASES = [(vocab.embedding, embedding_args, {}),
         (vocab.embedding_backward, embedding_grad_args, dict(vocab=9)),
         (vocab.cross_entropy, ce_args, {}),
         (vocab.cross_entropy_backward, ce_grad_args, {}),
         (paged.paged_attention_backward, attention_args, {})]


@pytest.mark.parametrize("f,shapes,numbers", CASES, ids=lambda x: getattr(x, "__name__", ""))
def test_tensors_lie_on_the_current_device(f, shapes, numbers, calls, monkeypatch):
    call(f, shapes, numbers, 0)
    assert [s for _, s in calls.calls] == [1000]
    calls.calls.clear()
    for name in shapes():                # one of them elsewhere
        with pytest.raises(ValueError):
            call(f, shapes, numbers, 0, other=name)
    for index in (1, -1):                # all of them, and host tensors
        with pytest.raises(ValueError):
            call(f, shapes, numbers, index)
    assert not calls.calls
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    call(f, shapes, numbers, 1)
    assert [s for _, s in calls.calls] == [1001]


@pytest.mark.parametrize("f,shapes,numbers", CASES, ids=lambda x: getattr(x, "__name__", ""))
def test_types_and_shapes(f, shapes, numbers, calls):
    for name, (shape, *dtype) in shapes().items():
        bads = [(*shape, 2)]
        if name != "q_start":            # any number of sequences is fine
            bads.append(shape[:-1] + (shape[-1] + 1,))
        if name not in ("table", "w", "q_start"):   # an empty vocabulary is the library's to refuse
            bads.append((0,) + shape[1:])
        for bad in bads:
            with pytest.raises(ValueError):
                call(f, lambda: dict(shapes(), **{name: (bad, *dtype)}), numbers, 0)
        with pytest.raises(ValueError):
            call(f, lambda: dict(shapes(), **{name: (shape, torch.float16)}), numbers, 0)
    assert not calls.calls


def test_outputs_are_contiguous(calls):
    wide = on(0, 3, 128)[:, :64]
    for f in (lambda: vocab.embedding(on(0, 9, 64), on(0, 3, dtype=I64), out=wide),
              lambda: vocab.embedding_backward(on(0, 3, dtype=I64), on(0, 3, 64), 3, dtable=wide),
              lambda: vocab.cross_entropy_backward(
                  on(0, 3, 64), on(0, 9, 64), on(0, 3, dtype=I64), on(0, 3, dtype=F32),
                  on(0, 3, dtype=F32), dx=wide)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ValueError):      # nothing to add to
        vocab.embedding_backward(on(0, 3, dtype=I64), on(0, 3, 64), 9, accumulate=True)
    with pytest.raises(ValueError):
        vocab.embedding_backward(on(0, 3, dtype=I64), on(0, 3, 64), 0)
    with pytest.raises(ValueError):      # ids apart
        vocab.embedding(on(0, 9, 64), on(0, 6, dtype=I64)[::2])
    assert not calls.calls


def test_rows_apart_keep_their_distance(calls):
    """Slices of one projection's output go to the library as they are."""
    qkv = on(0, 3, 8, 64)
    grads = on(0, 3, 8, 64)
    rows = on(0, 3, 4, 64)
    paged.paged_attention_backward(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], rows, on(0, 3, 4, dtype=F32),
                                   rows, on(0, 3, dtype=I32), dq=grads[:, :4], dk=grads[:, 4:6],
                                   dv=grads[:, 6:])
    assert [n for n, _ in calls.calls] == ["ultramem_paged_attention_backward"]
    with pytest.raises(ValueError):      # an output whose heads are apart
        paged.paged_attention_backward(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], rows,
                                       on(0, 3, 4, dtype=F32), rows, on(0, 3, dtype=I32),
                                       dq=on(0, 4, 3, 64).transpose(0, 1))


def test_sizes_past_32_bits_are_refused(calls):
    ids = on(0, 3, dtype=I64)
    with pytest.raises(ValueError):
        vocab.embedding_backward(ids, on(0, 3, 64), BIG)
    tall = on(0, 1, 64).expand(BIG, 64)      # a row of memory
    tall.index = 0
    for f in (lambda: vocab.embedding(tall, ids),
              lambda: vocab.cross_entropy(on(0, 3, 64), tall, ids)):
        with pytest.raises(ValueError):
            f()
    assert not calls.calls
