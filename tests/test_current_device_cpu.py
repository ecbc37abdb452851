"""The decoder-block functions launch on the current device's stream, so every
tensor has to lie on that device: stand-in tensors that name a device, a
stand-in library that records calls, no GPU."""
import pytest
import torch

from paper_2411_12364_gb300 import binding, norms, paged


class On(torch.Tensor):
    """A CPU tensor that says it is on a CUDA device."""
    index = 0

    @property
    def is_cuda(self):
        return self.index >= 0

    def get_device(self):
        return self.index


def on(index, *shape, dtype=torch.bfloat16):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(On)
    t.index = index
    return t


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("workspace"):
                return 64
            self.calls.append((name, args[-1]))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(binding, "_lib", r)
    monkeypatch.setattr(binding, "load", lambda: r)
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for module in (norms, paged):
        module._workspace.cache_clear()
    yield r
    for module in (norms, paged):
        module._workspace.cache_clear()


I32 = torch.int32


def plan_args():
    return dict(ctx_lens=((2,), I32), new_lens=((2,), I32), block_table=((2, 4), I32),
                free_pages=((8,), I32), free_count=((1,), I32), free_left=((1,), I32))


def append_args():
    return dict(k_cache=((4, 2, 16, 64),), v_cache=((4, 2, 16, 64),), k=((3, 2, 64),),
                v=((3, 2, 64),), slots=((3,), I32))


def attention_args():
    return dict(q=((3, 4, 64),), k_cache=((4, 2, 16, 64),), v_cache=((4, 2, 16, 64),),
                block_table=((2, 4), I32), q_start=((3,), I32), kv_lens=((2,), I32),
                out=((3, 4, 64),))


F32 = torch.float32


def norm_args():
    vector = ((64,), F32)
    return dict(y=((3, 64),), residual=((3, 64),), w_post=vector, b_post=vector, w_pre=vector,
                b_pre=vector, gate=vector, u=((3, 64),), n=((3, 64),))


def grad_args():
    vector = ((64,), F32)
    return dict(y=((3, 64),), u=((3, 64),), du=((3, 64),), dn=((3, 64),), w_post=vector,
                b_post=vector, w_pre=vector, b_pre=vector, gate=((3, 1),))


CASES = [
    (paged.paged_plan, plan_args, dict(page_size=16, n_tokens=3)),
    (paged.paged_append, append_args, {}),
    (paged.paged_attention, attention_args, dict(max_new=2)),
    (norms.block_norm, norm_args, dict(kind="layer")),
    (norms.block_norm_backward, grad_args, dict(kind="layer")),
]


def call(f, shapes, numbers, index, other=None):
    made = {}
    for name, (shape, *dtype) in shapes().items():
        made[name] = on(1 - index if name == other else index, *shape,
                        **(dict(dtype=dtype[0]) if dtype else {}))
    return f(**made, **numbers)


@pytest.mark.parametrize("f,shapes,numbers", CASES, ids=lambda x: getattr(x, "__name__", ""))
def test_tensors_lie_on_the_current_device(f, shapes, numbers, lib, monkeypatch):
    call(f, shapes, numbers, 0)
    assert [s for _, s in lib.calls] == [1000]
    lib.calls.clear()
    for name in shapes():                # one of them elsewhere
        with pytest.raises(ValueError):
            call(f, shapes, numbers, 0, other=name)
    with pytest.raises(ValueError):      # all of them
        call(f, shapes, numbers, 1)
    with pytest.raises(ValueError):      # host tensors
        call(f, shapes, numbers, -1)
    assert not lib.calls
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    call(f, shapes, numbers, 1)
    assert [s for _, s in lib.calls] == [1001]
