"""Argument checks of the decoder-block entry points: what they refuse, they
refuse before anything is launched (no device needed)."""
import ctypes as C

import pytest

from paper_2411_12364_gb300 import binding

FAKE = 4096    # never dereferenced


def _cache(**over):
    c = binding.KVCache(FAKE, FAKE, 8, 2, 16, 64, binding.BF16)
    for k, v in over.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [dict(k=None), dict(v=None), dict(k=4104), dict(v=4098), dict(n_pages=0),
              dict(n_pages=1 << 28), dict(kv_heads=0), dict(kv_heads=2000), dict(page_size=8),
              dict(page_size=24), dict(page_size=512), dict(head_dim=0), dict(head_dim=60),
              dict(head_dim=264), dict(dtype=2)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_invalid_caches_are_refused(bad):
    lib = binding.load()
    c = _cache(**bad)
    assert lib.ultramem_paged_append(C.byref(c), FAKE, 128, FAKE, 128, FAKE, 1,
                                     None) == binding.EINVAL
    assert lib.ultramem_paged_attention(C.byref(c), FAKE, 256, 4, FAKE, FAKE, FAKE, 4, 1, 1, 1,
                                        1.0, FAKE, None, FAKE, 1 << 40, None) == binding.EINVAL


def test_plan_arguments():
    lib = binding.load()
    good = [FAKE, 2 * FAKE, 2, 16, 3 * FAKE, 4, 4 * FAKE, 5 * FAKE, 7, 8, 6 * FAKE, 7 * FAKE,
            8 * FAKE, 9 * FAKE, 10 * FAKE, None]
    for at, bad in ((0, None), (1, None), (2, -1), (3, 0), (3, 17), (4, None), (5, -1), (6, None),
                    (7, None), (8, -1), (9, -1), (10, None), (11, None), (11, FAKE), (12, None),
                    (13, 5 * FAKE), (14, None), (14, 5 * FAKE), (14, 9 * FAKE)):
        args = list(good)
        args[at] = bad
        assert lib.ultramem_paged_plan(*args) == binding.EINVAL, (at, bad)


def test_append_arguments():
    lib = binding.load()
    c = _cache()
    good = [C.byref(c), FAKE, 128, FAKE, 128, FAKE, 4, None]
    for at, bad in ((0, None), (1, None), (1, 4097), (2, 127), (3, None), (4, 64), (5, None),
                    (6, -1)):
        args = list(good)
        args[at] = bad
        assert lib.ultramem_paged_append(*args) == binding.EINVAL, (at, bad)
    args = list(good)
    args[6] = 0
    assert lib.ultramem_paged_append(*args) == binding.OK


def test_attention_arguments():
    lib = binding.load()
    c = _cache()
    need = lib.ultramem_paged_attention_workspace(binding.BF16, 4, 2, 64, 1)
    assert need > 0
    good = [C.byref(c), FAKE, 256, 4, FAKE, FAKE, FAKE, 4, 1, 1, 1, 1.0, FAKE, None, FAKE, need,
            None]
    for at, bad in ((0, None), (1, None), (1, 4097), (2, 255), (3, 0), (3, 3), (3, 130), (4, None),
                    (5, None), (6, None), (7, -1), (8, -1), (9, -1), (10, -1), (11, 0.0),
                    (11, -1.0), (11, float("nan")), (11, float("inf")), (12, None), (14, None),
                    (14, 4100), (15, need - 1)):
        args = list(good)
        args[at] = bad
        assert lib.ultramem_paged_attention(*args) == binding.EINVAL, (at, bad)
    for at in (8, 9, 10):    # nothing to do
        args = list(good)
        args[at] = 0
        assert lib.ultramem_paged_attention(*args) == binding.OK
    for bad in ((2, 4, 2, 64, 1), (1, 3, 2, 64, 1), (1, 4, 0, 64, 1), (1, 4, 2, 63, 1),
                (1, 4, 2, 264, 1), (1, 4, 2, 64, -1), (1, 260, 2, 64, 1)):
        assert lib.ultramem_paged_attention_workspace(*bad) == 0


def _norm_args(**over):
    a = binding.BlockNormArgs(FAKE, None, None, None, None, None, 64, 64, 4, 64, binding.BF16, 0,
                              1, 1, 0, 1.0, 1.0, 1e-5)
    for k, v in over.items():
        setattr(a, k, v)
    return a


BAD_NORMS = [dict(y=None), dict(n_tokens=-1), dict(dim=0), dict(dim=8193), dict(dtype=2),
             dict(kind=2), dict(post=2), dict(pre=-1), dict(gate_mode=1), dict(gate=FAKE),
             dict(gate_mode=4, gate=FAKE), dict(eps=-1.0), dict(eps=float("nan")),
             dict(res_scale=float("nan")), dict(out_scale=float("inf")), dict(b_post=FAKE),
             dict(b_pre=FAKE), dict(ld_y=63), dict(ld_r=63)]


@pytest.mark.parametrize("bad", BAD_NORMS)
def test_invalid_norm_arguments_are_refused(bad):
    lib = binding.load()
    a = _norm_args(**bad)
    assert lib.ultramem_block_norm(C.byref(a), FAKE, FAKE, FAKE, None) == binding.EINVAL
    assert lib.ultramem_block_norm_backward(
        C.byref(a), FAKE, FAKE, 64, FAKE, 64, FAKE, FAKE, None, None, None, None, None, FAKE,
        1 << 30, None) == binding.EINVAL


def test_norm_pointers():
    lib = binding.load()
    a = _norm_args()
    assert lib.ultramem_block_norm(None, FAKE, FAKE, FAKE, None) == binding.EINVAL
    assert lib.ultramem_block_norm(C.byref(a), None, FAKE, FAKE, None) == binding.EINVAL
    assert lib.ultramem_block_norm(C.byref(a), FAKE, None, FAKE, None) == binding.EINVAL
    assert lib.ultramem_block_norm(C.byref(a), FAKE, FAKE, None, None) == binding.EINVAL
    off = _norm_args(pre=0)
    assert lib.ultramem_block_norm(C.byref(off), FAKE, FAKE, FAKE, None) == binding.EINVAL
    none = _norm_args(n_tokens=0)
    assert lib.ultramem_block_norm(C.byref(none), None, None, None, None) == binding.OK


def test_norm_backward_pointers():
    lib = binding.load()
    need = lib.ultramem_block_norm_backward_workspace(4, 64)
    assert need > 0
    assert lib.ultramem_block_norm_backward_workspace(4, 0) == 0
    assert lib.ultramem_block_norm_backward_workspace(-1, 64) == 0
    a = _norm_args()
    good = [C.byref(a), FAKE, FAKE, 64, FAKE, 64, FAKE, FAKE, None, FAKE, None, FAKE, None, FAKE,
            need, None]
    for at, bad in ((0, None), (1, None), (3, 63), (4, None), (5, 63), (8, FAKE), (10, FAKE),
                    (12, FAKE), (13, None), (13, 4100), (14, need - 1)):
        args = list(good)
        args[at] = bad
        assert lib.ultramem_block_norm_backward(*args) == binding.EINVAL, (at, bad)
    off = _norm_args(post=0)   # no first norm: no gradient of its gain
    args = list(good)
    args[0] = C.byref(off)
    assert lib.ultramem_block_norm_backward(*args) == binding.EINVAL


@pytest.mark.parametrize("dtype,es", [(binding.BF16, 2), (binding.F32, 4)])
def test_norm_pointers_inside_an_entry(dtype, es):
    lib = binding.load()
    need = lib.ultramem_block_norm_backward_workspace(4, 64)
    a = _norm_args(dtype=dtype)
    for at in (1, 2, 3):
        args = [C.byref(a), FAKE, FAKE, FAKE, None]
        args[at] = FAKE + es // 2
        assert lib.ultramem_block_norm(*args) == binding.EINVAL, at
    good = [C.byref(a), FAKE, FAKE, 64, FAKE, 64, FAKE, FAKE, None, FAKE, None, FAKE, None, FAKE,
            need, None]
    for at in (1, 2, 4, 6, 7):
        args = list(good)
        args[at] = FAKE + es // 2
        assert lib.ultramem_block_norm_backward(*args) == binding.EINVAL, at
    for at in (9, 11):       # fp32 whatever the rows are
        args = list(good)
        args[at] = FAKE + 2
        assert lib.ultramem_block_norm_backward(*args) == binding.EINVAL, at
    for name in ("y", "w_post", "w_pre"):
        off = _norm_args(dtype=dtype, **{name: FAKE + (es // 2 if name == "y" else 2)})
        assert lib.ultramem_block_norm(C.byref(off), FAKE, FAKE, FAKE, None) == binding.EINVAL
        args = [C.byref(off)] + good[1:]
        assert lib.ultramem_block_norm_backward(*args) == binding.EINVAL, name
    for mode, shift in ((1, 2), (2, es // 2), (3, es // 2)):
        off = _norm_args(dtype=dtype, gate_mode=mode, gate=FAKE + shift)
        assert lib.ultramem_block_norm(C.byref(off), FAKE, FAKE, FAKE, None) == binding.EINVAL
        off = _norm_args(dtype=dtype, gate_mode=mode, gate=FAKE)
        args = [C.byref(off)] + good[1:]
        args[8] = FAKE + shift
        assert lib.ultramem_block_norm_backward(*args) == binding.EINVAL, mode
