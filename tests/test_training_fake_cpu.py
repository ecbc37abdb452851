"""The embedding, the cross entropy and the attention's gradient against a
runtime of imaginary devices: what shares memory and is accepted, calls on a
second device, after a failed call of the runtime, and where the waits that
give up are recorded."""
import pytest

from tests.fake_runtime import fake_library, run  # noqa: F401

CALLS = """
M = 1 << 30


def embed(dtype=b.BF16):
    return lib.ultramem_embedding(M, 64, dtype, 100, 64, 2 * M, 8, 5, 1.0, 3 * M, None)


def embed_grad(T=5, accumulate=0):
    need = lib.ultramem_embedding_backward_workspace(T, 64)
    return lib.ultramem_embedding_backward(M, 8, T, 2 * M, 64, b.BF16, 100, 64, 1.0, 3 * M, b.BF16,
                                           accumulate, 4 * M, need, None)


def ce(dtype=b.BF16, T=300, V=5000, D=64):
    a = b.CrossEntropyArgs(M, 2 * M, 3 * M, D, D, T, V, D, dtype, 8, 1.0)
    need = lib.ultramem_cross_entropy_workspace(dtype, T, V, D)
    return lib.ultramem_cross_entropy(C.byref(a), 4 * M, 5 * M, 6 * M, need, None)


def ce_grad(dtype=b.BF16, T=300, V=5000, D=64):
    a = b.CrossEntropyArgs(M, 2 * M, 3 * M, D, D, T, V, D, dtype, 8, 1.0)
    need = lib.ultramem_cross_entropy_backward_workspace(dtype, T, V, D)
    return lib.ultramem_cross_entropy_backward(C.byref(a), 4 * M, 5 * M, 6 * M, 7 * M, 8 * M, need,
                                               None)


def attn_grad(dtype=b.BF16, dim=128, stride=None, **at):
    h, k = stride or 4 * dim, stride or 2 * dim
    p = dict(dict(q=M, out=2 * M, dout=3 * M, k=4 * M, v=5 * M, dq=6 * M, dk=7 * M, dv=8 * M,
                  lse=9 * M, q_start=10 * M), **at)
    a = b.AttentionGrad(**p, q_stride=h, out_stride=4 * dim, dout_stride=4 * dim, k_stride=k,
                        v_stride=k, dq_stride=h, dk_stride=k, dv_stride=k, n_tokens=200, n_seqs=3,
                        q_heads=4, kv_heads=2, head_dim=dim, dtype=dtype, scale=1.0)
    need = lib.ultramem_paged_attention_backward_workspace(dtype, 200, 3, 4, 2, dim)
    return lib.ultramem_paged_attention_backward(C.byref(a), 11 * M, need, None)


TRAINING = dict(embed=embed, embed_grad=embed_grad, add=lambda: embed_grad(accumulate=1),
                long=lambda: embed_grad(T=100000), ce=ce, ce32=lambda: ce(b.F32),
                odd=lambda: ce(D=63), ce_grad=ce_grad, grad32=lambda: ce_grad(b.F32),
                pieces=lambda: ce_grad(T=30000, V=50000), attn=attn_grad,
                narrow=lambda: attn_grad(dim=64), attn32=lambda: attn_grad(b.F32),
                wide=lambda: attn_grad(dim=256))
"""


def test_calls_on_a_second_device(fake_library):
    run(fake_library, CALLS + """
for device in (0, 1, 0):
    lib.fake_reset(device)
    for name, call in TRAINING.items():
        before = len(log())
        assert call() == b.OK, (device, name)
        assert sum(l.startswith("launch") for l in log()[before:]) > 0, name
print("done")
""")


@pytest.mark.parametrize("failing", [
    "cudaFuncSetAttribute", "cudaGetSymbolAddress", "cudaGetDriverEntryPointByVersion",
    "cudaDeviceGetAttribute", "launch"])
def test_a_failed_first_call_is_not_kept(fake_library, failing):
    """A call of the runtime that fails once fails at most that call."""
    run(fake_library, CALLS + f"""
for name, call in TRAINING.items():
    lib.fake_fail_once(b"{failing}")
    call()
    lib.fake_fail_once(b"")
    assert call() == b.OK, name
print("done")
""")


def test_slices_of_one_tensor(fake_library):
    """q, k and v, and dq, dk and dv, between one another's rows; not over them."""
    run(fake_library, CALLS + """
D, row = 128, 8 * 128
ins = dict(q=M, k=M + 4 * D * 2, v=M + 6 * D * 2)
outs = dict(dq=6 * M, dk=6 * M + 4 * D * 2, dv=6 * M + 6 * D * 2)
assert attn_grad(stride=row, **ins, **outs) == b.OK
launched = len(log())
for name, at in outs.items():
    for step in (-2, 2):
        assert attn_grad(stride=row, **ins, **dict(outs, **{name: at + step})) == b.EINVAL, name
    # the gradient in its input's place
    assert attn_grad(stride=row, **ins, **dict(outs, **{name: ins[name[1:]]})) == b.EINVAL
assert len(log()) == launched
print("done")
""")


def test_zeros_without_tokens(fake_library):
    run(fake_library, CALLS + """
lib.fake_reset(0)
assert lib.ultramem_embedding_backward(None, 8, 0, None, 64, b.BF16, 100, 64, 1.0, 3 * M, b.F32, 0,
                                       None, 0, None) == b.OK
a = b.CrossEntropyArgs(None, None, None, 64, 64, 0, 100, 64, b.BF16, 8, 1.0)
assert lib.ultramem_cross_entropy_backward(C.byref(a), None, None, None, 7 * M, None, 0,
                                           None) == b.OK
assert [l.split()[0] for l in log()] == ["memset", "memset"]
assert "bytes=%d" % (100 * 64 * 4) in log()[0] and "bytes=%d" % (100 * 64 * 2) in log()[1]
print("done")
""")


def test_pieces_bound_the_workspace(fake_library):
    """However long the vocabulary is, G and rearranged weights take a piece."""
    run(fake_library, CALLS + """
for dtype in (b.BF16, b.F32):
    for T, D in ((1000, 512), (20000, 1000)):
        sizes = [lib.ultramem_cross_entropy_backward_workspace(dtype, T, V, D)
                 for V in (1 << 17, 1 << 20, 1 << 23)]
        assert max(sizes) < 4 * (512 << 20) + 20 * T * D, sizes
print("done")
""")
