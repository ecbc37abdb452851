"""The forms that a vocabulary in pieces takes, by the launches on imaginary devices:
the cases of the comparison with 64 bits reach each of them."""
import pytest

from tests.fake_runtime import fake_library, run  # noqa: F401
from tests.test_cross_entropy_pieces_gpu import CASES
from tests.test_training_fake_cpu import CALLS


@pytest.mark.parametrize("T,V,D,piece", CASES)
def test_cases_have_several_pieces(fake_library, T, V, D, piece):
    """Logits, dx and dw a piece; more bytes: one piece."""
    run(fake_library, CALLS + f"""
def products():
    return sum("gemm_kernel" in line for line in log())


lib.ultramem_debug_cross_entropy_piece.argtypes = [C.c_int64]
for dtype in (b.BF16, b.F32):
    lib.fake_reset(0)
    assert ce_grad(dtype, {T}, {V}, {D}) == b.OK and products() == 3
    assert lib.ultramem_debug_cross_entropy_piece({piece}) == b.OK
    lib.fake_reset(0)
    assert ce_grad(dtype, {T}, {V}, {D}) == b.OK
    assert products() >= 6 and products() % 3 == 0
    lib.fake_reset(0)
    rows = max(256, {piece} // (-(-{D} // 64) * 64 * 6) // 256 * 256)   # rearranged weights
    assert ce(b.F32, {T}, {V}, {D}) == b.OK and (products() >= 2) == ({V} > rows)
    assert lib.ultramem_debug_cross_entropy_piece(0) == b.OK
    lib.fake_reset(0)
    assert ce_grad(dtype, {T}, {V}, {D}) == b.OK and products() == 3
assert lib.ultramem_debug_cross_entropy_piece(-1) == b.EINVAL
print("done")
""")
