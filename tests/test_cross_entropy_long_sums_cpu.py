"""How many terms of the cross entropy's gradient the tensor cores sum up before the
sums are joined in fp32, by the launches on imaginary devices (of 100 SMs)."""
import pytest

from tests.fake_runtime import fake_library, run  # noqa: F401
from tests.test_training_fake_cpu import CALLS


@pytest.mark.parametrize("T,V,D,joins", [
    (2560, 60000, 1280, 0),       # 10 x 5 tiles of dx for 50 pairs of SMs: no need to split
    (2560, 65536, 1280, 0),
    (2560, 65600, 1280, 1),       # sums over the vocabulary past 65536 terms
    (2560, 104000, 1280, 1),
    (140000, 1280, 2560, 1),      # sums over the tokens, 5 x 10 tiles of dw
    (60000, 1280, 2560, 0),
    (100000, 1280, 65536, 1),     # a dw whose partial sums are larger than a piece
])
def test_long_sums_are_split(fake_library, T, V, D, joins):
    run(fake_library, CALLS + f"""
M = 1 << 40                       # further apart than the largest of the tensors
assert ce_grad(T={T}, V={V}, D={D}) == b.OK
assert sum("sum_splits_kernel" in line for line in log()) == {joins}, log()
print("done")
""")
