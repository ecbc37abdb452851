"""Scales that the attention takes: positive, and finite in fp32 after the
factor log2(e) that turns exponents to base 2 (past it a score of 0 would be
0 times infinity).  Against a runtime of imaginary devices."""
from tests.fake_runtime import fake_library, run  # noqa: F401

SCALES = """
c = b.KVCache(FAKE, FAKE, 64, 2, 16, 64, b.BF16)


def status(scale, max_new):
    need = lib.ultramem_paged_attention_workspace(b.BF16, 4, 2, 64, max_new)
    return lib.ultramem_paged_attention(C.byref(c), FAKE, 256, 4, FAKE, FAKE, FAKE, 4, 1, max_new,
                                        max_new, scale, 2 * FAKE, None, 3 * FAKE, need, None)


for max_new in (1, 64):
    for good in (1e-45, 1e-30, 0.125, 1.0, 1e30, 2.3e38):
        assert status(good, max_new) == b.OK, good
    launched = len(log())
    for bad in (2.4e38, 3.4e38, float("inf"), float("nan"), 0.0, -0.0, -1.0):
        assert status(bad, max_new) == b.EINVAL, bad
    assert len(log()) == launched
print("done")
"""


def test_scales(fake_library):  # noqa: F811
    run(fake_library, SCALES)
