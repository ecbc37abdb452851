"""The check of the attention's error word reads and clears it in one step on
the GPU: between a copy of the word and a separate clearing of it, a kernel of
another stream could record a timeout that nobody sees.  Against a runtime of
imaginary devices."""
from tests.fake_runtime import fake_library, run  # noqa: F401

CHECK = """
assert lib.ultramem_paged_check(None) == b.OK          # finds the words
for device in (0, 1):
    lib.fake_reset(device)
    assert lib.ultramem_paged_check(None) == b.OK
    calls = [line.split() for line in log() if not line.startswith("symbol")]
    assert [c[0] for c in calls] == ["launch", "copy"], calls
    assert "take_error" in calls[0][2]
lib.fake_reset(0)
lib.fake_fail_once(b"launch")
assert lib.ultramem_paged_check(None) not in (b.OK, b.ETIMEOUT)
assert not any(line.startswith("copy") for line in log())
assert lib.ultramem_paged_check(None) == b.OK
print("done")
"""


def test_the_word_is_read_and_cleared_in_one_step(fake_library):  # noqa: F811
    run(fake_library, CHECK)
