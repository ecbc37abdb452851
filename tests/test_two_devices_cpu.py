"""The decoder-block entry points in a process that uses two GPUs, and after a
call of the runtime that failed: against a runtime of two imaginary devices,
which refuses a launch whose shared memory was not allowed on the current
device."""
import pytest

from tests.fake_runtime import fake_library, run  # noqa: F401


def test_calls_on_a_second_device(fake_library):
    run(fake_library, """
for device in (0, 1, 0):
    lib.fake_reset(device)
    for name, call in CALLS.items():
        assert call() == b.OK, (device, name)
print("done")
""")


def test_each_device_has_its_error_word(fake_library):
    run(fake_library, """
words = []
for device in (0, 1, 0):
    lib.fake_reset(device)
    assert lib.ultramem_paged_check(None) == b.OK
    words.append({line.split()[2] for line in log() if line.startswith(("copy", "memset"))})
assert words[0] == words[2] and words[0].isdisjoint(words[1]) and words[1]
print("done")
""")


def test_workspaces_follow_the_device(fake_library):
    run(fake_library, """
sizes = []
for device in (0, 1):
    lib.fake_reset(device)
    sizes.append(lib.ultramem_paged_attention_workspace(b.BF16, 4, 2, 128, 1))
assert sizes[1] > sizes[0]     # more SMs
assert attend() == b.OK
lib.fake_reset(0)
assert attend() == b.OK
print("done")
""")


@pytest.mark.parametrize("failing", [
    "cudaFuncSetAttribute", "cudaOccupancyMaxActiveBlocksPerMultiprocessor",
    "cudaGetSymbolAddress", "cudaGetDriverEntryPointByVersion", "cudaDeviceGetAttribute",
    "launch"])
def test_a_failed_first_call_is_not_kept(fake_library, failing):
    """A call of the runtime that fails once fails at most that call."""
    run(fake_library, f"""
for name, call in CALLS.items():
    lib.fake_fail_once(b"{failing}")
    call()
    lib.fake_fail_once(b"")
    assert call() == b.OK, name
print("done")
""")
