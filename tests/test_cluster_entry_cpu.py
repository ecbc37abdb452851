"""A block may touch its peer's shared memory only once the peer has started,
so a kernel launched in clusters needs a rendezvous of the cluster before its
first peer store.  A store that comes too early cannot be provoked safely on a
GPU, so the order is checked in the source."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2411_12364_gb300", "csrc")


def kernel_body(file, name):
    """The text of a __global__ function without comments."""
    text = open(os.path.join(CSRC, file)).read()
    text = re.sub(r"//[^\n]*", "", text)
    at = re.search(r"\b%s\s*\(" % name, text).end()
    start, level = text.index("{", at), 0
    for end in range(start, len(text)):
        level += {"{": 1, "}": -1}.get(text[end], 0)
        if level == 0:
            return text[start:end]
    raise AssertionError(f"{name} in {file} does not end")


# file, kernel, what first reaches the peer's shared memory
@pytest.mark.parametrize("file,kernel,peer_access", [
    ("um_norm.cu", "block_norm_backward_kernel", "sum("),
    ("um_tc_gemm.cu", "tc_gemm_kernel", "bulk_copy_to_peer("),
])
def test_the_cluster_meets_before_the_first_peer_access(file, kernel, peer_access):
    before = kernel_body(file, kernel).split(peer_access)[0]
    assert peer_access in kernel_body(file, kernel)
    meets = before.rfind("cluster_wait()") > before.rfind("cluster_arrive") >= 0
    assert meets or "cluster_sync()" in before, f"{kernel} may reach a peer that has not started"
