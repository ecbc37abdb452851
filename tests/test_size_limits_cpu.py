"""Sizes that reach 2^31: what the Python functions would cut to 32 bits is
refused, and the longest request's key numbers stay below 2^31, also those of
the block that a kernel looks at ahead of the last one."""
import os
import re

import pytest
import torch

from paper_2411_12364_gb300 import norms, paged
from tests.test_current_device_cpu import I32, lib, on  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BIG = 2 ** 31


def test_sizes_past_32_bits_are_refused(lib):  # noqa: F811
    ints = [on(0, n, dtype=I32) for n in (2, 2)]
    table, pages, count = on(0, 2, 4, dtype=I32), on(0, 8, dtype=I32), on(0, 1, dtype=I32)
    for page_size, n_tokens in ((16, BIG), (16, 2 ** 32 + 5), (2 ** 32 + 16, 5)):
        with pytest.raises(ValueError):
            paged.paged_plan(*ints, table, pages, count, page_size, n_tokens)
    q, k = on(0, 3, 4, 64), on(0, 4, 2, 16, 64)
    for max_new in (BIG, 2 ** 32 + 1):
        with pytest.raises(ValueError):
            paged.paged_attention(q, k, k, table, on(0, 3, dtype=I32), ints[0], max_new)
    for rows in (BIG, 2 ** 32 + 3):   # stride 0: a row of memory
        y = on(0, 1, 1).expand(rows, 1)
        y.index = 0
        for call in (lambda: norms.block_norm(y, y), lambda: norms.block_norm_backward(y, y, y, y)):
            with pytest.raises(ValueError):
                call()
    assert not lib.calls


def constant(name):
    text = open(os.path.join(ROOT, "paper_2411_12364_gb300", "csrc", "um_paged.cuh")).read()
    found = re.search(r"constexpr int %s = ([^;]+);" % name, text)
    assert found, f"{name} is not there"
    return eval(found.group(1).replace("INT32_MAX", str(BIG - 1)))


@pytest.mark.parametrize("block", [32, 64, 128])
def test_key_numbers_of_the_longest_request(block):
    """A producer reads the table for block j + 1 while it copies block j: the
    number of every key that it asks for, past the last block's end too, fits
    an int, so that none turns negative and passes for a key in range."""
    most = constant("kMaxKeys")
    assert most % 256 == 0                       # whole blocks and pages
    for kv in (most, most - 1, most - block, most - block + 1):
        blocks = -(-kv // block)
        assert kv + block - 1 < BIG              # the sum that the count is taken from
        last = (blocks - 1) * block + block - 1  # of the last block
        assert last + block < BIG                # and of the one after it
        assert torch.tensor(last + block, dtype=torch.int32).item() >= kv
