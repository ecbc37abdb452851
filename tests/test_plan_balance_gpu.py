"""What the plan's balance counts: the pages asked for up to the last request
that was served.  Refused requests show in kv_lens and slots, the free list's
length in free_left."""
import pytest
import torch

from paper_2411_12364_gb300.paged import paged_plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("needs,free,balance,left,served", [
    ([3, 3, 0, 5], 4, -2, 1, [1, 0, 1, 0]),   # a request of no page after a refused one
    ([3, 3], 4, 1, 1, [1, 0]),                # a refused one at the end does not count
    ([5, 5], 4, 4, 4, [0, 0]),                # none served
    ([1, 2, 0], 4, 1, 1, [1, 1, 1]),          # all served
    ([1, 5, 0, 2], 4, -2, 3, [1, 0, 1, 0]),   # -2 is not what the refused ones lack
])
def test_balance_counts_up_to_the_last_served_request(needs, free, balance, left, served,
                                                      gpu_lib):
    def i32(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    # a request of no page has one cached token and brings none
    ctx = [0 if n else 1 for n in needs]
    new = [16 * n for n in needs]
    table = torch.full((len(needs), 6), 9, dtype=torch.int32, device="cuda")
    free_left = i32([-1])
    _, kv, _, got = paged_plan(i32(ctx), i32(new), table, torch.arange(8, dtype=torch.int32,
                                                                       device="cuda"),
                               i32([free]), 16, sum(new), free_left=free_left)
    assert got.item() == balance and free_left.item() == left
    assert [int(k > 0) for k in kv.tolist()] == served
