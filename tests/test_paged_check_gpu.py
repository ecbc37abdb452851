"""The attention's error word: a wait that gave up (a probe whose barrier
nothing signals, with a limit of a few thousand cycles) is reported once, and
none is lost when another stream's check is under way."""
import pytest
import torch

from paper_2411_12364_gb300 import binding
from paper_2411_12364_gb300.paged import paged_attention, paged_check

pytestmark = pytest.mark.gpu


def test_a_timeout_is_reported_once(gpu_lib):
    assert paged_check() == binding.OK
    for _ in range(2):
        assert gpu_lib.ultramem_debug_paged_probe(binding._stream()) == binding.OK
        assert paged_check() == binding.ETIMEOUT
        assert paged_check() == binding.OK
    k = torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    ints = dict(dtype=torch.int32, device="cuda")
    out = paged_attention(torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda"), k,
                          torch.ones_like(k), torch.tensor([[2, 1]], **ints),
                          torch.tensor([0, 1], **ints), torch.tensor([20], **ints), 1)
    assert paged_check() == binding.OK and (out == 1).all()


def test_no_report_is_lost_between_streams(gpu_lib):
    side = torch.cuda.Stream()
    assert paged_check() == binding.OK
    lost = 0
    for _ in range(500):
        assert gpu_lib.ultramem_debug_paged_probe(side.cuda_stream) == binding.OK
        seen = [paged_check()]         # beside the probe, on the current stream
        side.synchronize()
        seen.append(paged_check())
        lost += binding.ETIMEOUT not in seen
        assert seen.count(binding.ETIMEOUT) <= 1
    assert lost == 0
