"""Results and buffers of calls on streams other than the current one."""
from __future__ import annotations

import pytest
import torch

from paper_2607_27269_gb300 import abi

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("raw", [False, True])
def test_results_written_on_another_stream(raw):
    """Work that the current stream still has queued on memory that it has given up does not reach the results, and the
    other way round."""
    x = torch.randn(50, 5000, device="cuda")
    t = torch.arange(50, dtype=torch.int32, device="cuda")
    want = [v.clone() for v in abi.token_logprobs(x, t, 7)]
    alpha = abi.acceptance_stats(x, x.flip(0).contiguous())[0].clone()
    y = x.flip(0).contiguous()
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side
    torch.cuda.synchronize()
    for _ in range(3):
        scratch = [torch.empty(v.shape, dtype=v.dtype, device="cuda") for v in want for _ in range(4)]
        torch.cuda._sleep(20_000_000)  # (ten milliseconds of the current stream, during which the side stream works)
        for s in scratch:
            s.fill_(7)
        del scratch, s
        got = abi.token_logprobs(x, t, 7, stream=stream)
        got_alpha = abi.acceptance_stats(x, y, stream=stream)[0]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(got_alpha, alpha)
    assert abi.check_status() == abi.MLA_OK
