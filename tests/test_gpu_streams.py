"""Results and buffers of calls on streams other than the current one, and calls on several streams at a time."""
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


def test_prompt_layers_on_another_stream():
    """A handle's buffers of its first call, made while the current stream is busy with memory it has given up; hidden
    states of another width; the current stream again."""
    H, G, d, n = 8, 2, 64, [70, 40]
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: (torch.randn(*s, generator=gen, device="cuda") * s[-1] ** -0.5).bfloat16()  # noqa: E731
    dims = abi.GqaDims(H, G, d, d ** -0.5)
    cache = abi.Cache(*(torch.zeros(2 * G, 128, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)), 128)
    cu, start, kv = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 70, 110], [0, 0], n))
    work = [(new(110, D), *(new(m * d, D) for m in (H, G, G)), new(D, H * d)) for D in (512, 896)]
    make = lambda: abi.GqaPrompt(dims, cache, 2, 110, 128)  # noqa: E731
    want = [make().from_hidden(*w, cu, start, kv).clone() for w in work]
    side, step = torch.cuda.Stream(), make()
    torch.cuda.synchronize()
    scratch = [torch.empty(110, m, dtype=torch.bfloat16, device="cuda") for m in (H * d, G * d, G * d, 512, 896) for _ in range(3)]
    torch.cuda._sleep(20_000_000)
    for s in scratch:
        s.fill_(7)
    del scratch, s
    got = [step.from_hidden(*w, cu, start, kv, stream=side) for w in work + work[:1]]
    torch.cuda.synchronize()
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[0])
    assert torch.equal(step.from_hidden(*work[1], cu, start, kv), want[1])
    assert abi.check_status() == abi.MLA_OK


def test_two_pools_and_two_layers_at_a_time():
    """Calls on two streams that nothing orders among one another: each pool ends as its own rules say, each handle's
    results are those that it has alone."""
    from tests.test_gpu_pages import Model
    from tests.test_gpu_prompt import Layer, cu_of, i32

    n, kv = [150, 3, 90], [4000, 60, 1500]
    layers = [Layer(14, 2, 64, kv, True, seed=50 + i) for i in range(2)]
    q = [L.normal(sum(n), 14, 64) for L in layers]
    steps = [abi.GqaPrompt(L.dims, L.cache, 3, sum(n), 4000) for L in layers]
    cu, lens = cu_of(n), i32(kv)
    want = [(s.attend(x, cu, lens).clone(), s.lse.clone()) for s, x in zip(steps, q)]
    pools = [Model(30, 2, 9, 500, (64, 64), 2, seed=52 + i) for i in range(2)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for turn in range(6):
        for i, side in enumerate(sides):
            with torch.cuda.stream(side):
                m = pools[i]
                m.reserve([turn], [100 + 60 * turn + i])
                m.fork([turn] * 3, [10 + 3 * turn, 11 + 3 * turn, 12 + 3 * turn], [100, 90 + 60 * turn, 64])
                got[i] = steps[i].attend(q[i], cu, lens)
                if turn % 2:
                    m.release([turn - 1, 10 + 3 * turn], [0, 0])
                    m.compact()
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(got[i], want[i][0]) and torch.equal(steps[i].lse, want[i][1])
        pools[i].check()
