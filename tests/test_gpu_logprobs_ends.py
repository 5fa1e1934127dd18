"""mla_token_logprobs at the ends of what logits can be."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2607_27269_gb300 import abi

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [9, 5000, 70000])
def test_logits_as_large_as_the_type_holds(vocab, dtype):
    """A token forced by a logit near the type's largest: probability 1, entropy 0, wherever it stands; two such tokens
    share it."""
    big = torch.finfo(dtype).max
    places = [0, 1, vocab // 2, vocab - 1]
    x = torch.randn(len(places) + 3, vocab, device="cuda").to(dtype)
    for r, at in enumerate(places):
        x[r, at] = big
    x[4, 3] = x[4, vocab - 2] = big
    x[5, 2] = 2.5e38
    x[5, 5:] = torch.finfo(dtype).min
    x[6, 4] = big
    x[6, 5:] = -math.inf
    t = torch.tensor(places + [3, 2, 4], dtype=torch.int32, device="cuda")
    lse = torch.empty(7, device="cuda")
    lp, ent, idx, top = abi.token_logprobs(x, t, 2, lse=lse)
    assert abi.check_status() == abi.MLA_OK
    # e^0 is exact, everything else underflows: ln 1 and ln 2 to a rounding
    want = torch.tensor([0.0] * 4 + [math.log(2)] + [0.0] * 2, device="cuda")
    assert ((ent - want).abs() <= 2.0 ** -21).all(), ent
    assert ((lp + want).abs() <= 2.0 ** -21).all()
    assert torch.equal(lse, x.gather(1, t.long()[:, None])[:, 0].float())
    assert torch.equal(idx[:, 0], t) and idx[4].tolist() == [3, vocab - 2]


@pytest.mark.parametrize("vocab,offset", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 1), (2 ** 31 - 100, 3)])
def test_vocabularies_up_to_the_largest(vocab, offset):
    """Rows of nearly 2^31 logits, most of them masked: what is left stands at the row's ends, around 2^30 and the
    slices' ends, and all of it counts once."""
    buf = torch.full((vocab + offset + 8,), -math.inf, dtype=torch.bfloat16, device="cuda")
    x = buf[offset:offset + vocab][None]
    buf[:offset] = buf[offset + vocab:] = 100.0   # the neighbours' logits, which are not this row's
    at = sorted({0, 1, 7, 8, 2 ** 29 - 1, 2 ** 30, 2 ** 30 + 2 ** 29, vocab - 9, vocab - 8, vocab - 2, vocab - 1})
    values = [i / 4 for i in range(len(at))]
    x[0, torch.tensor(at, device="cuda")] = torch.tensor(values, device="cuda").bfloat16()
    t = torch.tensor([vocab - 1], dtype=torch.int32, device="cuda")
    lse = torch.empty(1, device="cuda")
    lp, ent, idx, top = abi.token_logprobs(x, t, 16, lse=lse)
    assert abi.check_status() == abi.MLA_OK
    y = torch.tensor(values, dtype=torch.float64)
    assert idx[0].tolist() == at[::-1] + [-1] * (16 - len(at))
    logp = torch.log_softmax(y, 0)
    # eleven terms: a few roundings of 2^-24 and exponentials within 2^-22
    assert abs(float(lse) - float(torch.logsumexp(y, 0))) < 2 ** -18
    assert abs(float(lp) - float(logp[-1])) < 2 ** -18
    assert abs(float(ent) + float((logp.exp() * logp).sum())) < 2 ** -17
    assert (top[0, :len(at)].cpu().double() - logp.flip(0)).abs().max() < 2 ** -18


def test_a_plateau_at_the_end_of_the_largest_row():
    """More equal logits at the row's end than there is room for: its slice is gone over in pieces, past 2^31."""
    vocab, n = 2 ** 31 - 1, 10000
    x = torch.full((1, vocab), -math.inf, dtype=torch.bfloat16, device="cuda")
    x[0, vocab - n:] = 1.0
    x[0, vocab - 1] = 2.0
    t = torch.tensor([vocab - 2], dtype=torch.int32, device="cuda")
    lp, ent, idx, top = abi.token_logprobs(x, t, 8)
    assert abi.check_status() == abi.MLA_OK
    assert idx[0].tolist() == [vocab - 1] + list(range(vocab - n, vocab - n + 7))
    z = math.log(math.e + n - 1)
    assert abs(float(lp) + z) < 1e-4 and abs(float(top[0, 0]) - (1 - z)) < 1e-4
