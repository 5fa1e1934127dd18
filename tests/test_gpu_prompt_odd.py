"""Packed prompts whose offsets or queries are out of the ordinary: tokens that belong to no sequence, offsets that
fall, queries that are not finite (mla_gqa_prompt_append, mla_gqa_prompt_attn)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2607_27269_gb300 import abi
from tests.helpers import rope_complex
from tests.test_gpu_prompt import R8, Layer, cu_of, i32

pytestmark = pytest.mark.gpu


def turned(x, pos, got):
    """got = R_pos x within the bar of tests/test_gpu_prompt.py: one bf16 rounding and 6e-7 of the pair's magnitudes."""
    x = x.double().cpu().numpy()
    want, half = rope_complex(x, np.asarray(pos)[:, None]), x.shape[-1] // 2
    pair = np.abs(x[..., :half]) + np.abs(x[..., half:])
    bar = R8 * np.abs(want) + (1 + R8) * 6e-7 * np.concatenate([pair, pair], -1)
    return bool((np.abs(got.double().cpu().numpy() - want) <= bar).all())


def check_owners(cu, total, status, owned, G=2):
    """owned: (sequence, its first token's position, first token, end) of what has to be written, and nothing else."""
    H, d = 4 * G, 64
    L = Layer(H, G, d, [200] * (len(cu) - 1), True, seed=30)
    q, k, v = L.normal(total, H, d), L.normal(total, G, d), L.normal(total, G, d)
    rot = torch.full_like(q, 7.0)
    want = {"k": L.k.clone(), "v": L.v.clone(), "rot": rot.clone()}
    start = [3 * b % 150 for b in range(len(cu) - 1)]
    abi.gqa_prompt_append(L.dims, L.cache, q, k, v, i32(cu), i32(start), rot)
    assert abi.check_status() == status
    for b, skip, first, end in owned:
        pos = start[b] + skip + np.arange(end - first)
        assert turned(q[first:end], pos, rot[first:end])
        want["rot"][first:end] = rot[first:end]
        for g in range(G):
            at = L.at(b, g, end - first, start[b] + skip)
            assert turned(k[first:end, g:g + 1], pos, L.k[at][:, None])
            want["k"][at], want["v"][at] = L.k[at], v[first:end, g]
    for name, have in (("k", L.k), ("v", L.v), ("rot", rot)):
        assert torch.equal(have.view(torch.int16), want[name].view(torch.int16)), name


@pytest.mark.parametrize("cu,total,owned", [
    ([5, 12, 20], 25, [(0, 0, 5, 12), (1, 0, 12, 20)]),
    ([9, 9, 10], 10, [(1, 0, 9, 10)]),
    ([40, 40], 40, []),
])
def test_append_tokens_of_no_sequence(cu, total, owned):
    """Tokens before the first sequence and behind the last one are left alone, and are no fault."""
    check_owners(cu, total, abi.MLA_OK, owned)


@pytest.mark.parametrize("cu,total,owned", [
    ([3, 0, 10], 12, [(1, 0, 0, 10)]),           # no token tells: they all are the second sequence's
    ([-2, 0, 10], 10, [(1, 0, 0, 10)]),
    ([0, 13], 12, []),
])
def test_append_records_faulty_offsets(cu, total, owned):
    check_owners(cu, total, abi.MLA_ERR_DEVICE_BOUNDS, owned)


@pytest.mark.parametrize("cu,total,owned", [
    ([0, 50, 40, 110], 110, [(0, 0, 0, 50), (2, 10, 50, 110)]),
    ([0, 20, 10, 15, 30], 30, [(0, 0, 0, 20), (3, 5, 20, 30)]),
    ([0, 10, 10, 7], 10, [(0, 0, 0, 10)]),
    ([30, 20, 30, 5, 5], 40, [(1, 0, 20, 30)]),
    ([0, 10, 90, 15, 30], 30, [(0, 0, 0, 10), (3, 0, 15, 30)]),
])
def test_append_serves_sound_sequences_beside_faulty_ones(cu, total, owned):
    """A sequence whose own offsets are sound has all its tokens written, wherever others' fall; of two that claim a
    token the first has it."""
    check_owners(cu, total, abi.MLA_ERR_DEVICE_BOUNDS, owned)


def test_append_finds_sequences_far_down():
    """More sequences than a warp has lanes, empty ones among them, faulty ones too."""
    n = [(i * 5) % 4 for i in range(100)]
    cu = [0] + np.cumsum(n).tolist()
    check_owners(cu, cu[-1], abi.MLA_OK, [(b, 0, cu[b], cu[b + 1]) for b in range(100)], G=1)
    cu[70] = 1 << 30  # the 69th ends and the 70th begins past the tokens
    check_owners(cu, cu[-1], abi.MLA_ERR_DEVICE_BOUNDS, [(b, 0, cu[b], cu[b + 1]) for b in range(100) if b not in (69, 70)], G=1)
