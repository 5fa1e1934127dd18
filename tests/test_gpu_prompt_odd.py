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


@pytest.mark.parametrize("splits", [0, 1, 5, 40])
@pytest.mark.parametrize("H,G,d", [(14, 2, 64), (8, 2, 128)])
def test_queries_that_are_not_finite_show(H, G, d, splits):
    """NaN and infinities in a query reach its row of o and lse, whole items and cut ones alike, and no other row.  A row
    all of whose scores are -inf has the log-sum-exp -inf of the formula, and weights of 0 / 0."""
    n, kv = [40, 150, 30], [6000, 150, 300]
    L = Layer(H, G, d, kv, True, seed=32)
    for b in range(3):
        for g in range(G):
            at = L.at(b, g, kv[b])
            L.k[at[0], at[1], 2] = L.k[at[0], at[1], 2].abs() + 1  # (one sign: a score's infinity has the query's)
    q = L.normal(220, H, d)

    def run(x):
        step = abi.GqaPrompt(L.dims, L.cache, 3, 220, 6000, splits)
        return step.attend(x, cu_of(n), i32(kv)).clone(), step.lse.clone()

    o, lse = run(q)
    bad = q.clone()
    bad[17, 3, 9] = math.nan
    bad[18] = math.nan
    bad[20, 1, 2] = math.inf        # every score +inf
    bad[25, 5, 5] = math.inf        # scores of both infinities
    bad[60, 0] = math.inf           # infinities of both signs add to NaN
    bad[189, H - 1, 0] = math.nan   # the last token of its sequence
    bad[200, 2, 1] = -math.inf
    only = bad.clone()
    only[30, 4, 2] = -math.inf      # every score -inf
    only[100, 6, 2] = -math.inf
    o2, lse2 = run(only)
    assert abi.check_status() == abi.MLA_OK
    hit = torch.zeros(220, H, dtype=torch.bool, device="cuda")
    for t, h in ((17, 3), (18, slice(None)), (20, 1), (25, 5), (60, 0), (189, H - 1), (200, 2)):
        hit[t, h] = True
    dark = torch.zeros_like(hit)
    dark[30, 4] = dark[100, 6] = True
    assert torch.isnan(lse2[hit]).all() and torch.isneginf(lse2[dark]).all()
    assert torch.isnan(o2[hit | dark].float()).all()
    rest = ~(hit | dark)
    assert torch.equal(o2[rest], o[rest]) and torch.equal(lse2[rest], lse[rest])


def test_rows_without_keys_stay_empty():
    """Queries at negative positions see no key whatever they hold: o = 0, lse = -inf, in whole items and cut ones."""
    n, kv = [90, 700], [30, 4000]
    L = Layer(8, 2, 64, kv, False, seed=33)
    q = L.normal(790, 8, 64)
    q[:60] = math.nan
    for splits in (0, 1, 30):
        step = abi.GqaPrompt(L.dims, L.cache, 2, 790, 4000, splits)
        o = step.attend(q, cu_of(n), i32(kv))
        assert abi.check_status() == abi.MLA_OK
        assert (o[:60] == 0).all() and torch.isneginf(step.lse[:60]).all()
        assert torch.isfinite(o[60:].float()).all() and torch.isfinite(step.lse[60:]).all()
