"""Handles follow the caches that they were made for: a tensor put in the place of another is the one that counts."""
from __future__ import annotations

import pytest
import torch

from paper_2607_27269_gb300 import abi
from tests.test_gpu_prompt import Layer, cu_of, i32

pytestmark = pytest.mark.gpu


def test_a_prompt_handle_reads_the_caches_tensors_of_now():
    n = [70, 33]
    L = Layer(8, 2, 64, n, True, seed=40)
    q, k, v = L.normal(103, 8, 64), L.normal(103, 2, 64), L.normal(103, 2, 64)
    step = abi.GqaPrompt(L.dims, L.cache, 2, 103, 70)
    old = L.k, L.v, L.bt
    want = step(q, k, v, cu_of(n), i32([0, 0]), i32(n)).clone()
    untouched = [t.clone() for t in old]
    # the pages in the opposite order, in new tensors
    L.cache.c_kv, L.cache.k_rope = (torch.zeros_like(t) for t in (L.v, L.k))
    L.cache.block_table = torch.where(L.bt >= 0, L.n_pages - 1 - L.bt, L.bt)
    got = step(q, k, v, cu_of(n), i32([0, 0]), i32(n))
    assert abi.check_status() == abi.MLA_OK
    assert torch.equal(got, want)
    assert all(torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else a.dtype),
                           b.view(torch.int16 if b.dtype == torch.bfloat16 else b.dtype)) for a, b in zip(old, untouched))
    assert float(L.cache.k_rope.float().abs().max()) > 0


def test_a_pool_reads_the_caches_tensors_of_now():
    bt = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(8, dtype=torch.int32, device="cuda")
    new = lambda x: [torch.full((8, 64, 8), x, dtype=torch.bfloat16, device="cuda") for _ in range(2)]  # noqa: E731
    cache = abi.Cache(*new(1.0), 128, bt, 64, 8)
    pool = abi.PagePool([cache], bt, refs)
    pool.reserve(i32([0]), i32([70]))
    old = cache.c_kv, cache.k_rope
    cache.c_kv, cache.k_rope = new(2.0)
    for t in (cache.c_kv, cache.k_rope):
        t[1, :6] = 5.0
    pool.fork(i32([0]), i32([1]), i32([70]))
    assert abi.check_status() == abi.MLA_OK
    assert all(float(t.min()) == 1.0 == float(t.max()) for t in old)
    assert all((t[2, :6] == 5).all() and (t[2, 6:] == 2).all() for t in (cache.c_kv, cache.k_rope))
    # and the table and the counts of now
    pool.block_table, pool.refs = bt.clone(), refs.clone()
    pool.release(i32([1]), i32([0]))
    assert abi.check_status() == abi.MLA_OK
    assert bt[1].tolist() == [0, 2] and pool.block_table[1].tolist() == [-1, -1]
    assert refs[:3].tolist() == [2, 1, 1] and pool.refs[:3].tolist() == [1, 1, 0]
