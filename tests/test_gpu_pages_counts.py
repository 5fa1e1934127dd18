"""mla_pages_*: what the calls make of tables whose entries and counts disagree, and of forks served in part."""
from __future__ import annotations

import pytest
import torch

from paper_2607_27269_gb300 import abi
from tests.test_gpu_pages import Model, i32

pytestmark = pytest.mark.gpu


def uncount(m, page):
    """Nothing counts the page, although a table entry holds it."""
    m.refs[page] = 0
    m.pool.refs[page] = 0


@pytest.mark.parametrize("page", [0, 1, 2])
def test_compaction_records_uncounted_pages(page):
    """An entry that names a page below those in use that nothing counts: another page moves there."""
    m = Model(3, 1, 5, 40, seed=20)
    m.reserve([0, 1], [150, 170])
    m.check()
    uncount(m, page)
    used, moved = m.compact()
    assert used == 5 and moved == 1
    m.bt[0][page] = page  # (the faulty entry is left as it is)
    m.check(abi.MLA_ERR_DEVICE_BOUNDS)


def test_compaction_records_uncounted_pages_above():
    m = Model(3, 1, 5, 40, seed=21)
    m.reserve([0, 1], [150, 170])
    uncount(m, 5)
    assert m.compact() == (5, 0)
    m.check(abi.MLA_ERR_DEVICE_BOUNDS)


def test_sound_compactions_record_nothing():
    """Holes, moves and pages that stay, with a table of several rounds."""
    m = Model(40, 2, 6, 700, (8, 8), 1, seed=22)
    m.reserve(list(range(40)), [(i * 37) % 380 for i in range(40)])
    m.release(list(range(0, 40, 3)), [0] * 14)
    m.compact()
    m.check()


def test_fork_refuses_uncounted_partial_pages():
    m = Model(4, 1, 5, 20, seed=23)
    m.reserve([0], [150])
    uncount(m, 2)                                # the partial last page
    m.pool.fork(i32([0, 0]), i32([1, 2]), i32([150, 128]))
    for kid in (1, 2):
        m.bt[kid][:2] = [0, 1]
        m.refs[0] += 1
        m.refs[1] += 1
    m.check(abi.MLA_ERR_DEVICE_BOUNDS)


@pytest.mark.parametrize("pages", [20, 40000])
def test_fork_refuses_uncounted_full_pages(pages):
    """Whether the same call hands the page out again or not."""
    m = Model(6, 1, 5, pages, (8, 8), seed=24)
    m.reserve([0, 3], [150, 150])
    uncount(m, 1)
    uncount(m, 4)
    m.pool.fork(i32([0, 0, 3]), i32([1, 2, 4]), i32([150, 128, 192 - 1]))
    # two partial pages, copied to the lowest free ones: 1 and 4
    for pair in m.want:
        for c in pair:
            c[1, :22] = c[2, :22]
            c[4, :63] = c[5, :63]
    m.bt[1][:3], m.bt[2][:2], m.bt[4][:3] = [0, -1, 1], [0, -1], [3, -1, 4]
    m.refs[0], m.refs[1], m.refs[3], m.refs[4] = 3, 1, 2, 1
    m.check(abi.MLA_ERR_DEVICE_BOUNDS)


def test_fork_beyond_a_round_of_the_plan():
    """Uncounted pages that the plan has not looked at, since enough free ones lie below."""
    pages, width = 200000, 4
    bt = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    bt[0, :3] = i32([199000, 150000, 7])
    refs[[199000, 7]] = 1
    c = [torch.randn(pages, 64, 8, device="cuda").bfloat16() for _ in range(2)]
    pool = abi.PagePool([abi.Cache(*c, width * 64, bt, 64, pages)], bt, refs)
    pool.fork(i32([0]), i32([1]), i32([130]))
    assert abi.check_status() == abi.MLA_ERR_DEVICE_BOUNDS
    assert bt[1].tolist() == [199000, -1, 0, -1]
    assert refs[[0, 7, 150000, 199000]].tolist() == [1, 1, 0, 2]
    assert all(torch.equal(x[0, :2], x[7, :2]) for x in c)
    refs[150000] = 1
    pool.fork(i32([0]), i32([2]), i32([130]))
    assert abi.check_status() == abi.MLA_OK
    assert bt[2].tolist() == [199000, 150000, 1, -1]
    assert refs[[0, 1, 7, 150000, 199000]].tolist() == [1, 1, 1, 2, 3]


def test_what_a_fork_served_in_part_leaves():
    """A child that holds a page already keeps it and its count; a parent that holds fewer pages than asked for shares
    those that it has, once each."""
    m = Model(5, 1, 4, 20, seed=25)
    m.reserve([0, 1], [150, 64])
    m.pool.fork(i32([0]), i32([1]), i32([150]))   # child 1 holds page 3 in its first entry
    m.bt[1][:3] = [3, 1, 4]
    m.refs[1], m.refs[4] = 2, 1
    for pair in m.want:
        for c in pair:
            c[4, :22] = c[2, :22]
    m.check(abi.MLA_ERR_DEVICE_BOUNDS)
    m.pool.fork(i32([0]), i32([2]), i32([250]))   # the parent holds three entries, the fourth is partial
    m.bt[2][:3] = [0, 1, 2]
    for p in (0, 1, 2):
        m.refs[p] += 1
    m.check(abi.MLA_ERR_DEVICE_BOUNDS)
    m.release([1, 2], [0, 0])
    m.check()
