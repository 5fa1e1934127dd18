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
