"""The bounded wait that counts its looks: it runs out, says so, and takes the time that its count was chosen for."""
from __future__ import annotations

import os
import re

import pytest
import torch

from paper_2607_27269_gb300 import abi

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_27269_gb300", "csrc",
                      "prompt_attn.cu")


@pytest.mark.gpu
def test_counted_wait_runs_out_in_time():
    assert abi.check_status() == abi.MLA_OK
    ns = torch.zeros(1, dtype=torch.int64, device="cuda")
    abi.selftest_wait_looks(ns)
    assert abi.check_status() == abi.MLA_ERR_DEVICE_TIMEOUT
    assert abi.check_status() == abi.MLA_OK
    looks = int(re.search(r"constexpr int kLooks = (\d+);", open(SOURCE).read()).group(1))
    # the kernel's wait: about a second, no less than a third of one (a busy GPU's longest launch), no more than three
    assert 1e9 / 3 < int(ns) / 1000 * looks < 3e9
    abi.selftest_wait_looks()
    assert abi.check_status() == abi.MLA_ERR_DEVICE_TIMEOUT


def test_counted_wait_refusals():
    assert abi.lib().mla_selftest_wait_looks(0x10004, None) == abi.MLA_ERR_INVALID_ARG
