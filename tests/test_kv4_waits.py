"""Waits of the attention kernels whose lanes work together behind them: when one of them runs out while others' phases have ended, all lanes of
the warp have to take the same way, or those that go on wait for the others without a limit.  Such a time cannot be arranged on a GPU; the
sources are looked at (CPU)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2309_15531_b200", "csrc")


@pytest.mark.parametrize("name", ["kv4_few.cu", "kv4_many.cu"])
def test_waits_have_one_answer_for_a_warp(name):
    with open(os.path.join(CSRC, name)) as f:
        source = f.read()
    assert re.search(r"mbar_wait_warp\(", source) and not re.search(r"mbar_wait\(", source)
