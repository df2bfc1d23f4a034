"""The DRAM traffic that the bench prints was captured with the kernel sources that are built: a source that changes takes a
new capture with it."""
import glob
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
RECORDS = sorted(os.path.basename(p)[:-len(".traffic.json")] for p in glob.glob(os.path.join(ROOT, "profiles", "*.traffic.json")))


@pytest.mark.parametrize("name", RECORDS)
def test_traffic_belongs_to_the_present_sources(name):
    import bench
    got = bench.measured_traffic(name)
    assert got["traffic"], got["traffic_note"]
    assert got["traffic"] >= got["traffic_algorithmic"]
