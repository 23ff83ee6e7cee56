"""DRAM traffic that bench.py reports: taken while the kernel's source was what it is now, from a profile that is there and says so."""
import os

import pytest

import bench


@pytest.mark.parametrize("workload", sorted(bench.NCU_TRAFFIC))
def test_captures_are_of_the_present_sources(workload):
    traffic, source = bench.ncu_traffic(workload)
    assert traffic == bench.NCU_TRAFFIC[workload]["bytes"], source
    with open(os.path.join(bench.ROOT, bench.NCU_TRAFFIC[workload]["profile"])) as f:
        assert f"{traffic / 1e6:.1f} MB" in f.read()
