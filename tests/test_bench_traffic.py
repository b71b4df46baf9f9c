"""The DRAM figures that the benchmark quotes: every profile it names was captured on the sources of this tree.  (A change to
those sources wants the counters captured anew; what other kernels need does not belong in them.)"""
import pytest

import bench


@pytest.mark.parametrize("kind,workload", sorted(bench.TRAFFIC_PROFILES))
def test_quoted_counters_belong_to_the_sources(kind, workload):
    value, source = bench.ncu_traffic(kind, workload)
    assert value is not None and value > 0, source
