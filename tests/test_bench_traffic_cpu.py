"""The HBM bytes that the bench reports come from committed counters of the kernels as they are."""
import pytest

import bench


@pytest.mark.parametrize("key", sorted(bench.TRAFFIC))
def test_traffic_is_of_these_sources(key):
    assert bench.measured_traffic(*bench.TRAFFIC[key]), f"{bench.TRAFFIC[key][0]} was taken on other kernel sources"
