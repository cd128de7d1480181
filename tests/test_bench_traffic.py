"""The DRAM traffic that bench.py reports was counted on the kernels' sources as they are: a change to them, or to the headers
that their device code takes, has the counters taken again."""
import pytest

import bench


@pytest.mark.parametrize("source", sorted(bench.NCU_TRAFFIC_SOURCES))
def test_traffic_figures_belong_to_the_sources(source):
    assert bench.source_digest(source) == bench.NCU_TRAFFIC_SOURCES[source]
