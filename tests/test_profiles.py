"""The counter summaries that bench.py reads are those of the present kernels (else what it says of their traffic is null)."""
import pytest

import bench


@pytest.mark.parametrize("summary,sources", [("fused_search_large_sweep.txt", bench.FUSED_SOURCES), ("cp_local_critical_path_stress.txt", bench.CP_SOURCES)])
def test_summaries_name_the_present_sources(summary, sources):
    assert bench.profiled_traffic(summary, sources) > 0
