"""The verify pass's DRAM traffic that the benchmark reports is of the sources as they are."""
import os

import bench


def test_recorded_traffic_is_of_the_present_sources():
    """The figure is left out where a source of the verify pass's kernels has changed since it was taken
    (profiles/verify_7b_2layers_k4_ctx2048_dram.md says how it is)."""
    got = bench.recorded_traffic()
    assert got is not None, "taken on other sources: " + ", ".join(bench.VERIFY_SOURCES)


def test_operators_for_a_callers_own_layers_are_not_among_them():
    """What op_attention alone needs does not make that figure stale."""
    csrc = os.path.join(bench.ROOT, "paper_2608_10362_gb300", "csrc")
    for name in bench.VERIFY_SOURCES:
        with open(os.path.join(csrc, name)) as fh:
            assert "encode_cache" not in fh.read(), name
