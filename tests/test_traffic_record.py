"""The indexer's recorded HBM traffic belongs to the committed sources, so that the benchmark's line has it."""
import os

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_record_is_of_these_sources():
    v = bench.measured_traffic(os.path.join(ROOT, "profiles", "index_scores_traffic.json"))
    assert v is not None and v > 4.5e9      # at least the score matrix that it writes


def test_the_record_outlives_the_rules_of_other_kernels():
    for f in bench.TRAFFIC_SOURCES:
        assert "prefix_plan" not in open(os.path.join(ROOT, f)).read()
