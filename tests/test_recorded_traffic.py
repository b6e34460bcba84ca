"""The DRAM traffic that the benchmark reports beside its roofline comes from captures of the present sources (CPU)."""
import importlib.util
import os

import pytest

from paper_2511_21862_b200 import inputs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def bench():
    spec = importlib.util.spec_from_file_location("bench_for_traffic", os.path.join(ROOT, "bench.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("workload", sorted(inputs.CONFIGS))
def test_traffic_is_of_the_present_kernel(bench, workload):
    algorithmic = 10 ** 9
    moved, how = bench.ncu_traffic(workload, algorithmic)
    assert moved is not None, how
    if how.startswith("scaled"):
        assert 0.98 * algorithmic <= moved <= 1.05 * algorithmic   # a stream read once, partial rows beside it
