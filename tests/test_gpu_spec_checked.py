"""Tree attention through the checked build (the library compiled with -DOOCO_CHECKS), on well-formed inputs.

Its kernels range-check every index they derive from device data and every shared-memory destination of an asynchronous
copy; the status word must stay at zero (run_tree asserts it) and the outputs must match the oracle.
"""
import pytest

from paper_2511_21862_b200 import binding, build

import test_gpu_spec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _checked_library():
    build.build()
    previous = binding.use_library(build.build(checked=True))
    assert binding.checked_build()
    yield
    binding.use_library(previous)
    assert not binding.checked_build()


@pytest.mark.parametrize("name", list(test_gpu_spec.TREE_CASES))
def test_tree_cases(name):
    test_gpu_spec.test_tree_attention(name)


@pytest.mark.parametrize("fp8", [None, (0.02, 0.03)], ids=["bf16", "fp8"])
@pytest.mark.parametrize("hq,N", [(16, 9), (40, 8), (32, 16)])
def test_many_short_units(hq, N, fp8):
    test_gpu_spec.test_tree_attention_many_short_units(hq, N, fp8)


def test_random_shapes_and_far_apart_scores():
    test_gpu_spec.test_tree_attention_random_shapes()
    test_gpu_spec.test_tree_attention_scores_far_apart(48, 8, (0.02, 0.03))
    test_gpu_spec.test_tree_attention_scores_far_apart(16, 9, None)
