"""Shapes and rotary handles may be copied, sent to other processes and collected, before and after their first use (CPU)."""
import copy
import ctypes
import gc
import pickle
import subprocess
import sys

import pytest

from paper_2511_21862_b200 import binding, build, spec


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def shape():
    return binding.Shape(4, 8, 2, 128, 16, 64, 8, 2 * 16 * 128, 16 * 128, 128)


def used():
    """A Shape that `spec` has met."""
    s = shape()
    spec.plan_slots_workspace_bytes(s)
    spec._address(s)
    return s


def contents(address):
    c = binding.ooco_shape_t.from_address(address)
    return [getattr(c, name) for name, _ in c._fields_]


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda s: pickle.loads(pickle.dumps(s))],
                         ids=["copy", "deepcopy", "pickle"])
def test_copied_shapes_have_structs_of_their_own(how):
    first = used()
    second = how(first)
    assert second == first
    assert spec._address(second) == ctypes.addressof(spec._shape(second))
    want = contents(spec._address(first))
    if how is not copy.copy:
        assert spec._address(second) != spec._address(first)
    del first
    gc.collect()
    assert contents(spec._address(second)) == want == contents(ctypes.addressof(shape().c()))


def test_a_used_shape_in_another_process():
    code = ("import ctypes, pickle, sys\n"
            "from paper_2511_21862_b200 import spec\n"
            "s = pickle.loads(sys.stdin.buffer.read())\n"
            "assert spec._address(s) == ctypes.addressof(spec._shape(s))\n"
            "print(spec.tree_workspace_bytes(s, 8), spec._shape(s).num_blocks)\n")
    s = used()
    out = subprocess.run([sys.executable, "-c", code], input=pickle.dumps(s), capture_output=True, timeout=300)
    assert out.returncode == 0, out.stderr.decode()
    assert out.stdout.split() == [str(spec.tree_workspace_bytes(s, 8)).encode(), b"64"]
