"""Shapes and rotary handles may be copied, sent to other processes and collected, before and after their first use (CPU)."""
import copy
import ctypes
import gc
import os
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
    out = subprocess.run([sys.executable, "-c", code], input=pickle.dumps(s), capture_output=True, timeout=300,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert out.returncode == 0, out.stderr.decode()
    assert out.stdout.split() == [str(spec.tree_workspace_bytes(s, 8)).encode(), b"64"]


def test_threads_that_meet_a_shape_at_once_get_one_struct():
    """A struct that another thread has put in meanwhile stays: a call may already hold its address."""
    class Interrupted(binding.Shape):
        def c(self):
            if not hasattr(self, "others"):
                object.__setattr__(self, "others", None)
                object.__setattr__(self, "others", spec._shape(self))   # the other thread's whole turn
            return super().c()

    s = Interrupted(4, 8, 2, 128, 16, 64, 8, 2 * 16 * 128, 16 * 128, 128)
    assert spec._shape(s) is s.others is spec._shape(s)
    assert spec._address(s) == ctypes.addressof(s.others)


class FakeFrequencies:
    """What a Rope asks of its tensor, without a GPU."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, n):
        import torch
        self.n, self.dtype, self.shape = n, torch.float32, (n,)

    def is_contiguous(self):
        return True

    def numel(self):
        return self.n

    def data_ptr(self):
        return id(self)


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r))],
                         ids=["copy", "deepcopy", "pickle"])
def test_copied_rotary_handles(how):
    first = spec.Rope(32, True, FakeFrequencies(16), 1.25)
    second = how(first)
    assert (second.rot_dim, second.interleaved, second.magnitude) == (32, True, 1.25)
    assert (second.inv_freq is first.inv_freq) == (how is copy.copy)
    assert second._address == ctypes.addressof(second._c) != first._address
    del first
    gc.collect()
    c = spec.ooco_rope_t.from_address(second._address)
    assert (c.rot_dim, c.interleaved, c.magnitude, c.reserved) == (32, 1, 1.25, 0)


@pytest.mark.gpu
def test_a_rotary_handle_uses_the_tensor_it_has():
    """Frequencies put elsewhere (a module moved, a tensor's data replaced) and copies of the handle give the same rows."""
    import torch
    T, hq, hkv, D = 5, 8, 2, 128
    sh = binding.Shape(1, hq, hkv, D, 16, 2, 1, hkv * 16 * D, 16 * D, D)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((T, h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    pos, slots = (torch.arange(T, dtype=torch.int32, device="cuda") * s for s in (100, 3))
    kc, vc = (torch.zeros((2, hkv, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    inv = spec.rope_frequencies(D)[0].to("cuda")

    def rotated(rope):
        out = torch.empty_like(q)
        spec.rope_kv_append(sh, rope, q, k, v, pos, slots, out, kc, vc)
        return out

    want = rotated(spec.Rope(D, False, inv))
    held = torch.zeros_like(inv)
    rope = spec.Rope(D, False, held)
    assert not torch.equal(rotated(rope), want)           # no frequencies: nothing turns
    held.data = inv
    for handle in (rope, copy.deepcopy(rope), pickle.loads(pickle.dumps(rope))):
        assert torch.equal(rotated(handle), want)
