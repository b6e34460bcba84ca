"""Calls whose outputs share memory with what is still to be read are refused before anything is enqueued (CPU).

Every call here is one that must be refused: none may reach a GPU, the addresses are made up."""
import ctypes

import pytest

from paper_2511_21862_b200 import build, spec

from test_spec_host import SHAPE, shape

B, MB, ROWS = 4, 8, 32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def at(i):
    """Address of made-up buffer i: 64 KiB apart."""
    return (1 << 20) + (i << 16)


SLOTS = dict(ctx=at(0), new=at(1), table=at(2), held=at(3), free=at(4), n_free=8, head=at(5), held_out=None, head_out=None,
             row_len=0, rows=ROWS, parents=at(6), slot=at(7), pos=at(8), first=at(9), granted=at(10), total=at(11), ws=at(12),
             ws_bytes=1 << 15, status=at(13))


def slots(**kw):
    a = dict(SLOTS, **kw)
    return spec._lib().ooco_plan_slots(ctypes.byref(shape().c()), *a.values(), None)


@pytest.mark.parametrize("out", ["slot", "pos", "first", "granted", "total", "held_out", "head_out", "table", "ws", "status"])
@pytest.mark.parametrize("into", ["ctx", "new", "held", "free", "head", "parents"])
def test_plan_slots_outputs_over_inputs(out, into):
    if (out, into) in (("held_out", "held"), ("head_out", "head")):
        pytest.skip("in place")
    assert slots(**{out: SLOTS[into]}) == SHAPE


def test_plan_slots_outputs_over_outputs_and_partly():
    assert slots(granted=SLOTS["total"]) == SHAPE and slots(pos=SLOTS["slot"]) == SHAPE and slots(first=SLOTS["granted"]) == SHAPE
    assert slots(total=SLOTS["ctx"] + 4 * (B - 1)) == SHAPE           # the last of the context's lengths
    assert slots(pos=SLOTS["parents"] + 4 * (ROWS - 1)) == SHAPE
    assert slots(slot=SLOTS["table"] + 4 * (B * MB - 1)) == SHAPE
    assert slots(held_out=SLOTS["held"] + 4) == SHAPE                 # in place means in place


@pytest.mark.parametrize("name", ["ooco_kv_keep_path", "ooco_kv_keep_path_fp8"])
def test_keep_path_lengths_over_inputs(name):
    N = 8

    def keep(out):
        return getattr(spec._lib(), name)(ctypes.byref(shape().c()), N, at(0), at(1), at(2), at(3), at(4), at(5), out, None)

    for out in (at(2), at(2) + 4 * (B * MB - 1), at(3), at(3) + 4 * (B - 1), at(3) - 4 * (B - 1), at(4), at(4) + 4 * (B * N - 1),
                at(5), at(5) + 4):
        assert keep(out) == SHAPE, hex(out)


@pytest.mark.parametrize("T", [1, 2, 50])
def test_rotated_queries_over_other_rows(T):
    """q, k, v as parts of one projection's rows (8, 2 and 2 heads of 128 in rows of 1536): q_out may be q or another buffer."""
    stride, X = 1536, at(1)

    def rope(q_out, q_out_stride=stride, q=X, k=X + 2 * 1024, v=X + 2 * 1280, ks=stride):
        r = spec.ooco_rope_t(64, 0, 1.0, 0, at(0))
        return spec._lib().ooco_rope_kv_append(ctypes.byref(shape().c()), ctypes.byref(r), T, q, stride, k, ks, v, stride, at(30),
                                               at(31), q_out, q_out_stride, at(40), at(60), None)

    for out in (X + 2 * 512, X + 2 * 1024, X + 2 * 1280, X + 2 * 1528, X - 2 * 512):
        assert rope(out) == SHAPE, out - X
    assert rope(X + 2 * 128) == SHAPE                                  # one head further
    assert rope(X + 2 * stride * (T - 1) + 2 * 1016, 1024) == SHAPE    # begins in the last row
    assert rope(at(20), 1024, k=at(20) + 2 * (1024 * T - 8), ks=256) == SHAPE
    assert rope(at(20), 1024, v=at(20)) == SHAPE and rope(at(20), 1024, k=at(20), ks=256) == SHAPE
