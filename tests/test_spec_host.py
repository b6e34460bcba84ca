"""Host-only checks of the speculative-decoding ABI: every refusal happens before anything could be enqueued (CPU)."""
import ctypes

import pytest
import torch

from paper_2511_21862_b200 import binding, build, spec

NULL, SHAPE, UNSUP, WS = -1, -2, -3, -4
X = 1 << 20   # a 256-byte aligned address that is never dereferenced


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def shape(**kw):
    d = dict(batch=4, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=16, num_blocks=64, max_blocks_per_seq=8)
    d.update(kw)
    D, bs, h = d["head_dim"], d["block_size"], d["num_kv_heads"]
    st = dict(kv_block_stride=h * bs * D, kv_head_stride=bs * D, kv_token_stride=D)
    st.update({k: d.pop(k) for k in list(d) if k.startswith("kv_")})
    return binding.Shape(**d, **st)


def call(name, *args):
    return getattr(spec._lib(), name)(*args, None)


def slots(sh=None, null=None, **kw):
    sh = sh or shape()
    a = dict(ctx=X, new=X, table=X, held=X, free=X, n_free=8, head=X, held_out=None, head_out=None, row_len=0, rows=32,
             parents=None, slot=X, pos=X, first=X, granted=X, total=X, ws=X, ws_bytes=1 << 20, status=None)
    a.update(kw)
    if null:
        a[null] = None
    return call("ooco_plan_slots", ctypes.byref(sh.c()), *a.values())


def test_plan_slots_refusals():
    for k in ("ctx", "new", "table", "held", "free", "head", "slot", "pos", "first", "granted", "total", "ws"):
        assert slots(null=k) == NULL, k
    assert slots(n_free=-1) == SHAPE and slots(row_len=-1) == SHAPE and slots(rows=-1) == SHAPE
    assert slots(row_len=8, rows=33) == SHAPE                       # B * row_len is 32
    assert slots(shape(batch=0)) == SHAPE and slots(shape(block_size=24)) == UNSUP
    assert slots(shape(num_blocks=1 << 27)) == UNSUP                 # 2^31 slots
    need = spec.plan_slots_workspace_bytes(shape())
    assert need > 0 and slots(ws_bytes=need - 1) == WS and slots(ws=X + 128) == WS
    assert spec._lib().ooco_plan_slots_workspace_bytes(ctypes.byref(shape(head_dim=96).c())) == 0


def rope(fp8=False, sh=None, rope_kw=None, **kw):
    sh = sh or shape()
    r = dict(rot_dim=128, interleaved=0, magnitude=1.0, reserved=0, inv_freq=X)
    r.update(rope_kw or {})
    a = dict(T=3, q=X, qs=1024, k=X, ks=256, v=X, vs=256, pos=X, slot=X, qo=X + 4096, qos=1024, kc=X, vc=X)
    a.update(kw)
    extra = (a.pop("k_scale", 1.0), a.pop("v_scale", 1.0)) if fp8 else ()
    return call("ooco_rope_kv_append" + ("_fp8" if fp8 else ""), ctypes.byref(sh.c()),
                ctypes.byref(spec.ooco_rope_t(*r.values())), *a.values(), *extra)


def test_rope_refusals():
    for k in ("q", "k", "v", "pos", "slot", "qo", "kc", "vc"):
        assert rope(**{k: None}) == NULL, k
    assert rope(rope_kw=dict(inv_freq=None)) == NULL
    assert rope(T=-1) == SHAPE
    for bad in (dict(rot_dim=0), dict(rot_dim=144), dict(interleaved=2), dict(reserved=1), dict(magnitude=float("nan")),
                dict(magnitude=float("inf"))):
        assert rope(rope_kw=bad) == SHAPE, bad
    assert rope(rope_kw=dict(rot_dim=24)) == UNSUP
    for k, v in (("qs", 1016), ("ks", 248), ("vs", 0), ("qos", 8)):  # shorter than a row
        assert rope(**{k: v}) == SHAPE, k
    for k, v in (("qs", 1028), ("ks", 257), ("vs", 260), ("qos", 1025)):  # not 16 bytes
        assert rope(**{k: v}) == UNSUP, k
    for k in ("q", "k", "v", "qo", "kc", "vc"):
        assert rope(**{k: X + 8}) == UNSUP, k
    assert rope(qo=X, qos=2048) == SHAPE                              # in place with another stride
    assert rope(sh=shape(num_blocks=1 << 27)) == UNSUP
    assert rope(T=0, q=None, k=None, v=None, pos=None, slot=None, qo=None) == 0   # nothing to do
    assert rope(fp8=True, k_scale=0.0) == SHAPE and rope(fp8=True, v_scale=float("nan")) == SHAPE
    assert rope(fp8=True, sh=shape(head_dim=64), rope_kw=dict(rot_dim=64)) == UNSUP
    assert rope(fp8=True, sh=shape(kv_token_stride=136)) == UNSUP


def test_frequency_refusals():
    L, inv, mag = spec._lib(), (ctypes.c_float * 64)(), ctypes.c_float()

    def f(rot=64, base=1e4, sc=None, out=inv, m=mag):
        return L.ooco_rope_frequencies(rot, base, ctypes.byref(spec.ooco_rope_scaling_t(*sc)) if sc else None, out,
                                       ctypes.byref(m) if m is not None else None)

    assert f() == 0 and f(out=None) == NULL and f(m=None) == NULL
    assert f(rot=0) == SHAPE and f(rot=7) == SHAPE and f(base=1.0) == SHAPE and f(base=float("nan")) == SHAPE
    assert f(sc=(5, 0, 1.0, 0, 0)) == SHAPE and f(sc=(-1, 0, 1.0, 0, 0)) == SHAPE
    assert f(sc=(1, 0, 0.5, 0, 0)) == SHAPE and f(sc=(1, 0, float("inf"), 0, 0)) == SHAPE
    for kind in (3, 4):
        assert f(sc=(kind, 0, 2.0, 1.0, 4.0)) == SHAPE and f(sc=(kind, 4096, 2.0, 4.0, 4.0)) == SHAPE
        assert f(sc=(kind, 4096, 2.0, 0.0, 4.0)) == SHAPE and f(sc=(kind, 4096, 2.0, 1.0, 4.0)) == 0
    assert f(rot=2, sc=(2, 0, 2.0, 0, 0)) == SHAPE


def tree(fp8=False, sh=None, nodes=8, **kw):
    sh = sh or shape()
    a = dict(q=X, kc=X, vc=X, table=X, ctx=X, parents=X, sizes=None, scale=0.1)
    a.update({k: kw[k] for k in kw if k in a})
    tail = dict(out=X, ws=X, ws_bytes=1 << 40)
    tail.update({k: kw[k] for k in kw if k in tail})
    extra = (kw.get("k_scale", 1.0), kw.get("v_scale", 1.0)) if fp8 else ()
    return call("ooco_tree_attention" + ("_fp8" if fp8 else ""), ctypes.byref(sh.c()), nodes, *a.values(), *extra,
                *tail.values())


def test_tree_refusals():
    for k in ("q", "kc", "vc", "table", "ctx", "parents", "out", "ws"):
        assert tree(**{k: None}) == NULL, k
    assert tree(nodes=0) == SHAPE and tree(nodes=-3) == SHAPE and tree(nodes=257) == UNSUP
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert tree(scale=s) == SHAPE, s
    for k in ("q", "kc", "vc", "out"):
        assert tree(**{k: X + 8}) == UNSUP, k
    need = spec.tree_workspace_bytes(shape(), 8)
    assert need > binding.workspace_bytes_mq(shape(), 8)
    assert tree(ws_bytes=need - 1) == WS and tree(ws=X + 64) == WS
    L = spec._lib()
    for sh, n in ((shape(), 0), (shape(), 257), (shape(head_dim=32), 4)):
        assert L.ooco_tree_workspace_bytes(ctypes.byref(sh.c()), n) == 0
    assert tree(fp8=True, k_scale=-1.0) == SHAPE and tree(fp8=True, sh=shape(head_dim=64)) == UNSUP
    assert tree(sh=shape(num_q_heads=9)) == SHAPE and tree(sh=shape(num_q_heads=34)) == UNSUP


def verify(null=None, **kw):
    c = dict(batch=2, nodes=4, vocab=100, reserved=0, ts=400, tn=100, ds=400, dn=100)
    c.update({k: kw.pop(k) for k in list(kw) if k in c})
    a = dict(p=X, q=X, tokens=X, parents=X, sizes=X, u=X, path=X, out=X, count=X)
    a.update(kw)
    if null:
        a[null] = None
    return call("ooco_verify_drafts", ctypes.byref(spec.ooco_verify_t(*c.values())), *a.values())


def test_verify_refusals():
    for k in ("p", "tokens", "u", "path", "out", "count"):
        assert verify(null=k) == NULL, k
    assert call("ooco_verify_drafts", None, X, X, X, X, X, X, X, X, X) == NULL
    for k in ("batch", "nodes", "vocab"):
        assert verify(**{k: 0}) == SHAPE, k
    assert verify(reserved=1) == SHAPE and verify(ts=-1) == SHAPE and verify(dn=-1) == SHAPE
    assert verify(nodes=257) == UNSUP and verify(vocab=(1 << 20) + 1) == UNSUP and verify(p=X + 2) == UNSUP


def keep(fp8=False, sh=None, nodes=8, **kw):
    a = dict(kc=X, vc=X, table=X, base=X, path=X, count=X, out=X + 4096)
    a.update(kw)
    return call("ooco_kv_keep_path" + ("_fp8" if fp8 else ""), ctypes.byref((sh or shape()).c()), nodes, *a.values())


def test_keep_path_refusals():
    for k in ("kc", "vc", "table", "base", "path", "count"):
        assert keep(**{k: None}) == NULL, k
    assert keep(nodes=0) == SHAPE and keep(nodes=257) == UNSUP and keep(out=X) == SHAPE
    assert keep(kc=X + 8) == UNSUP and keep(vc=X + 4) == UNSUP
    assert keep(fp8=True, sh=shape(head_dim=64)) == UNSUP and keep(fp8=True, sh=shape(kv_head_stride=2056)) == UNSUP


def test_python_side_refuses_cpu_tensors():
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        spec.plan_slots(shape(), z, z, z, z, z, z, z, z, z, z, z, z)
    with pytest.raises(ValueError, match="CUDA"):
        spec.verify_drafts(torch.zeros(1, 2, 3), None, z, None, z, z, z, z)
    with pytest.raises(ValueError, match="CUDA"):
        spec.Rope(16, False, torch.zeros(8))
