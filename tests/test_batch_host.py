"""Host-only checks of the continuous-batching ABI: every refusal happens before anything could be enqueued (CPU)."""
import ctypes
import math

import pytest
import torch

from paper_2511_21862_b200 import batch, binding, build, spec

NULL, SHAPE, UNSUP, WS = -1, -2, -3, -4
X = 1 << 20      # a 256-byte aligned address that is never dereferenced
STEP = 1 << 20   # buffers that lie apart


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
    return getattr(batch._lib(), name)(*args, None)


def apart(names, first=1):
    return {k: (first + i) * STEP for i, k in enumerate(names)}


FORK = ("parents", "children", "lens", "ctx", "table", "held", "free", "n_free", "head", "shares", "ctx_out", "held_out", "head_out",
        "shares_out", "src", "dst", "granted", "ws", "ws_bytes", "status")


def fork(sh=None, n=3, **kw):
    sh = sh or shape()
    a = dict(apart(FORK), n_free=8, ws_bytes=1 << 20, status=None)
    a.update(kw)
    return call("ooco_fork_pages", ctypes.byref(sh.c()), n, *a.values())


def test_fork_refusals():
    for k in ("parents", "children", "ctx", "table", "held", "free", "head", "shares", "src", "dst", "granted", "ws"):
        assert fork(**{k: None}) == NULL, k
    assert fork(n=-1) == SHAPE and fork(n_free=-1) == SHAPE and fork(shape(batch=0)) == SHAPE
    assert fork(n=batch.MAX_PAGE_ROWS + 1) == UNSUP and fork(shape(batch=batch.MAX_PAGE_ROWS + 1)) == UNSUP
    assert fork(shape(max_blocks_per_seq=1 << 20), n=1 << 11) == UNSUP     # 2^31 entries
    need = batch.pages_workspace_bytes(shape(), 3)
    assert fork(ws_bytes=need - 1) == WS and fork(ws=X + 128) == WS
    b = apart(FORK)
    for k in ("src", "dst", "granted", "table", "ctx_out", "head_out", "shares_out"):   # outputs over inputs and one another
        for other in ("parents", "children", "lens", "free", "ctx", "held", "shares"):
            if k != other + "_out":                                               # (that is in place)
                assert fork(**{k: b[other]}) == SHAPE, (k, other)
    assert fork(src=b["dst"]) == SHAPE and fork(ctx_out=b["held_out"]) == SHAPE and fork(status=b["ws"]) == SHAPE
    assert batch._lib().ooco_pages_workspace_bytes(ctypes.byref(shape().c()), -1) == 0


REL = ("rows", "lens", "ctx", "table", "held", "free", "n_free", "head", "shares", "ctx_out", "held_out", "head_out", "shares_out", "ws",
       "ws_bytes", "status")


def release(sh=None, n=3, **kw):
    sh = sh or shape()
    a = dict(apart(REL), n_free=8, ws_bytes=1 << 20, status=None)
    a.update(kw)
    return call("ooco_release_pages", ctypes.byref(sh.c()), n, *a.values())


def test_release_refusals():
    for k in ("rows", "ctx", "table", "held", "free", "head", "shares", "ws"):
        assert release(**{k: None}) == NULL, k
    assert release(n=-1) == SHAPE and release(n_free=-1) == SHAPE and release(n=batch.MAX_PAGE_ROWS + 1) == UNSUP
    assert release(ws_bytes=256) == WS and release(ws=X + 8) == WS
    b = apart(REL)
    for k in ("free", "ctx_out", "held_out", "head_out", "shares_out"):
        for other in ("rows", "lens", "table", "ctx", "shares"):
            if k != other + "_out":
                assert release(**{k: b[other]}) == SHAPE, (k, other)


def norm(fp8=False, sh=None, rope_kw=None, norm_kw=None, no_norm=False, **kw):
    sh = sh or shape()
    r = dict(rot_dim=128, interleaved=0, magnitude=1.0, reserved=0, inv_freq=X)
    r.update(rope_kw or {})
    h = dict(eps=1e-6, weight_offset=0.0, q_weight=X, k_weight=None)
    h.update(norm_kw or {})
    a = dict(T=3, q=X, qs=1024, k=2 * STEP, ks=256, v=3 * STEP, vs=256, pos=X, slot=X, qo=4 * STEP, qos=1024, kc=X, vc=X)
    a.update(kw)
    extra = (a.pop("k_scale", 1.0), a.pop("v_scale", 1.0)) if fp8 else ()
    return call("ooco_norm_rope_kv_append" + ("_fp8" if fp8 else ""), ctypes.byref(sh.c()),
                ctypes.byref(spec.ooco_rope_t(*r.values())), None if no_norm else ctypes.byref(batch.ooco_head_norm_t(*h.values())),
                *a.values(), *extra)


def test_norm_refusals():
    for k in ("q", "k", "v", "pos", "slot", "qo", "kc", "vc"):
        assert norm(**{k: None}) == NULL, k
    assert norm(no_norm=True) == NULL and norm(rope_kw=dict(inv_freq=None)) == NULL
    for bad in (dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=math.inf), dict(weight_offset=float("nan")),
                dict(weight_offset=math.inf)):
        assert norm(norm_kw=bad) == SHAPE, bad
    assert norm(norm_kw=dict(q_weight=X + 8)) == UNSUP and norm(norm_kw=dict(k_weight=X + 2)) == UNSUP
    assert norm(T=-1) == SHAPE and norm(rope_kw=dict(rot_dim=24)) == UNSUP and norm(qs=1016) == SHAPE
    assert norm(qo=2 * STEP) == SHAPE and norm(qo=X, qos=2048) == SHAPE        # over k; in place with another stride
    assert norm(fp8=True, k_scale=0.0) == SHAPE and norm(fp8=True, sh=shape(head_dim=64), rope_kw=dict(rot_dim=64)) == UNSUP
    assert norm(T=0, q=None, k=None, v=None, pos=None, slot=None, qo=None) == 0


def chunk(fp8=False, sh=None, rows=10, most=5, **kw):
    sh = sh or shape()
    a = dict(q=X, qs=1024, kc=X, vc=X, table=X, ctx=X, first=X, lens=None, scale=0.1)
    a.update({k: kw[k] for k in kw if k in a})
    tail = dict(out=2 * STEP, os=1024, ws=X, ws_bytes=1 << 40)
    tail.update({k: kw[k] for k in kw if k in tail})
    extra = (kw.get("k_scale", 1.0), kw.get("v_scale", 1.0)) if fp8 else ()
    return call("ooco_chunk_attention" + ("_fp8" if fp8 else ""), ctypes.byref(sh.c()), rows, most, *a.values(), *extra,
                *tail.values())


def test_chunk_refusals():
    for k in ("q", "kc", "vc", "table", "ctx", "first", "out", "ws"):
        assert chunk(**{k: None}) == NULL, k
    assert chunk(rows=-1) == SHAPE and chunk(most=-1) == SHAPE and chunk(most=11) == SHAPE and chunk(most=0) == SHAPE
    for s in (0.0, -1.0, float("nan"), math.inf):
        assert chunk(scale=s) == SHAPE, s
    for k in ("q", "kc", "vc", "out"):
        assert chunk(**{k: X + 8}) == UNSUP, k
    assert chunk(qs=1016) == SHAPE and chunk(os=8) == SHAPE and chunk(qs=1028) == UNSUP and chunk(os=1026) == UNSUP
    assert chunk(out=X) == SHAPE and chunk(out=X + 4096) == SHAPE           # over q
    need = batch.chunk_workspace_bytes(shape(), 10, 5)
    assert chunk(ws_bytes=need - 1) == WS and chunk(ws=X + 64) == WS
    assert chunk(rows=1 << 30, most=5) == UNSUP
    L = batch._lib()
    for sh, r, m in ((shape(), 10, 11), (shape(), 10, 0), (shape(), -1, 0), (shape(head_dim=32), 4, 1), (shape(), 1 << 30, 1)):
        assert L.ooco_chunk_workspace_bytes(ctypes.byref(sh.c()), r, m) == 0
    assert chunk(fp8=True, k_scale=-1.0) == SHAPE and chunk(fp8=True, v_scale=math.inf) == SHAPE
    assert chunk(fp8=True, sh=shape(head_dim=64)) == UNSUP and chunk(fp8=True, sh=shape(kv_token_stride=136)) == UNSUP
    assert chunk(sh=shape(num_q_heads=9)) == SHAPE and chunk(sh=shape(num_q_heads=34)) == UNSUP
    assert chunk(rows=0, most=0, q=None, out=None) == 0                      # nothing to do


def test_chunk_workspace_grows_with_what_it_bounds():
    w = lambda rows, most, **kw: batch.chunk_workspace_bytes(shape(**kw), rows, most)  # noqa: E731
    assert w(100, 1) <= w(100, 100) and w(100, 100) < w(4000, 4000) and w(100, 1) < w(100, 1, batch=4000)


LOG = ("logits", "temperature", "repetition", "frequency", "presence", "history", "hlens", "plens", "tokens", "parents", "sizes",
       "btok", "bval", "mask", "out", "probs")


def logits(null=None, **kw):
    c = dict(batch=2, nodes=3, vocab=100, fp32=1, width=20, bias=4, ls=300, ln=100, os=300, on=100, ps=300, pn=100, ms=12, mn=4)
    c.update({k: kw.pop(k) for k in list(kw) if k in c})
    a = apart(LOG)
    a.update(kw)
    for k in null or ():
        a[k] = None
    return call("ooco_shape_logits", ctypes.byref(batch.ooco_logits_t(*c.values())), *a.values())


def test_logits_refusals():
    assert logits(null=["logits"]) == NULL and logits(null=["out", "probs"]) == NULL
    assert call("ooco_shape_logits", None, *apart(LOG).values()) == NULL
    assert logits(null=["history"]) == NULL and logits(null=["hlens"]) == NULL          # the penalties need them
    assert logits(null=["btok"]) == NULL and logits(null=["bval"]) == NULL
    for k in ("batch", "nodes", "vocab"):
        assert logits(**{k: 0}) == SHAPE, k
    assert logits(fp32=2) == SHAPE and logits(width=-1) == SHAPE and logits(bias=-1) == SHAPE
    assert logits(nodes=257) == UNSUP and logits(vocab=batch.MAX_SHAPED_VOCAB + 1) == UNSUP and logits(bias=batch.MAX_BIAS + 1) == UNSUP
    assert logits(batch=(1 << 24) + 1) == UNSUP
    for k in ("ls", "ln", "ms", "mn"):
        assert logits(**{k: -1}) == SHAPE, k
    for k in ("os", "on", "ps", "pn"):                                        # rows of an output that meet
        assert logits(**{k: 99}) == SHAPE, k
    assert logits(out=X + 2) == UNSUP and logits(mask=30 * STEP + 1) == UNSUP and logits(logits=X + 2) == UNSUP
    b = apart(LOG)
    for k in ("out", "probs"):
        for other in LOG[1:14]:
            assert logits(**{k: b[other]}) == SHAPE, (k, other)
    assert logits(out=b["probs"]) == SHAPE
    assert logits(out=b["logits"], os=400) == SHAPE and logits(probs=b["logits"] + 4) == SHAPE   # in place with other rows
    assert logits(out=b["logits"], fp32=0) == SHAPE


def test_python_side_refuses():
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        batch.fork_pages(shape(), z, z, z, z, z, z, z, z, z, z, z, z)
    with pytest.raises(ValueError, match="CUDA"):
        batch.release_pages(shape(), z, z, z, z, z, z, z, z)
    with pytest.raises(ValueError, match="CUDA"):
        batch.shape_logits(torch.zeros(2, 8), probs=torch.zeros(2, 8))
    with pytest.raises(ValueError, match="CUDA"):
        batch.HeadNorm(1e-6, torch.zeros(128, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="CUDA"):
        batch.chunk_attention(shape(), torch.zeros(2, 8, 128, dtype=torch.bfloat16), z, z, z, z, z, 1, 0.1, z, z)
    with pytest.raises(binding.OocoError):
        batch.chunk_workspace_bytes(shape(), 3, 4)
    with pytest.raises(binding.OocoError):
        batch.pages_workspace_bytes(shape(), -1)


def test_constants_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ooco_batch.h")).read()
    for name, value in (("OOCO_MAX_PAGE_ROWS", batch.MAX_PAGE_ROWS), ("OOCO_MAX_SHAPED_VOCAB", batch.MAX_SHAPED_VOCAB),
                        ("OOCO_MAX_BIAS", batch.MAX_BIAS)):
        assert eval(re.search(rf"#define {name} (.+)", text).group(1)) == value, name
