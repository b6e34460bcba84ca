"""The continuous-batching operators on the GPU against their 64-bit definitions, through the C ABI."""
import math

import numpy as np
import pytest
import torch

from oracle import batch_oracle as bo
from paper_2511_21862_b200 import batch, binding, build, spec

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def gpu(a, dtype=I32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).to(DEV)


def pool_shape(B, hq, hkv, D, bs, NB, MB, layout="head_major"):
    st = (hkv * bs * D, bs * D, D) if layout == "head_major" else (bs * hkv * D, D, hkv * D)
    return binding.Shape(B, hq, hkv, D, bs, NB, MB, *st)


def host(t):
    return t.detach().cpu().double().numpy()


# ------------------------------------------------------------------------------------------------ pages
def random_pool(rng, B, bs, ctx_hi, spare, extra_rows=0, MB=None):
    """(ctx, held, table, free ids, pool size); the last extra_rows rows hold nothing."""
    ctx = rng.integers(0, ctx_hi + 1, B)
    ctx[B - extra_rows:] = 0
    held = -(-ctx // bs)
    MB = MB or max(1, int(held.max())) + 1
    NB = int(held.sum()) + spare
    perm = rng.permutation(NB)
    table, at = np.full((B, MB), -1), 0
    for b in range(B):
        table[b, : held[b]] = perm[at: at + held[b]]
        at += held[b]
    return ctx, held, table, perm[at:], NB


def run_fork(parents, children, lens, ctx, table, held, free, head, shares, *, bs, NB, in_place=False):
    B, MB = table.shape
    F = len(parents)
    sh = pool_shape(B, 1, 1, 64, bs, NB, MB)
    want = bo.fork_pages(np.asarray(parents), np.asarray(children), lens, ctx, table, held, free, head, shares, block_size=bs,
                         num_blocks=NB)
    t = dict(table=gpu(table), ctx=gpu(ctx), held=gpu(held), head=gpu([head]), shares=gpu(shares))
    o = {} if in_place else dict(context_lens_out=gpu(np.full(B, -9)), blocks_held_out=gpu(np.full(B, -9)),
                                 free_head_out=gpu([-9]), shares_out=gpu(np.full(NB, -9)))
    src, dst, granted = (torch.full((F,), -77, dtype=I32, device=DEV) for _ in range(3))
    status = gpu([0])
    ws = torch.full((batch.pages_workspace_bytes(sh, F),), 255, dtype=torch.uint8, device=DEV)
    batch.fork_pages(sh, gpu(parents), gpu(children), t["ctx"], t["table"], t["held"], gpu(free), t["head"], t["shares"], src, dst,
                     granted, ws, shared_lens=None if lens is None else gpu(lens), status=status, **o)
    got = dict(table=t["table"], copy_src=src, copy_dst=dst, granted=granted, status=status, ctx=o.get("context_lens_out", t["ctx"]),
               held=o.get("blocks_held_out", t["held"]), head=o.get("free_head_out", t["head"]),
               shares=o.get("shares_out", t["shares"]))
    for k, v in got.items():
        assert np.array_equal(v.cpu().numpy().reshape(-1), np.asarray(want[k]).reshape(-1)), k
    if not in_place:
        assert np.array_equal(t["ctx"].cpu().numpy(), ctx) and np.array_equal(t["shares"].cpu().numpy(), shares)
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed,B,F,bs,hi,cut,short", [(0, 9, 5, 16, 100, False, 0), (1, 40, 33, 16, 700, True, 0),
                                                      (2, 40, 30, 32, 700, True, 9), (3, 7, 1, 256, 5000, False, 0),
                                                      (4, 700, 600, 16, 3000, True, 0), (5, 60, 20, 16, 60000, True, 2)])
def test_fork(seed, B, F, bs, hi, cut, short, in_place):
    rng = np.random.default_rng(seed)
    ctx, held, table, free, NB = random_pool(rng, B, bs, hi, F + 5 - short, extra_rows=F)
    children = B - F + rng.permutation(F)
    parents = rng.integers(0, B - F, F)
    lens = rng.integers(-3, hi + 50, F) if cut else None
    want = run_fork(parents, children, lens, ctx, table, held, free, 2, rng.integers(0, 3, NB), bs=bs, NB=NB, in_place=in_place)
    assert want["granted"].any()


def test_fork_refusals_and_edges():
    rng = np.random.default_rng(7)
    ctx, held, table, free, NB = random_pool(rng, 12, 16, 200, 20, extra_rows=6)
    ctx[:6] = [100, 96, 0, 1, 15, 200]
    held[:6] = [7, 6, 0, 1, 1, 13]
    table = np.full((12, 14), -1)
    at = 0
    for b in range(6):
        table[b, : held[b]] = np.arange(at, at + held[b])
        at += held[b]
    NB, free = at + 10, np.arange(at, at + 10)
    shares = np.zeros(NB, np.int64)
    kw = dict(bs=16, NB=NB)
    # named twice, a parent as child, itself, out of range on both sides, a row that holds pages, empty parent, whole pages
    run_fork([0, 0, 1, 2, 0, 99, -1, 0, 2, 1], [6, 6, 0, 2, 12, 7, 8, 3, 9, 10], None, ctx, table, held, free, 0, shares, **kw)
    run_fork([], [], None, ctx, table, held, free, 3, shares, **kw)
    # a parent that holds fewer pages than its length needs; a list that runs out in the middle and serves who needs none
    few = held.copy()
    few[5] = 12
    run_fork([5, 0, 1], [6, 7, 8], None, ctx, table, few, free, 0, shares, **kw)
    want = run_fork([0, 3, 4, 1, 2, 0], [6, 7, 8, 9, 10, 11], [100, 1, 15, 96, 0, 48], ctx, table, held, free, 8, shares, **kw)
    assert list(want["granted"]) == [1, 1, 0, 1, 1, 1] and want["head"] == 10
    run_fork([0, 1], [6, 7], None, ctx, table, held, free, -4, shares, **kw)
    run_fork([0, 1], [6, 7], None, ctx, table, held, free, 99, shares, **kw)
    run_fork([0, 1], [6, 7], None, ctx, table, held, free[:0], 0, shares, **kw)
    # ids outside the pool, in the parent's row and in the list
    bad = table.copy()
    bad[0, 2], bad[0, 6], bad[4, 0] = NB, -5, 1 << 30
    run_fork([0, 4, 1], [6, 7, 8], None, ctx, bad, held, free, 0, shares, **kw)
    run_fork([0, 4], [6, 7], None, ctx, table, held, np.array([-1, NB]), 0, shares, **kw)


def run_release(rows, keep, ctx, table, held, free, head, shares, *, bs, NB, in_place=False):
    B, MB = table.shape
    sh = pool_shape(B, 1, 1, 64, bs, NB, MB)
    want = bo.release_pages(np.asarray(rows), keep, ctx, table, held, free, head, shares, block_size=bs, num_blocks=NB)
    t = dict(free=gpu(free), ctx=gpu(ctx), held=gpu(held), head=gpu([head]), shares=gpu(shares))
    o = {} if in_place else dict(context_lens_out=gpu(np.full(B, -9)), blocks_held_out=gpu(np.full(B, -9)),
                                 free_head_out=gpu([-9]), shares_out=gpu(np.full(NB, -9)))
    status = gpu([0])
    ws = torch.full((batch.pages_workspace_bytes(sh, len(rows)),), 255, dtype=torch.uint8, device=DEV)
    batch.release_pages(sh, gpu(rows), t["ctx"], gpu(table), t["held"], t["free"], t["head"], t["shares"], ws,
                        keep_lens=None if keep is None else gpu(keep), status=status, **o)
    got = dict(free=t["free"], status=status, ctx=o.get("context_lens_out", t["ctx"]), held=o.get("blocks_held_out", t["held"]),
               head=o.get("free_head_out", t["head"]), shares=o.get("shares_out", t["shares"]))
    for k, v in got.items():
        assert np.array_equal(v.cpu().numpy().reshape(-1), np.asarray(want[k]).reshape(-1)), k
    return want


def shared_state(rng, B, bs, hi, spare):
    """A pool whose rows share prefixes: (ctx, held, table, free list as a stack, head, shares, NB)."""
    ctx, held, table, _, NB = random_pool(rng, B, bs, hi, spare)
    for b in range(1, B, 2):
        k = int(rng.integers(0, B // 2 + 1)) // 2 * 2 % B
        n = min(int(held[b]), int(held[k]), int(rng.integers(0, 6)))
        table[b, :n] = table[k, :n]
    uses = np.zeros(NB, np.int64)
    for b in range(B):
        np.add.at(uses, table[b, : held[b]], 1)
    dead = np.flatnonzero(uses == 0)
    free = np.full(NB, -1)
    free[NB - len(dead):] = dead
    return ctx, held, table, free, NB - len(dead), np.maximum(uses - 1, 0), NB


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed,B,R,bs,hi,cut", [(0, 8, 3, 16, 100, False), (1, 60, 60, 16, 400, True), (2, 33, 20, 32, 3000, False),
                                                (3, 5, 1, 16, 70000, True), (4, 500, 480, 16, 3000, True), (5, 3, 0, 16, 50, False)])
def test_release(seed, B, R, bs, hi, cut, in_place):
    rng = np.random.default_rng(seed)
    ctx, held, table, free, head, shares, NB = shared_state(rng, B, bs, hi, 7)
    rows = rng.permutation(B)[:R]
    keep = np.where(rng.random(R) < 0.5, 0, rng.integers(-5, hi + 5, R)) if cut else None
    run_release(rows, keep, ctx, table, held, free, head, shares, bs=bs, NB=NB, in_place=in_place)


def test_release_refusals_and_edges():
    rng = np.random.default_rng(11)
    ctx, held, table, free, head, shares, NB = shared_state(rng, 10, 16, 300, 4)
    kw = dict(bs=16, NB=NB)
    run_release([1, 1, 2, 10, -1, 3], None, ctx, table, held, free, head, shares, **kw)        # twice, out of range
    run_release([1, 2, 3], None, ctx, table, held, free, 2, shares, **kw)                       # no room for all
    run_release([1, 2, 3], None, ctx, table, held, free, -3, shares, **kw)
    run_release([1, 2], None, ctx, table, held, free, NB + 50, shares, **kw)
    run_release([0, 1, 2, 3], None, ctx, table, held, free, head, np.zeros_like(shares), **kw)  # given back more often than held
    bad = table.copy()
    bad[0, 0], bad[1, 0] = NB, -7
    run_release([0, 1], None, ctx, bad, held, free, head, shares, **kw)
    many = held.copy()
    many[0], many[1] = 1 << 20, -3                                                              # clamped to the row
    run_release([0, 1], None, ctx, np.where(table < 0, NB - 1, table), many, free, head, shares, **kw)


def test_fork_and_release_return_to_the_start():
    """Children fork, their tails are copied, all of them end: the counts and the set of free pages are as before; in between
    every child reads what its parent holds."""
    rng = np.random.default_rng(3)
    B, F, bs, hkv, D = 20, 10, 16, 2, 64
    ctx, held, table, free, NB = random_pool(rng, B, bs, 200, 2 * F, extra_rows=F)
    sh = pool_shape(B, hkv, hkv, D, bs, NB, table.shape[1])
    kc, vc = (torch.randn((NB, hkv, bs, D), device=DEV).to(torch.bfloat16) for _ in range(2))
    t = dict(ctx=gpu(ctx), table=gpu(table), held=gpu(held), head=gpu([0]), shares=gpu(np.zeros(NB)), free=gpu(free))
    parents, children = gpu(rng.integers(0, B - F, F)), gpu(np.arange(B - F, B))
    src, dst, granted = (torch.empty(F, dtype=I32, device=DEV) for _ in range(3))
    ws = torch.empty(batch.pages_workspace_bytes(sh, F), dtype=torch.uint8, device=DEV)
    batch.fork_pages(sh, parents, children, t["ctx"], t["table"], t["held"], t["free"], t["head"], t["shares"], src, dst, granted, ws)
    binding.kv_copy_blocks(sh, kc, vc, src, dst)
    assert granted.all()
    for p, c in zip(parents.tolist(), children.tolist()):
        n = int(t["ctx"][c])
        assert n == int(t["ctx"][p])
        rows = [kc[t["table"][b, : -(-n // bs)].long()].transpose(1, 2).flatten(0, 1)[:n] for b in (p, c)]
        assert torch.equal(*rows)
    batch.release_pages(sh, children, t["ctx"], t["table"], t["held"], t["free"], t["head"], t["shares"], ws)
    assert int(t["head"]) == 0 and not t["shares"].any() and sorted(t["free"].tolist()) == sorted(free.tolist())
    assert np.array_equal(t["held"].cpu().numpy()[: B - F], held[: B - F]) and not t["held"][B - F:].any()


# ------------------------------------------------------------------------------------------------ norms, rotation, append
@pytest.mark.parametrize("T,hq,hkv,D,rot,inter,fp8,weights,offset,layout", [
    (1, 8, 2, 128, 128, False, False, True, 0.0, "head_major"), (7, 5, 5, 64, 48, False, False, True, 1.0, "token_major"),
    (33, 16, 1, 128, 32, True, False, False, 0.5, "head_major"), (9, 40, 8, 128, 128, False, True, True, 0.0, "token_major"),
    (21, 8, 8, 128, 16, True, True, True, -0.5, "head_major"), (700, 4, 2, 64, 64, True, False, True, 0.0, "head_major"),
    (3, 3, 1, 128, 112, False, True, False, 0.0, "head_major")])
def test_norm_rope_append(T, hq, hkv, D, rot, inter, fp8, weights, offset, layout):
    rng = np.random.default_rng(T + D + rot)
    bs, NB = 16, T // 16 + 3
    sh = pool_shape(1, hq, hkv, D, bs, NB, 1, layout)
    x = rng.standard_normal((T, hq + 2 * hkv, D)) * np.exp(2 * rng.standard_normal((1, hq + 2 * hkv, 1)))
    x[0, 0], x[0, -1] = 0.0, 0.0                        # a head of zeros: eps alone
    qkv = torch.as_tensor(x).to(torch.bfloat16).to(DEV)
    q, k, v = qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
    w = [torch.as_tensor(rng.standard_normal(D)).to(torch.bfloat16).to(DEV) if weights else None for _ in range(2)]
    inv, _ = spec.rope_frequencies(rot, 1e4)
    pos = rng.integers(0, 1 << 20, T)
    slots = rng.permutation(NB * bs)[:T]
    if T > 4:
        pos[2], slots[3], slots[4] = -1, -1, NB * bs    # padding; rows without a slot
    cell, cells = (torch.uint8, (NB, hkv, bs, D)) if fp8 else (torch.bfloat16, (NB, hkv, bs, D))
    if layout == "token_major":
        cells = (NB, bs, hkv, D)
    kc, vc = (torch.full(cells, 7, dtype=cell, device=DEV) for _ in range(2))
    out = torch.full((T, hq, D), 3.0, dtype=torch.bfloat16, device=DEV)
    rope, norm = spec.Rope(rot, inter, inv.to(DEV), 1.25), batch.HeadNorm(1e-5, w[0], w[1], offset)
    args = (sh, rope, norm, q, k, v, gpu(pos), gpu(slots), out, kc, vc)
    ks, vs = 0.05, 0.3
    if fp8:
        batch.norm_rope_kv_append_fp8(*args, ks, vs)
    else:
        batch.norm_rope_kv_append(*args)
    hw = [None if z is None else host(z) for z in w]
    qn, kn = bo.head_norm(host(q), hw[0], 1e-5, offset), bo.head_norm(host(k), hw[1], 1e-5, offset)
    qr, kr = (bo.turn(z, pos, inv.double().numpy(), inter, 1.25) for z in (qn, kn))
    # fp32 up to the last rounding: a sum of 128 squares in a tree of 20 levels, a reciprocal root, three products, cosine and
    # sine to 2^-22, two products and a sum: below 2^-18 of the head's largest value, which bounds both members of a pair
    near = lambda z: 2.0 ** -18 * np.abs(z).max(-1, keepdims=True) * 1.25 * 2 + 1e-30  # noqa: E731
    live = pos >= 0
    err = np.abs(host(out) - qr)
    assert (err <= 2.0 ** -8 * np.abs(qr) + near(qn))[live].all()
    assert (host(out)[~live] == 3.0).all()
    kc, vc = ((z if layout == "head_major" else z.transpose(1, 2)) for z in (kc, vc))
    touched = np.zeros((NB, bs), bool)
    for t in range(T):
        if not live[t] or not 0 <= slots[t] < NB * bs:
            continue
        blk, off = divmod(int(slots[t]), bs)
        touched[blk, off] = True
        a, b = kc[blk, :, off], vc[blk, :, off]
        if fp8:
            a, b = host(a.view(torch.float8_e4m3fn)), host(b.view(torch.float8_e4m3fn))
            ka, va = np.clip(kr[t] / ks, -448, 448), np.clip(host(v)[t] / np.float32(vs), -448, 448)
            for got, want, slack in ((a, ka, near(kn[t]) / ks), (b, va, 2.0 ** -23 * np.abs(va))):
                assert (np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) + 1.0625 * slack).all()
        else:
            assert (np.abs(host(a) - kr[t]) <= 2.0 ** -8 * np.abs(kr[t]) + near(kn[t])).all()
            assert torch.equal(b, v[t])
    for z in (kc, vc):
        assert (z.transpose(1, 2).cpu()[torch.as_tensor(~touched)] == 7).all()


def test_norm_rope_in_place_and_empty():
    sh = pool_shape(1, 4, 2, 64, 16, 2, 1)
    x = torch.randn((5, 8, 64), device=DEV).to(torch.bfloat16)
    inv, _ = spec.rope_frequencies(64)
    rope, norm = spec.Rope(64, False, inv.to(DEV)), batch.HeadNorm(1e-6)
    kc, vc = (torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pos, slots = gpu(np.arange(5)), gpu(np.arange(5))
    out = torch.empty((5, 4, 64), dtype=torch.bfloat16, device=DEV)
    batch.norm_rope_kv_append(sh, rope, norm, x[:, :4], x[:, 4:6], x[:, 6:], pos, slots, out, kc, vc)
    batch.norm_rope_kv_append(sh, rope, norm, x[:, :4], x[:, 4:6], x[:, 6:], pos, slots, x[:, :4], kc, vc)
    assert torch.equal(out, x[:, :4])
    batch.norm_rope_kv_append(sh, rope, norm, x[:0, :4], x[:0, 4:6], x[:0, 6:], pos[:0], slots[:0], out[:0], kc, vc)
    with pytest.raises(binding.OocoError):   # q_out over k
        batch.norm_rope_kv_append(sh, rope, norm, x[:, :4], x[:, 4:6], x[:, 6:], pos, slots, x[:, 2:6], kc, vc)


# ------------------------------------------------------------------------------------------------ attention of packed chunks
def tolerance(q, k, v, mag, spread, scale, fp8):
    """bf16 outputs.  Weights are rounded to 16 bits (bf16 2^-8, f16 2^-11, below 2^-14 of the reference 2^-25 of it), the sum of
    weights is not, the output is rounded to bf16 (2^-8): both relative to sum w |v|, which bounds |out|.  Over the 8-bit cache
    the query is rounded to f16 (2^-11, or 2^-25 absolutely).  Scores are fp32 sums of exact products: 128 terms in at most 8
    instructions, 2^-15.8 of sum |q_d k_d| with their factors (see tree_tolerance.py); a score off by e changes a quotient of
    sums of weights by exp(2 e).  Exponentials, sums, merge: 2^-12."""
    weight = 2.0 ** -11 if fp8 else 2.0 ** -8
    q_err = np.maximum(2.0 ** -11 * np.abs(q).max(-1), 2.0 ** -25) if fp8 else np.zeros(q.shape[:2])
    score = 2.0 ** -15.8 * spread + q_err * np.abs(k).sum(-1).max(initial=0.0) * scale
    rel = (1 + weight) * (1 + 2.0 ** -8) - 1 + 2.0 ** -12 + np.expm1(2 * score)
    tiny = 2.0 ** -25 * k.shape[0] * np.abs(v).max(initial=0.0) if fp8 else 0.0
    return rel[..., None] * mag + tiny + 1e-30


def run_chunk(new, ctx, *, hq=8, hkv=2, D=128, bs=16, fp8=False, layout="head_major", seed=0, scale=None, pad=3, max_chunk=None,
              chunk_lens=None, strided=False, spread=1.0, check=True, holes=7, room=0):
    """Runs the call on random data (slots behind a context hold NaN, table padding is out of range) and checks every row.
    room: tokens that the table has room for, if more than the longest context."""
    rng = np.random.default_rng(seed)
    B = len(new)
    scale = scale or 1 / math.sqrt(D)
    held = [-(-max(0, t) // bs) for t in ctx]
    MB, NB = max(1, max(held), room // bs), sum(held) + holes
    perm = rng.permutation(NB)
    table, at = np.full((B, MB), 2 ** 31 - 1), 0
    for b in range(B):
        table[b, : held[b]] = perm[at: at + held[b]]
        at += held[b]
    ks, vs = (0.07, 0.11) if fp8 else (1.0, 1.0)
    g = torch.Generator(device=DEV).manual_seed(seed)
    cells = (NB, hkv, bs, D) if layout == "head_major" else (NB, bs, hkv, D)
    caches, vals = [], []
    for _ in range(2):
        x = torch.randn(cells, generator=g, device=DEV) * spread
        c = (x * 16).to(torch.float8_e4m3fn) if fp8 else x.to(torch.bfloat16)
        hm = c if layout == "head_major" else c.transpose(1, 2)
        vals.append(hm.double() * (ks if len(vals) == 0 else vs) if fp8 else hm.double())
        for b in range(B):                     # what lies behind a context is never used
            if ctx[b] > 0 and ctx[b] % bs:
                tail = hm[int(table[b, held[b] - 1])][:, ctx[b] % bs:]
                if not fp8:
                    tail.fill_(float("nan"))
        caches.append(c.view(torch.uint8) if fp8 else c)
    first = np.concatenate([[0], np.cumsum(new)])
    rows = int(first[-1]) + pad
    wide = torch.randn((rows, hq + (3 if strided else 0), D), generator=g, device=DEV).to(torch.bfloat16)
    q = wide[:, :hq]
    out_wide = torch.full((rows, hq + (2 if strided else 0), D), 5.0, dtype=torch.bfloat16, device=DEV)
    out = out_wide[:, :hq]
    max_chunk = max(1, max(new)) if max_chunk is None else max_chunk
    sh = pool_shape(B, hq, hkv, D, bs, NB, MB, layout)
    ws = torch.full((batch.chunk_workspace_bytes(sh, rows, max_chunk),), 255, dtype=torch.uint8, device=DEV)
    args = (gpu(table), gpu(ctx), gpu(first), max_chunk, scale)
    cl = None if chunk_lens is None else gpu(chunk_lens)
    call = (lambda: batch.chunk_attention_fp8(sh, q, *caches, *args, ks, vs, out, ws, chunk_lens=cl)) if fp8 else \
        (lambda: batch.chunk_attention(sh, q, *caches, *args, out, ws, chunk_lens=cl))
    call()
    if max(new) <= max_chunk:
        assert binding.workspace_status(ws) == 0
    got = host(out)
    if check:
        qh, live = host(q), np.zeros(rows, bool)
        for b in range(B):
            n = new[b] if chunk_lens is None else min(new[b], max(0, chunk_lens[b]))
            if n == 0 or n > max_chunk:
                continue
            r0, T = int(first[b]), max(0, ctx[b])
            live[r0: r0 + n] = True
            ids = torch.as_tensor(table[b, : held[b]], device=DEV).long()
            k, v = (x[ids].transpose(1, 2).flatten(0, 1)[:T].cpu().numpy() for x in vals)
            want, mag, spr = bo.chunk_attention(qh[r0: r0 + n], k, v, n, scale)
            tol = np.stack([tolerance(qh[r0: r0 + n, h: h + 1], k[:, h // (hq // hkv)], v[:, h // (hq // hkv)], mag[:, h: h + 1],
                                      spr[:, h: h + 1], scale, fp8)[:, 0] for h in range(hq)], 1)
            err = np.abs(got[r0: r0 + n] - want)
            assert not np.isnan(got[r0: r0 + n]).any(), b
            assert (err <= tol).all(), (b, float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
        assert (got[~live] == 5.0).all()
        assert strided is False or (out_wide[:, hq:] == 5.0).all()
    return out.clone(), call, ws, out


@pytest.mark.parametrize("D,fp8", [(128, False), (64, False), (128, True)])
@pytest.mark.parametrize("new,ctx", [
    ([1], [1]), ([1], [300]), ([3], [3]), ([1, 1, 1, 1], [17, 64, 130, 256]), ([0, 1, 0, 2], [50, 1, 0, 700]),
    ([5, 1, 40, 0, 33, 1], [5, 900, 41, 77, 1000, 128]), ([70, 1, 130], [70, 2000, 400]), ([7, 2], [3, 0]), ([65], [600])])
def test_chunk(new, ctx, D, fp8):
    for room in (0, 8192):   # narrow tables of few pairs are one launch
        run_chunk(new, ctx, D=D, fp8=fp8, seed=len(new) + D, room=room)


@pytest.mark.parametrize("hq,hkv,D,bs,fp8,layout", [(8, 8, 128, 32, False, "token_major"), (5, 1, 64, 16, False, "head_major"),
                                                    (16, 1, 128, 64, False, "head_major"), (10, 2, 128, 128, True, "token_major"),
                                                    (16, 1, 128, 256, True, "head_major"), (9, 1, 128, 16, False, "head_major"),
                                                    (6, 2, 64, 256, False, "token_major"), (7, 1, 128, 16, True, "head_major")])
def test_chunk_heads_blocks_layouts(hq, hkv, D, bs, fp8, layout):
    for room in (0, 8192):
        run_chunk([1, 9, 0, 30, 2], [400, 30, 9, 333, 1], hq=hq, hkv=hkv, D=D, bs=bs, fp8=fp8, layout=layout, seed=hq, strided=True, room=room)


def test_chunk_lens_and_bounds():
    for room in (0, 8192):
        run_chunk([5, 4, 3, 6], [50, 40, 30, 60], chunk_lens=[2, 9, 0, -1], seed=1, room=room)
        _, call, ws, _ = run_chunk([2, 9, 1, 4], [50, 40, 30, 60], max_chunk=4, seed=2, room=room)   # the second brings too many
        assert binding.workspace_status(ws) == 128
        ws.fill_(255)
        call()
        assert binding.workspace_status(ws) == 128


def test_chunk_splits_long_contexts():
    """One long sequence among short ones: its tokens are cut over many CTAs and merged."""
    for D, fp8 in ((128, False), (64, False), (128, True)):
        run_chunk([1, 2, 3], [20000, 70, 9000], hq=4, hkv=1, D=D, fp8=fp8, bs=64, seed=5)
    run_chunk([60], [9000], hq=8, hkv=1, D=128, bs=64, seed=6)


def test_chunk_large_scores_and_equal_runs():
    """Scores far apart raise the reference maximum again and again; equal calls give equal bits."""
    a, call, _, out = run_chunk([40, 1, 200], [500, 800, 300], spread=6.0, seed=9)
    call()
    assert torch.equal(a, out)


def test_chunk_equals_uniform_operator_within_rounding():
    """Where every sequence brings as many tokens, the uniform operator computes the same."""
    B, n, hq, hkv, D, bs, T = 3, 20, 8, 2, 128, 16, 200
    NB = B * -(-T // bs)
    g = torch.Generator(device=DEV).manual_seed(0)
    kc, vc = (torch.randn((NB, hkv, bs, D), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    table = gpu(np.random.default_rng(0).permutation(NB).reshape(B, -1))
    sh = pool_shape(B, hq, hkv, D, bs, NB, table.shape[1])
    q = torch.randn((B, n, hq, D), generator=g, device=DEV).to(torch.bfloat16)
    lens = gpu([T, T - 3, T - 60])
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws = torch.empty(binding.workspace_bytes_mq(sh, n), dtype=torch.uint8, device=DEV)
    binding.decode_attention_mq(sh, q, kc, vc, table, lens, 0.1, a, ws)
    ws = torch.empty(batch.chunk_workspace_bytes(sh, B * n, n), dtype=torch.uint8, device=DEV)
    batch.chunk_attention(sh, q.view(-1, hq, D), kc, vc, table, lens, gpu([0, n, 2 * n, 3 * n]), n, 0.1, b.view(-1, hq, D), ws)
    assert (a.double() - b.double()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -10) * vc.abs().max().double()


def test_chunk_in_a_graph_on_another_stream():
    """Captured on a side stream and replayed with other lengths in the same buffers."""
    B, hq, hkv, D, bs, MB = 4, 8, 2, 128, 16, 20
    g = torch.Generator(device=DEV).manual_seed(1)
    kc, vc = (torch.randn((B * MB, hkv, bs, D), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    table = gpu(np.random.default_rng(1).permutation(B * MB).reshape(B, MB))
    sh = pool_shape(B, hq, hkv, D, bs, B * MB, MB)
    q = torch.randn((64, hq, D), generator=g, device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(q)
    ws = torch.empty(batch.chunk_workspace_bytes(sh, 64, 40), dtype=torch.uint8, device=DEV)
    lens, first = gpu([30, 200, 320, 1]), gpu([0, 1, 11, 51, 52])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    batch.chunk_attention(sh, q, kc, vc, table, lens, first, 40, 0.1, out, ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        batch.chunk_attention(sh, q, kc, vc, table, lens, first, 40, 0.1, out, ws)
    for l, f in (([30, 200, 320, 1], [0, 1, 11, 51, 52]), ([9, 0, 33, 300], [0, 5, 5, 38, 39]), ([300] * 4, [0, 16, 32, 48, 64])):
        lens.copy_(gpu(l))
        first.copy_(gpu(f))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        again = torch.zeros_like(q)
        batch.chunk_attention(sh, q, kc, vc, table, lens, first, 40, 0.1, again, ws)
        assert torch.equal(out, again)
        assert out[f[-1]:].eq(0).all()


# ------------------------------------------------------------------------------------------------ logits
def run_logits(B, N, V, *, dtype=torch.bfloat16, pen=True, bias=0, mask=True, tree=True, temperature=True, out=True, probs=True, L=50,
               seed=0, sizes=None, special=False, pad=0, in_place=None, greedy=0):
    rng = np.random.default_rng(seed)
    x = torch.as_tensor(rng.standard_normal((B, N, V + pad)) * 3).to(dtype)
    if special:
        x[0, 0, 0], x[0, 0, V // 2], x[-1, -1, V - 1] = float("nan"), float("-inf"), float("inf")
    wide = x.to(DEV)
    logits = wide[..., :V]
    history = rng.integers(-2, V + 2, (B, L))
    history[:, L // 2:] = history[:, :1] if L > 1 else history
    lens = rng.integers(0, L + 3, B)
    prompt = rng.integers(-1, L + 1, B)
    rep, fr, pr = 1 + 0.5 * rng.random(B), rng.random(B) - 0.3, rng.random(B) - 0.3
    temp = 0.3 + rng.random(B)
    temp[:greedy] = 0.0
    tokens, parents = rng.integers(-1, V + 1, (B, N)), np.stack([np.array([-1] + [rng.integers(-1, i) for i in range(1, N)]) for _ in range(B)])
    bt = rng.integers(-1, V + 1, (B, bias)) if bias else None
    if bias > 3:
        bt[:, 1] = bt[:, 0] = bt[:, 2]
    bv = rng.standard_normal((B, bias)) * 4
    words = (V + 31) // 32
    bits = rng.integers(0, 2 ** 32, (B, N, words), dtype=np.uint64).astype(np.uint32)
    if mask and B * N > 1:
        bits[0, 0] = 0                                                # nothing is allowed
    f32 = lambda a: gpu(np.asarray(a, np.float64), torch.float32)    # noqa: E731
    kw = {}
    if pen:
        kw.update(repetition=f32(rep), frequency=f32(fr), presence=f32(pr), history=gpu(history), history_lens=gpu(lens),
                  prompt_lens=gpu(prompt))
        if tree and N > 1:
            kw.update(tokens=gpu(tokens), parents=gpu(parents))
    if temperature:
        kw["temperature"] = f32(temp)
    if bias:
        kw.update(bias_tokens=gpu(bt), bias_values=f32(bv))
    if mask:
        kw["mask"] = torch.as_tensor(bits.view(np.int32)).to(DEV)
    if sizes is not None:
        kw["tree_sizes"] = gpu(sizes)
    xh = host(logits)
    o = torch.full((B, N, V), 9.0, device=DEV) if out else None
    p = torch.full((B, N, V), 9.0, device=DEV) if probs else None
    if in_place == "out":
        o = logits
    if in_place == "probs":
        p = logits
    batch.shape_logits(logits, out=o, probs=p, **kw)
    hist = [[int(t) for t in history[b, : max(0, min(L, lens[b]))]] for b in range(B)]
    f = lambda a: float(np.float32(a))  # noqa: E731
    for b in range(B):
        for i in range(N):
            if sizes is not None and i >= sizes[b]:
                for t in (o, p):
                    assert t is None or (t[b, i] == 9.0).all()
                continue
            branch, k = [], i
            while tree and N > 1 and k > 0:
                branch.append(tokens[b, k])
                k = int(parents[b, k])
            allowed = ((bits[b, i][np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1) > 0 if mask else None
            pen_kw = dict(repetition=f(rep[b]), frequency=f(fr[b]), presence=f(pr[b]), text=hist[b],
                          prompt=max(0, min(len(hist[b]), prompt[b])), branch=branch) if pen else {}
            bias_list = [(int(t), f(z)) for t, z in zip(bt[b], bv[b])] if bias else ()
            T = f(temp[b]) if temperature else 1.0
            want, prob = bo.shape_logits(xh[b, i].copy(), temperature=T, bias=bias_list, allowed=allowed, **pen_kw)
            # every operation rounds to 2^-24 of its result; results are bounded by the sum of the terms' magnitudes
            size = 2 * np.abs(np.where(np.isfinite(xh[b, i]), xh[b, i], 0)).max() + (L + N) * 1.0 + sum(abs(z) for _, z in bias_list)
            err = (4 + len(bias_list)) * 2.0 ** -24 * size if pen or bias else 0.0
            if o is not None:
                got = host(o[b, i])
                assert np.array_equal(np.isneginf(got), np.isneginf(want)) and np.array_equal(np.isposinf(got), np.isposinf(want))
                fin = np.isfinite(want)
                assert (np.abs(got[fin] - want[fin]) <= err).all()
            if p is not None:
                got = host(p[b, i])
                assert not np.isnan(got).any()
                if T > 0:
                    # the exponent: off by 2 err / T and by three roundings of (l - r) / T, where r may lie 16 binary orders (11.1
                    # in units of T) beside the largest; exp, sum and quotient: 2^-19
                    d = np.where(prob > 0, -np.log(np.maximum(prob, 1e-300) / max(prob.max(), 1e-300)), 0)
                    rel = np.expm1(2 * err / T + 3 * 2.0 ** -24 * (d + 11.1)) + 2.0 ** -19
                    assert (np.abs(got - prob) <= rel * prob + 1e-37).all(), (b, i)
                else:
                    assert np.array_equal(got, prob)
    return o, p


@pytest.mark.parametrize("B,N,V,kw", [
    (1, 1, 1, dict()), (2, 1, 31, dict(bias=2)), (3, 5, 257, dict(special=True, bias=7)), (4, 1, 5003, dict(greedy=2)),
    (2, 16, 32000, dict(sizes=[16, 3])), (1, 1, 128256, dict(L=9000, bias=300)), (2, 1, 152064, dict(dtype=torch.float32, bias=5)),
    (3, 2, 50257, dict(special=True)), (2, 3, 1000, dict(pen=False)), (2, 3, 1000, dict(pen=False, mask=False, temperature=False)),
    (2, 3, 4099, dict(out=False)), (2, 3, 4099, dict(probs=False)), (3, 1, 4096, dict(pad=5)), (3, 1, 4096, dict(pad=8, L=1)),
    (1, 2, 300000, dict(L=100)), (1, 1, 409600, dict(mask=False, bias=3, L=40000)), (320, 1, 200, dict(bias=1, dtype=torch.float32)),
    (330, 3, 300, dict(bias=2, sizes=[i % 4 for i in range(330)])), (90, 7, 4097, dict(L=30, out=False)),   # more rows than fit the GPU at a time
    (2, 4, 777, dict(dtype=torch.float32, in_place="out", probs=True)), (2, 4, 1024, dict(dtype=torch.float32, in_place="probs"))])
def test_logits(B, N, V, kw):
    run_logits(B, N, V, seed=B + V, **kw)


@pytest.mark.parametrize("V", [700, 40000])
def test_logits_whose_largest_falls(V):
    """The largest logit is named by the text and falls a little, far, to just above the rest, or behind everything; or it rises."""
    falls = [0.0, 1.0, 9.0, 20.0, 26.0, 27.5, 60.0, 300.0, -5.0, float("inf")]
    B = len(falls)
    g = torch.Generator().manual_seed(V)
    x = torch.randn((B, V), generator=g)
    x[:, 5] = 30.0
    x[1, 17] = 29.5
    text = torch.tensor([5, 40, 77, 5, 300])
    pres = torch.tensor(falls)
    out, probs = torch.empty((B, V), device=DEV), torch.empty((B, V), device=DEV)
    for temp in (0.25, 1.0, 0.0):
        t = torch.full((B,), temp)
        batch.shape_logits(x.to(DEV), temperature=t.to(DEV), presence=pres.to(DEV), history=gpu(text.repeat(B, 1)),
                           history_lens=gpu([5] * B), out=out, probs=probs)
        want = x.double().clone()
        want[:, text.unique()] -= pres.double()[:, None]
        want[torch.isnan(want)] = -math.inf
        got, p = host(out), host(probs)
        fin = np.isfinite(want.numpy())
        assert np.array_equal(np.isfinite(got), fin)
        assert (np.abs(got[fin] - want.numpy()[fin]) <= 2.0 ** -24 * 330).all()           # one rounding of at most 330
        if temp == 0.0:
            assert np.array_equal(p.argmax(-1), got.argmax(-1)) and (p.sum(-1) == 1).all()
            continue
        z = torch.from_numpy(got).double() / temp                                       # of the logits as they were rounded
        prob = torch.softmax(z, -1).numpy()
        d = np.where(prob > 0, (z.max(-1, keepdim=True).values - z).numpy(), 0)
        rel = np.expm1(3 * 2.0 ** -24 * (d + 11.1)) + 2.0 ** -19                     # as in run_logits
        assert (np.abs(p - prob) <= rel * prob + 1e-37).all()


def test_logits_equal_runs_and_shared_masks():
    a = run_logits(3, 2, 9000, seed=4, out=False)[1]
    b = run_logits(3, 2, 9000, seed=4, out=False)[1]
    assert torch.equal(a, b)
    x = torch.randn((3, 100), device=DEV)
    mask = torch.full((4,), 0x0f0f0f0f, dtype=I32, device=DEV)
    p, q = torch.empty_like(x), torch.empty_like(x)
    batch.shape_logits(x, probs=p, mask=mask.expand(3, 4))
    batch.shape_logits(x, probs=q, mask=mask.repeat(3, 1))
    assert torch.equal(p, q) and (p[:, 4:8] == 0).all() and (p[:, :4] > 0).all()


def test_logits_greedy_ties_and_odd_temperatures():
    x = torch.zeros((5, 1000), device=DEV)
    x[:, 700] = x[:, 300] = 2.0
    t = torch.tensor([0.0, -1.0, float("nan"), float("inf"), 1e-40], device=DEV)
    p = torch.empty_like(x)
    batch.shape_logits(x, probs=p, temperature=t)
    for r in (0, 1, 2):
        assert p[r, 300] == 1 and p[r].sum() == 1
    assert torch.allclose(p[3], torch.full((1000,), 1e-3, device=DEV), rtol=1e-5)
    assert p[4, 300] == 0.5 and p[4, 700] == 0.5 and p[4].sum() == 1


def test_logits_huge_values_and_temperatures():
    """Products of logit and factor that overflow, infinite logits at an infinite temperature; in one CTA and across a cluster."""
    inf = float("inf")
    for V in (8, 30000):
        x = torch.full((6, V), -3e38, device=DEV)
        x[:, 1], x[:, V - 2], x[:, 3] = 3e38, 3e38, 1.0
        x[2, 5] = inf
        x[3, 5], x[4, 5] = inf, 2.9e38
        t = torch.tensor([0.25, 1.0, inf, 0.25, 1e37, inf], device=DEV)
        p = torch.empty_like(x)
        batch.shape_logits(x, probs=p, temperature=t)
        assert not torch.isnan(p).any()
        for row in (0, 1):
            assert p[row, 1] == 0.5 and p[row, V - 2] == 0.5 and p[row].sum() == 1
        for row in (2, 3):
            assert p[row, 5] == 1 and p[row].sum() == 1
        want = torch.softmax(x[4].double() / t[4].double(), 0)
        # differences of exponents of up to 87 binary orders: factor and difference rounded, 2 * 2^-24 * 87 * ln 2 = 7.2e-6; exp, sum, quotient 2^-19
        assert torch.allclose(p[4].double(), want, rtol=1e-5, atol=1e-37)
        assert torch.allclose(p[5], torch.full_like(p[5], 1.0 / V), rtol=1e-5)


# ------------------------------------------------------------------------------------------------ together
def test_one_step_of_a_mixed_batch():
    """Fork, slots, norms with rotation and append, attention, logits, in this order, as a serving loop runs them: two
    decodes, a prompt and a fork of it, against plain attention over what each sequence has been given."""
    rng = np.random.default_rng(2)
    B, hq, hkv, D, bs, V, MB, NB = 4, 8, 2, 64, 16, 500, 8, 40
    sh = pool_shape(B, hq, hkv, D, bs, NB, MB)
    g = torch.Generator(device=DEV).manual_seed(3)
    kc, vc = (torch.randn((NB, hkv, bs, D), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    ctx, held, table, free, _ = np.array([37, 5, 0, 0]), np.array([3, 1, 0, 0]), np.full((B, MB), -1), np.arange(4, NB), NB
    table[0, :3], table[1, 0] = [0, 1, 2], 3
    t = dict(ctx=gpu(ctx), table=gpu(table), held=gpu(held), head=gpu([0]), shares=gpu(np.zeros(NB)), free=gpu(free))
    src, dst, granted = (torch.empty(1, dtype=I32, device=DEV) for _ in range(3))
    ws = torch.empty(batch.pages_workspace_bytes(sh, 1), dtype=torch.uint8, device=DEV)
    batch.fork_pages(sh, gpu([0]), gpu([3]), t["ctx"], t["table"], t["held"], t["free"], t["head"], t["shares"], src, dst, granted, ws)
    binding.kv_copy_blocks(sh, kc, vc, src, dst)
    new = np.array([1, 1, 30, 4])
    rows = int(new.sum())
    slot, pos = (torch.empty(rows, dtype=I32, device=DEV) for _ in range(2))
    first, got, total = torch.empty(B + 1, dtype=I32, device=DEV), *(torch.empty(B, dtype=I32, device=DEV) for _ in range(2))
    ws2 = torch.empty(spec.plan_slots_workspace_bytes(sh), dtype=torch.uint8, device=DEV)
    spec.plan_slots(sh, t["ctx"], gpu(new), t["table"], t["held"], t["free"], t["head"], slot, pos, first, got, total, ws2)
    before = [kc.clone(), vc.clone()]
    qkv = torch.randn((rows, hq + 2 * hkv, D), generator=g, device=DEV).to(torch.bfloat16)
    inv, _ = spec.rope_frequencies(D)
    q = torch.empty((rows, hq, D), dtype=torch.bfloat16, device=DEV)
    batch.norm_rope_kv_append(sh, spec.Rope(D, False, inv.to(DEV)), batch.HeadNorm(1e-6), qkv[:, :hq], qkv[:, hq: hq + hkv],
                              qkv[:, hq + hkv:], pos, slot, q, kc, vc)
    out = torch.empty_like(q)
    ws3 = torch.empty(batch.chunk_workspace_bytes(sh, rows, 30), dtype=torch.uint8, device=DEV)
    batch.chunk_attention(sh, q, kc, vc, t["table"], total, first, 30, 0.125, out, ws3, chunk_lens=got)
    assert got.tolist() == new.tolist() and total.tolist() == [38, 6, 30, 41]
    tb, f = t["table"].cpu().numpy(), first.tolist()
    for b in range(B):
        T, n = int(total[b]), int(new[b])
        ids = torch.as_tensor(tb[b, : -(-T // bs)], device=DEV).long()
        k, v = (host(x[ids].transpose(1, 2).flatten(0, 1)[:T]) for x in (kc, vc))
        want, mag, spr = bo.chunk_attention(host(q[f[b]: f[b] + n]), k, v, n, 0.125)
        tol = tolerance(host(q[f[b]: f[b] + n]), k.reshape(T, -1), v, mag, spr, 0.125, False)
        assert (np.abs(host(out[f[b]: f[b] + n]) - want) <= tol).all(), b
    # the fork left its parent's rows alone: what row 0 held before its own token is unchanged
    ids = torch.as_tensor(tb[0, :3], device=DEV).long()
    for x, y in zip((kc, vc), before):
        assert torch.equal(x[ids].transpose(1, 2).flatten(0, 1)[:37], y[ids].transpose(1, 2).flatten(0, 1)[:37])
    # last rows to logits, one of them greedy, then a draw by the verification of a chain without drafts
    last = (first[1:].long() - 1)
    logits = (out[last].flatten(1).float() @ torch.randn((hq * D, V), generator=g, device=DEV)).view(B, 1, V)
    probs = torch.empty_like(logits)
    batch.shape_logits(logits, probs=probs, temperature=torch.tensor([0.0, 1.0, 0.7, 1.3], device=DEV))
    path, tok = (torch.empty((B, 1), dtype=I32, device=DEV) for _ in range(2))
    count = torch.empty(B, dtype=I32, device=DEV)
    spec.verify_drafts(probs, None, torch.zeros((B, 1), dtype=I32, device=DEV), None, torch.full((B, 1), 0.5, device=DEV), path, tok, count)
    assert int(tok[0, 0]) == int(logits[0, 0].argmax())
    assert all(float(probs[b, 0, int(tok[b, 0])]) > 0 for b in range(B))
