"""The speculative-decoding operators on the GPU against their 64-bit definitions, through the C ABI."""
import math

import numpy as np
import pytest
import torch

from oracle import spec_oracle as so
from paper_2511_21862_b200 import binding, build, inputs, spec
from util import fp32_output

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


def as_head_major(cache, layout):
    """[NB, Hkv, bs, D] view of a pool."""
    return cache if layout == "head_major" else cache.transpose(1, 2)


def empty_pool(NB, hkv, bs, D, layout, dtype=torch.bfloat16):
    return torch.empty((NB, hkv, bs, D) if layout == "head_major" else (NB, bs, hkv, D), dtype=dtype, device=DEV)


# ------------------------------------------------------------------------------------------------ plan_slots
def run_slots(ctx, new, table, held, free, head, *, bs, NB, row_len=0, rows=None, parents=None, in_place=False):
    B, MB = table.shape
    rows = rows if rows is not None else (B * row_len if row_len else int(np.maximum(new, 0).sum()))
    sh = pool_shape(B, 1, 1, 64, bs, NB, MB)
    t = dict(table=gpu(table), held=gpu(held), head=gpu([head]), slot=torch.full((rows,), -77, dtype=I32, device=DEV),
             pos=torch.full((rows,), -77, dtype=I32, device=DEV), first=gpu(np.zeros(B + 1)), granted=gpu(np.zeros(B)),
             total=gpu(np.zeros(B)), status=gpu([0]))
    held_out, head_out = (None, None) if in_place else (gpu(np.zeros(B)), gpu([0]))
    ws = torch.full((spec.plan_slots_workspace_bytes(sh),), 255, dtype=torch.uint8, device=DEV)
    spec.plan_slots(sh, gpu(ctx), gpu(new), t["table"], t["held"], gpu(free), t["head"], t["slot"], t["pos"], t["first"],
                    t["granted"], t["total"], ws, row_len=row_len, parents=None if parents is None else gpu(parents),
                    blocks_held_out=held_out, free_head_out=head_out, status=t["status"])
    want = so.plan_slots(np.asarray(ctx), np.asarray(new), np.asarray(table), np.asarray(held), np.asarray(free), head,
                         block_size=bs, num_blocks=NB, row_len=row_len, num_rows=rows, parents=parents)
    got = dict(table=t["table"], slot_map=t["slot"], positions=t["pos"], first_token=t["first"], granted=t["granted"],
               total=t["total"], held=t["held"] if in_place else held_out)
    for k, v in got.items():
        assert np.array_equal(v.cpu().numpy(), want[k]), k
    assert int(t["head"] if in_place else head_out) == want["head"] and int(t["status"]) == want["status"]
    if not in_place:
        assert np.array_equal(t["held"].cpu().numpy(), held) and int(t["head"]) == head
    return want


def slots_case(seed, B, bs, ctx_hi, new_hi, short=0, extra_held=0):
    rng = np.random.default_rng(seed)
    ctx, new = rng.integers(0, ctx_hi + 1, B), rng.integers(0, new_hi + 1, B)
    held = -(-ctx // bs) + rng.integers(0, extra_held + 1, B)
    MB = max(1, int((-(-(ctx + new) // bs)).max()), int(held.max()))
    need = int(np.maximum(0, -(-(ctx + new) // bs) - held).sum())
    NB = int(held.sum()) + need + 8
    perm = rng.permutation(NB)
    table, at = np.full((B, MB), -1), 0
    for b in range(B):
        table[b, : held[b]] = perm[at: at + held[b]]
        at += held[b]
    return ctx, new, table, held, np.concatenate([[-5, -6], perm[at: at + max(0, need - short)]]), 2, dict(bs=bs, NB=NB)


@pytest.mark.parametrize("B,bs,ctx_hi,new_hi,row_len,short,extra", [
    (1, 16, 0, 1, 0, 0, 0), (1, 16, 40, 1, 1, 0, 0), (7, 16, 100, 5, 0, 0, 0), (7, 32, 100, 5, 5, 0, 2),
    (64, 16, 500, 16, 19, 0, 1), (64, 256, 500, 16, 16, 3, 0), (300, 16, 50, 40, 0, 0, 0), (33, 64, 1000, 700, 0, 5, 0),
    (1025, 16, 30, 9, 9, 0, 0), (2500, 16, 20, 3, 0, 40, 0), (5, 16, 10, 4001, 0, 0, 0), (3, 128, 10, 2001, 2001, 0, 3)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_slots(B, bs, ctx_hi, new_hi, row_len, short, extra, in_place):
    ctx, new, table, held, free, head, kw = slots_case(B * 7 + bs, B, bs, ctx_hi, new_hi, short, extra)
    want = run_slots(ctx, new, table, held, free, head, row_len=row_len, in_place=in_place, **kw)
    assert (want["status"] != 0) == (short > 0)


@pytest.mark.parametrize("B,new_hi,row_len", [(40000, 2, 0), (30000, 3, 3), (9, 60000, 0), (600, 400, 0)])
def test_plan_slots_many_rows(B, new_hi, row_len):
    """Rows over many CTAs: runs of sequences without new tokens, sequences that end inside a thread's rows."""
    ctx, new, table, held, free, head, kw = slots_case(B, B, 16, 20, new_hi)
    new[B // 3: B // 2] = 0
    run_slots(ctx, new, table, held, free, head, row_len=row_len, **kw)


def test_plan_slots_tree_positions():
    rng = np.random.default_rng(5)
    for B, L in ((3, 7), (40, 64), (9, 256), (700, 12)):
        ctx, new, table, held, free, head, kw = slots_case(L, B, 16, 60, L, 0, 0)
        par = np.stack([[-1] + [int(rng.integers(-1, i)) for i in range(1, L)] for _ in range(B)])
        par[0] = np.arange(L) - 1               # a chain
        par[1] = rng.integers(-3, L + 3, L)      # values that are no parents count as none
        run_slots(ctx, new, table, held, free, head, row_len=L, parents=par.reshape(-1), **kw)


def test_plan_slots_refuses_whole_sequences():
    # (a) padded rows too short for one, (b) packed rows too few, (c) a table row too short, (d) held does not cover ctx
    table = np.array([[0, -1, -1], [1, -1, -1], [2, 3, -1]])
    base = dict(bs=16, NB=20)
    free = np.arange(5, 15)
    w = run_slots([10, 5, 20], [4, 9, 4], table, [1, 1, 2], free, 0, row_len=5, **base)
    assert list(w["granted"]) == [4, 0, 4]
    w = run_slots([10, 5, 20], [4, 9, 4], table, [1, 1, 2], free, 0, rows=9, **base)
    assert list(w["granted"]) == [4, 0, 0]
    w = run_slots([10, 40, 20], [4, 9, 30], table, [1, 3, 2], free, 0, rows=64, **base)
    assert list(w["granted"]) == [4, 0, 0]      # 49 and 50 tokens in rows of 48
    w = run_slots([10, 17, 20], [4, 9, 4], table, [1, 1, 2], free, 0, rows=64, **base)
    assert list(w["granted"]) == [4, 0, 4]
    # negative lengths count as none; blocks outside the pool only lose their slots
    w = run_slots([-3, 5, 20], [4, -9, 14], table, [0, 1, 2], [20, -1, 7], 0, rows=40, **base)
    assert w["status"] == 4 and list(w["granted"]) == [4, 0, 14] and set(w["slot_map"][:4]) == {-1}
    # no rows at all, and an empty free list
    run_slots([3, 5, 0], [0, 0, 0], table, [1, 1, 2], free[:0], 0, rows=0, **base)


# ------------------------------------------------------------------------------------------------ rope_kv_append
E4M3 = torch.float8_e4m3fn


def rope_case(T, hq, hkv, D, rot, inter, bs, layout, fp8, seed, pos_hi=1 << 20, fused=True, magnitude=1.0):
    g = torch.Generator().manual_seed(seed)
    NB = -(-T // bs) + 3
    if fused:
        qkv = torch.randn((T, (hq + 2 * hkv) * D + 8), generator=g).to(torch.bfloat16).to(DEV)
        q, k, v = (qkv[:, a * D: b * D].unflatten(1, (b - a, D)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    else:
        q, k, v = (torch.randn((T, h, D), generator=g).to(torch.bfloat16).to(DEV) for h in (hq, hkv, hkv))
    pos = torch.randint(0, pos_hi, (T,), generator=g, dtype=I32)
    slots = torch.randperm(NB * bs, generator=g)[:T].to(I32)
    if T > 4:
        pos[1], slots[2], slots[3] = -1, -1, NB * bs   # padding, and two rows without a slot
    inv, _ = spec.rope_frequencies(rot, 10000.0)
    shape = pool_shape(1, hq, hkv, D, bs, NB, 1, layout)
    kc, vc = (empty_pool(NB, hkv, bs, D, layout, torch.uint8 if fp8 else torch.bfloat16) for _ in range(2))
    for c in (kc, vc):
        c.view(torch.uint8).fill_(0x3c)
    return shape, spec.Rope(rot, inter, inv.to(DEV), magnitude), q, k, v, pos.to(DEV), slots.to(DEV), kc, vc


def check_rope(shape, rope, q, k, v, pos, slots, q_in, k_in, q_out, kc, vc, layout, scales, sentinel):
    p, s = pos.cpu().numpy(), slots.cpu().numpy()
    inv = rope.inv_freq.cpu().numpy()
    bs, n_slots = shape.block_size, shape.num_blocks * shape.block_size
    for x, got, sc in ((q_in, q_out, None), (k_in, kc, scales and scales[0]), (v, vc, scales and scales[1])):
        x64 = x.cpu().double().numpy()
        turned = x is not v
        want = so.rope(x64, np.maximum(p, 0), inv, rope.rot_dim, rope.interleaved, rope.magnitude) if turned else x64
        # fp32 arithmetic: reduced angle 2^-24 relative of up to pi, sine and cosine 2^-23, two products and a sum
        arith = 1e-6 * rope.magnitude * (np.abs(x64).max(-1, keepdims=True) * 2) if turned else 0.0
        if got is q_out:
            rows = [r for r in range(len(p)) if p[r] >= 0]
            res = q_out.cpu().double().numpy()
            tol = 2.0 ** -8 * np.abs(want) + arith
            assert np.all(np.abs(res - want)[rows] <= tol[rows])
            untouched = [r for r in range(len(p)) if p[r] < 0]
            if sentinel is not None:
                assert torch.equal(q_out[untouched].view(torch.int16), sentinel[untouched].view(torch.int16))
            continue
        flat = as_head_major(got, layout).permute(0, 2, 1, 3).reshape(n_slots, shape.num_kv_heads, shape.head_dim)
        rows = [r for r in range(len(p)) if p[r] >= 0 and 0 <= s[r] < n_slots]
        at = torch.as_tensor(s[rows], device=DEV).long()
        if sc is None:
            res = flat[at].cpu().double().numpy()
            if turned:
                assert np.all(np.abs(res - want[rows]) <= 2.0 ** -8 * np.abs(want[rows]) + arith[rows])
            else:
                assert torch.equal(flat[at].view(torch.int16), v[torch.as_tensor(rows, device=DEV).long()].contiguous().view(torch.int16))
        else:
            res = flat[at].view(E4M3).cpu().double().numpy()
            y = np.clip(want[rows] / sc, -448, 448)
            # half a step: 2^-4 relative, 2^-10 among the subnormals; the division and arithmetic before it in fp32
            slack = (arith[rows] if turned else 0.0) / sc + 2.0 ** -23 * np.abs(y)
            assert np.all(np.abs(res - y) <= np.maximum(2.0 ** -4 * (np.abs(y) + slack), 2.0 ** -10) + slack)
        other = torch.ones(n_slots, dtype=torch.bool, device=DEV)
        other[at] = False
        assert bool((flat[other].contiguous().view(torch.uint8) == 0x3c).all())   # no other slot was written


@pytest.mark.parametrize("T,hq,hkv,D,rot,inter,bs,layout", [
    (1, 32, 8, 128, 128, False, 16, "head_major"), (1, 8, 2, 64, 64, True, 16, "token_major"),
    (5, 8, 2, 64, 16, False, 16, "head_major"), (40, 40, 8, 128, 128, True, 32, "head_major"),
    (37, 16, 1, 128, 48, False, 64, "token_major"), (33, 7, 7, 64, 32, True, 16, "head_major"),
    (700, 8, 2, 128, 96, False, 256, "head_major"), (1500, 4, 1, 64, 64, True, 128, "head_major")])
@pytest.mark.parametrize("fp8", [False, True])
def test_rope_kv_append(T, hq, hkv, D, rot, inter, bs, layout, fp8):
    if fp8 and D != 128:
        pytest.skip("the 8-bit cache has head_dim 128")
    magnitude = 1.0 if T % 2 else 1.25
    sh, rope, q, k, v, pos, slots, kc, vc = rope_case(T, hq, hkv, D, rot, inter, bs, layout, fp8, T + rot, magnitude=magnitude)
    out = torch.full((T, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    sent = out.clone()
    if fp8:
        spec.rope_kv_append_fp8(sh, rope, q, k, v, pos, slots, out, kc, vc, 0.021, 0.004)
    else:
        spec.rope_kv_append(sh, rope, q, k, v, pos, slots, out, kc, vc)
    check_rope(sh, rope, q, k, v, pos, slots, q, k, out, kc, vc, layout, (0.021, 0.004) if fp8 else None, sent)


@pytest.mark.parametrize("inter", [False, True])
def test_rope_in_place_and_strided_output(inter):
    sh, rope, q, k, v, pos, slots, kc, vc = rope_case(21, 8, 2, 128, 64, inter, 16, "head_major", False, 3)
    before = q.clone()
    wide = torch.full((21, 8 * 128 + 16), 3.0, dtype=torch.bfloat16, device=DEV)
    out = wide[:, 16:].unflatten(1, (8, 128))
    spec.rope_kv_append(sh, rope, q, k, v, pos, slots, out, kc, vc)
    assert bool((wide[:, :16] == 3.0).all())
    spec.rope_kv_append(sh, rope, q, k, v, pos, slots, q, kc, vc)
    check_rope(sh, rope, q, k, v, pos, slots, before, k, q.contiguous(), kc, vc, "head_major", None, before.contiguous())
    live = pos >= 0
    assert torch.equal(out[live].contiguous().view(torch.int16), q[live].contiguous().view(torch.int16))


def test_rope_no_tokens_and_refusals():
    sh, rope, q, k, v, pos, slots, kc, vc = rope_case(6, 8, 2, 128, 64, False, 16, "head_major", False, 4)
    spec.rope_kv_append(sh, rope, q[:0], k[:0], v[:0], pos[:0], slots[:0], q[:0], kc, vc)
    with pytest.raises(ValueError):
        spec.rope_kv_append(sh, rope, q.float(), k, v, pos, slots, q, kc, vc)
    with pytest.raises(ValueError):
        spec.rope_kv_append(sh, rope, q, k, v, pos.long(), slots, q, kc, vc)
    with pytest.raises(ValueError):
        spec.rope_kv_append(sh, rope, q, k, v, pos, slots, q, kc[:-1], vc)
    with pytest.raises(binding.OocoError):
        spec.rope_kv_append(sh, spec.Rope(24, False, torch.ones(12, device=DEV)), q, k, v, pos, slots, q, kc, vc)


# ------------------------------------------------------------------------------------------------ tree attention
def random_parents(rng, B, N, kind="tree"):
    if kind == "chain":
        return np.tile(np.arange(N) - 1, (B, 1))
    if kind == "star":
        return np.tile(np.array([-1] + [0] * (N - 1)), (B, 1))
    if kind == "forest":                              # several roots, entries that are no parents among them
        return np.stack([[-1] + [int(rng.integers(-3, i + 2)) if rng.random() < 0.3 else int(rng.integers(-1, i))
                                 for i in range(1, N)] for _ in range(B)])
    return np.stack([[-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, N)] for _ in range(B)])


def tree_case(lens, hq, hkv, D, bs, N, seed, *, sizes=None, layout="head_major", kind="tree", fp8=None, sigma=1.0, pad=3):
    rng = np.random.default_rng(seed)
    B = len(lens)
    lens = np.asarray(lens)
    nblk = -(-lens // bs)
    NB, MB = int(nblk.sum()) + pad, max(1, int(nblk.max())) + 1
    perm = rng.permutation(NB)
    table, at = np.full((B, MB), 2 ** 31 - 1, dtype=np.int64), 0
    dead = np.ones((NB, bs), bool)
    for b in range(B):
        ids = perm[at: at + nblk[b]]
        table[b, : nblk[b]] = ids
        at += nblk[b]
        for j, blk in enumerate(ids):
            dead[blk, : max(0, min(bs, lens[b] - j * bs))] = False
    g = torch.Generator(device=DEV).manual_seed(seed)
    caches = []
    for i in range(2):
        x = torch.randn((NB, hkv, bs, D), generator=g, device=DEV) * sigma
        if fp8:
            x = (x / fp8[i]).clamp(-448, 448).to(E4M3).view(torch.uint8)
            x[torch.as_tensor(dead, device=DEV)[:, None].expand(NB, hkv, bs)] = 0x7f       # NaN in every slot not in use
        else:
            x = x.to(torch.bfloat16)
            x[torch.as_tensor(dead, device=DEV)[:, None].expand(NB, hkv, bs)] = float("nan")
        caches.append((x if layout == "head_major" else x.transpose(1, 2)).contiguous())
    q = (torch.randn((B, N, hq, D), generator=g, device=DEV) * sigma).to(torch.bfloat16)
    par = random_parents(rng, B, N, kind)
    if sizes is not None:
        for b in range(B):
            q[b, max(0, min(N, int(sizes[b]))):] = float("nan")                                # rows of nodes that do not exist
    return dict(lens=lens, table=table, par=par, sizes=sizes, q=q, k=caches[0], v=caches[1], N=N, hq=hq, hkv=hkv, D=D, bs=bs,
                shape=pool_shape(B, hq, hkv, D, bs, NB, MB, layout), layout=layout, fp8=fp8, scale=1 / math.sqrt(D))


def run_tree(c, f32=False, stream=None, ws=None):
    ws = ws if ws is not None else torch.full((spec.tree_workspace_bytes(c["shape"], c["N"]),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full(c["q"].shape, 11.0, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    tail = dict(tree_sizes=None if c["sizes"] is None else gpu(c["sizes"]), stream=stream)
    args = (c["shape"], c["q"], c["k"], c["v"], gpu(c["table"].astype(np.int32)), gpu(c["lens"]), gpu(c["par"]), c["scale"])
    if c["fp8"]:
        spec.tree_attention_fp8(*args, *c["fp8"], out, ws, **tail)
    else:
        spec.tree_attention(*args, out, ws, **tail)
    assert binding.workspace_status(ws, stream) == 0
    torch.cuda.synchronize()
    return out


def check_tree(c, out32, out16, seqs=None):
    B, N, hq, hkv, D, bs = len(c["lens"]), c["N"], c["hq"], c["hkv"], c["D"], c["bs"]
    G = hq // hkv
    q = c["q"].cpu().double().numpy()
    km, vm = (as_head_major(x, c["layout"]) for x in (c["k"], c["v"]))
    o32, o16 = out32.cpu().double().numpy(), out16.cpu()
    assert torch.equal(o16.view(torch.int16), out32.cpu().to(torch.bfloat16).view(torch.int16))
    for b in range(B):
        T = int(c["lens"][b])
        n = N if c["sizes"] is None else max(0, min(N, int(c["sizes"][b])))
        assert np.all(o32[b, n:] == 11.0)             # rows of nodes that do not exist are left as they were
        if n == 0 or (seqs is not None and b not in seqs):
            continue
        ids = torch.as_tensor(c["table"][b, : -(-T // bs)], device=DEV).long()
        k, v = ((x[ids].view(E4M3).double() * s if c["fp8"] else x[ids].double()).permute(1, 0, 2, 3).flatten(1, 2)[:, :T].cpu().numpy()
                for x, s in ((km, c["fp8"] and c["fp8"][0]), (vm, c["fp8"] and c["fp8"][1])))
        for h in range(hkv):
            want, mag, spread = so.tree_attention(q[b, :n, h * G:(h + 1) * G], k[h], v[h], c["par"][b], n, c["scale"])
            # weights rounded to 16 bits in numerator and denominator (2^-8 each for bf16, f16 is finer); over the
            # 8-bit cache the query too (at least as fine as bf16's 2^-8 per dim, so the scores are off by at most
            # 2^-8 of sum |q_d k_d|, and a weight by twice that); fp32 sums add 2^-24 per term
            tol = (2.0 ** -7 + 1e-4 + (2 * 2.0 ** -8 * spread[..., None] if c["fp8"] else 0)) * mag + 1e-6
            err = np.abs(o32[b, :n, h * G:(h + 1) * G] - want)
            assert np.all(err <= tol), (b, h, float((err / np.maximum(tol, 1e-30)).max()))


def both(c, **kw):
    o16 = run_tree(c)
    with fp32_output():
        o32 = run_tree(c, f32=True)
    check_tree(c, o32, o16, **kw)
    return o16


TREE_CASES = {
    # name: (lens, hq, hkv, D, bs, N, options); columns = hq / hkv * N choose the kernel
    "n1": ([1, 2, 16, 17, 300], 32, 8, 128, 16, 1, {}),
    "cols8-decode": ([2, 3, 15, 16, 17, 64, 65, 130, 700], 32, 8, 128, 16, 2, {}),
    "cols8-g1": ([8, 9, 23, 24, 25, 64, 200], 4, 4, 128, 16, 8, {}),
    "cols8-d64": ([5, 17, 64, 130, 256], 8, 2, 64, 16, 2, {}),
    "cols5-d64": ([5, 17, 64, 130, 256], 2, 2, 64, 16, 5, dict(kind="star")),
    "cols16-row16": ([4, 5, 15, 16, 17, 63, 64, 65, 66, 67, 68, 69, 300], 32, 8, 128, 16, 4, {}),
    "cols16-g1-forest": ([16, 17, 31, 33, 64, 100, 500], 4, 4, 128, 32, 16, dict(kind="forest")),
    "cols15-d64": ([3, 64, 65, 66, 67, 130], 10, 2, 64, 16, 3, {}),
    "cols20-tc2": ([5, 6, 64, 65, 127, 128, 129, 132, 133, 400], 32, 8, 128, 16, 5, {}),
    "cols64-tc2": ([16, 17, 64, 100, 128, 130, 140, 1000], 32, 8, 128, 16, 16, {}),
    "cols128-tc2": ([32, 33, 100, 128, 129, 159, 160, 161, 900], 32, 8, 128, 32, 32, dict(kind="forest")),
    "cols132-tc2-two-tiles": ([33, 60, 128, 160, 161, 700], 32, 8, 128, 16, 33, {}),
    "cols320-tc2": ([64, 70, 128, 191, 192, 193, 1200], 40, 8, 128, 16, 64, {}),
    "cols512-n256": ([256, 257, 300, 383, 384, 700], 8, 4, 128, 64, 256, dict(kind="forest")),
    "cols400-n200-chain": ([200, 333, 512], 8, 4, 128, 16, 200, dict(kind="chain")),
    "d64-chunk-32": ([9, 63, 64, 70, 72, 73, 300], 8, 2, 64, 16, 8, {}),
    "d64-chunk-64": ([16, 64, 80, 81, 300], 8, 2, 64, 32, 16, dict(kind="forest")),
    "d64-chunk-n130": ([130, 140, 192, 500], 8, 2, 64, 16, 130, {}),
    "short-context": ([0, 1, 2, 3, 4, 5, 6, 7], 32, 8, 128, 16, 6, {}),          # fewer tokens than nodes
    "short-context-small": ([0, 1, 2, 1, 2], 8, 8, 128, 16, 3, {}),
    "ragged-small": ([10, 20, 30, 40, 64, 1], 8, 4, 128, 16, 4, dict(sizes=[0, 1, 2, 4, 3, 1])),
    "ragged-row16": ([10, 20, 30, 40, 64, 65], 16, 4, 128, 16, 4, dict(sizes=[0, 1, 2, 4, 3, -2])),
    "ragged-tc2": ([10, 200, 130, 64, 65, 0, 1], 32, 8, 128, 16, 10, dict(sizes=[0, 1, 10, 7, 99, 5, 1])),
    "ragged-two-tiles": ([70, 200, 130, 64], 40, 8, 128, 16, 48, dict(sizes=[48, 1, 25, 26])),
    "ragged-d64": ([70, 200, 130, 64], 8, 2, 64, 16, 12, dict(sizes=[12, 0, 5, 1])),
    "token-major": ([40, 100, 129], 16, 4, 128, 16, 12, dict(layout="token_major")),
    "split-small": ([5000, 4097, 9], 32, 8, 128, 16, 2, {}),
    "split-row16": ([5000, 2049, 2050, 2051, 70], 32, 8, 128, 16, 4, dict(sizes=[4, 3, 4, 1, 0])),
    "split-tc2": ([9000, 2049, 2063, 2064, 70], 32, 8, 128, 16, 16, dict(sizes=[16, 7, 16, 16, 1])),
    "split-two-tiles": ([9000, 4100], 64, 8, 128, 32, 40, {}),
    "split-d64": ([6000, 2050, 100], 8, 2, 64, 16, 9, {}),
    "fp8-cols8": ([2, 15, 16, 17, 127, 128, 129, 130, 700], 32, 8, 128, 16, 2, dict(fp8=(0.02, 0.03))),
    "fp8-cols16": ([4, 127, 128, 129, 130, 131, 132, 3000], 32, 8, 128, 16, 4, dict(fp8=(0.02, 0.03), sizes=[4, 4, 4, 4, 3, 4, 1, 4])),
    "fp8-cols40-tc2": ([8, 100, 128, 130, 135, 136, 2500], 40, 8, 128, 16, 8, dict(fp8=(0.02, 0.03))),
    "fp8-cols128-ragged": ([40, 128, 159, 300], 32, 8, 128, 16, 32, dict(fp8=(0.02, 0.03), sizes=[3, 32, 31, 0])),
    "fp8-cols256-tc": ([64, 100, 127, 128, 129, 900], 32, 8, 128, 16, 64, dict(fp8=(0.02, 0.03), kind="forest")),
    "fp8-cols200-ragged-split": ([5000, 70], 40, 8, 128, 32, 40, dict(fp8=(0.02, 0.03), sizes=[40, 13])),
}


@pytest.mark.parametrize("name", list(TREE_CASES))
def test_tree_attention(name):
    lens, hq, hkv, D, bs, N, opt = TREE_CASES[name]
    both(tree_case(lens, hq, hkv, D, bs, N, seed=sum(map(ord, name)), sigma=0.7, **opt))


def test_tree_attention_chain_is_causal_attention():
    """A chain over the same inputs is the causal operator, bit for bit where both run the same kernels (9 to 64 score
    columns have a kernel of their own for trees)."""
    for N, hq, hkv in ((2, 32, 8), (1, 64, 8), (40, 32, 8)):
        c = tree_case([N, 100, 300, 3000], hq, hkv, 128, 16, N, seed=N, kind="chain")
        got = run_tree(c)
        out = torch.empty_like(c["q"])
        ws = torch.empty(binding.workspace_bytes_mq(c["shape"], N), dtype=torch.uint8, device=DEV)
        binding.decode_attention_mq(c["shape"], c["q"], c["k"], c["v"], gpu(c["table"].astype(np.int32)), gpu(c["lens"]), c["scale"], out, ws)
        assert bool((got.view(torch.int16) == out.view(torch.int16)).all()), N


@pytest.mark.parametrize("fp8", [None, (0.02, 0.03)], ids=["bf16", "fp8"])
@pytest.mark.parametrize("hq,N", [(16, 9), (40, 8), (32, 16), (48, 16)])
def test_tree_attention_many_short_units(hq, N, fp8):
    """Several units of one to three stages of 128 tokens per CTA: odd counts leave one of its two pipelines without tokens
    at a unit's end, single stages for the whole unit, again and again."""
    rng = np.random.default_rng(hq * N)
    lens = [int(x) for x in rng.integers(N, 385, 56)] + [128, 129, 256, 257, 384, 1, 0, 16]
    c = tree_case(lens, hq, 8, 128, 16, N, seed=N, fp8=fp8, sigma=0.7, sizes=[N if i % 3 else 1 + i % N for i in range(64)])
    first = both(c, seqs=[0, 7, 20, 41, 56, 57, 58, 59, 60, 61, 62, 63])
    ws = torch.full((spec.tree_workspace_bytes(c["shape"], c["N"]),), 255, dtype=torch.uint8, device=DEV)
    for _ in range(20):
        assert torch.equal(run_tree(c, ws=ws).view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("fp8", [None, (0.02, 0.03)], ids=["bf16", "fp8"])
@pytest.mark.parametrize("hq,N", [(16, 2), (32, 4), (16, 9), (48, 8), (48, 16), (64, 16)])
def test_tree_attention_scores_far_apart(hq, N, fp8):
    """Scores of hundreds, whose running maximum rises again and again by more than the weights' types can hold."""
    c = tree_case([N, 200, 700, 1500], hq, 8, 128, 16, N, seed=N + hq, fp8=fp8, sigma=1.0)
    for x in (c["q"],):
        x.mul_(torch.logspace(-1, 1.3, x.shape[2], device=DEV)[None, None, :, None])
    ramp = torch.linspace(0.05, 1.0, c["k"].shape[0], device=DEV)[:, None, None, None]
    if fp8:
        k = c["k"].view(E4M3).float()
        c["k"] = (k * ramp).to(E4M3).view(torch.uint8)
    else:
        c["k"] = c["k"] * ramp.to(torch.bfloat16)
    both(c)


def test_tree_attention_random_shapes():
    rng = np.random.default_rng(99)
    for i in range(24):
        D = int(rng.choice([64, 128]))
        hkv = int(rng.choice([1, 2, 4]))
        hq = hkv * int(rng.choice([1, 2, 3, 4, 5, 8, 16]))
        N = int(rng.choice([1, 2, 3, 5, 7, 8, 13, 16, 31, 48, 65, 100]))
        bs = int(rng.choice([16, 32, 64, 128, 256]))
        B = int(rng.integers(1, 6))
        lens = [int(x) for x in rng.integers(0, 700, B)]
        sizes = [int(x) for x in rng.integers(-1, N + 2, B)] if rng.random() < 0.6 else None
        fp8 = (0.02, 0.03) if D == 128 and rng.random() < 0.4 else None
        kind = str(rng.choice(["tree", "forest", "chain", "star"]))
        both(tree_case(lens, hq, hkv, D, bs, N, seed=1000 + i, sizes=sizes, fp8=fp8, kind=kind, sigma=0.7))


@pytest.mark.parametrize("fp8", [None, (0.02, 0.03)], ids=["bf16", "fp8"])
@pytest.mark.parametrize("hq,N", [(16, 2), (32, 4), (16, 9), (40, 8), (32, 12), (48, 16)])
def test_tree_attention_tiny_and_zero_queries(hq, N, fp8):
    """Rows of the smallest queries (all weights alike), zeros, and ordinary ones beside them."""
    c = tree_case([N, 130, 300, 520], hq, 8, 128, 16, N, seed=N * hq, fp8=fp8, sigma=0.7, sizes=[N, N, max(1, N - 3), N])
    c["q"][:, :, ::3] *= 2.0 ** -60
    c["q"][:, :, ::3] *= 2.0 ** -66                       # around the smallest normal number, and below it
    c["q"][:, :, 1::5] = 0.0
    c["q"][2, max(1, N - 3):] = float("nan")
    both(c)


@pytest.mark.parametrize("fp8,hq,N", [(None, 8, 2), (None, 16, 16), (None, 32, 16), ((0.02, 0.03), 8, 2), ((0.02, 0.03), 32, 8),
                                      ((0.02, 0.03), 64, 16)])
def test_pools_beyond_32_bits(fp8, hq, N):
    """Blocks at the far end of pools of more than 2^31 elements give what they give in a small pool; so do the append
    and the moves of accepted tokens there."""
    c = tree_case([N, 60, 300, 700], hq, 8, 128, 16, N, seed=hq, fp8=fp8, sigma=0.7)
    small_nb, NB = c["k"].shape[0], 140000
    assert NB * 8 * 16 * 128 > 2 ** 31
    far = dict(c, table=np.where(c["table"] >= 0, NB - small_nb + c["table"], -1), k=None, v=None)
    for name in "kv":
        far[name] = torch.empty((NB,) + tuple(c[name].shape[1:]), dtype=c[name].dtype, device=DEV)
        far[name][NB - small_nb:] = c[name]
    far["shape"] = pool_shape(4, hq, 8, 128, 16, NB, c["table"].shape[1], "head_major")
    near_out, far_out = run_tree(c), run_tree(far)
    assert torch.equal(near_out.view(torch.int16), far_out.view(torch.int16))
    # append the trees' tokens again, then keep the nodes 0, 1, 3, 4 ..
    rope = spec.Rope(128, False, torch.logspace(0, -3, 64, device=DEV))
    rows = torch.arange(4, device=DEV).repeat_interleave(N)
    at = (gpu(c["lens"]) - N)[rows] + torch.arange(N, device=DEV, dtype=I32).repeat(4)
    path = torch.full((4, N), -1, dtype=I32, device=DEV)
    kept = [0] + [i for i in range(1, N) if i != 2]
    path[:, : len(kept)] = torch.tensor(kept, dtype=I32, device=DEV)
    count = torch.full((4,), len(kept) - 1, dtype=I32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(5)
    qkv = torch.randn((4 * N, hq + 16, 128), generator=g, device=DEV).to(torch.bfloat16)
    for x in (c, far):
        table = gpu(x["table"])
        slots = (table[rows, (at // 16).long()] * 16 + at % 16).to(I32)
        args = (x["shape"], rope, qkv[:, :hq], qkv[:, hq: hq + 8], qkv[:, hq + 8:], at.to(I32), slots,
                torch.empty((4 * N, hq, 128), dtype=torch.bfloat16, device=DEV), x["k"], x["v"])
        base, lens_out = gpu(c["lens"] - N), torch.empty(4, dtype=I32, device=DEV)
        if fp8:
            spec.rope_kv_append_fp8(*args, *fp8)
            spec.kv_keep_path_fp8(x["shape"], x["k"], x["v"], table, base, path, count, lens_out)
        else:
            spec.rope_kv_append(*args)
            spec.kv_keep_path(x["shape"], x["k"], x["v"], table, base, path, count, lens_out)
    torch.cuda.synchronize()
    for name in "kv":
        assert torch.equal(far[name][NB - small_nb:].view(torch.uint8), c[name].view(torch.uint8))


# ------------------------------------------------------------------------------------------------ verification
def run_verify(p, q, tokens, parents, uniforms, sizes, stream=None):
    B, N, V = p.shape
    path, out, count = (torch.full(s, -9, dtype=I32, device=DEV) for s in ((B, N), (B, N), (B,)))
    spec.verify_drafts(p, q, gpu(tokens), None if parents is None else gpu(parents), gpu(uniforms, torch.float32), path, out,
                       count, tree_sizes=None if sizes is None else gpu(sizes), stream=stream)
    torch.cuda.synchronize()
    return path.cpu().numpy(), out.cpu().numpy(), count.cpu().numpy()


def check_verify(p, q, tokens, parents, uniforms, sizes=None):
    got = run_verify(p, q, tokens, parents, uniforms, sizes)
    P, Q = p.cpu().numpy(), None if q is None else q.cpu().numpy()
    for b in range(P.shape[0]):
        n = P.shape[1] if sizes is None else max(0, min(P.shape[1], int(sizes[b])))
        path, out, count, margin = so.verify(P[b], None if Q is None else Q[b], tokens[b], None if parents is None else parents[b],
                                             n, uniforms[b])
        assert margin > 1e-11 or P.shape[2] < 3, (b, margin)   # 64-bit sums of up to 2^20 terms are off by less
        assert np.array_equal(got[0][b], path) and np.array_equal(got[1][b], out) and got[2][b] == count, (b, n)
    return got


def verify_inputs(seed, B, N, V, kind, drawn, noise=0.5, dups=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    logits = torch.randn((B, N, V), generator=g, device=DEV) * 2
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits + noise * torch.randn((B, N, V), generator=g, device=DEV), -1)
    par = random_parents(rng, B, N, kind)
    tokens = np.zeros((B, N), np.int64)
    for b in range(B):
        for i in range(1, N):
            up = int(par[b, i]) if 0 <= par[b, i] < i else 0
            tokens[b, i] = int(torch.multinomial(q[b, up], 1, generator=g)) if not (dups and rng.random() < 0.3) else tokens[b, i - 1]
    return p, q if drawn else None, tokens, par, rng.random((B, N)).astype(np.float32)


@pytest.mark.parametrize("B,N,V", [(1, 1, 7), (1, 5, 511), (2, 4, 512), (3, 8, 513), (5, 16, 4097), (9, 64, 1000),
                                   (2, 256, 300), (4, 5, 152064), (40, 6, 32000), (130, 4, 1111), (600, 3, 600), (3, 3, 1 << 20)])
@pytest.mark.parametrize("drawn", [True, False])
def test_verify_drafts(B, N, V, drawn):
    kind = ["tree", "star", "forest"][(B + N + V) % 3]
    p, q, tokens, par, u = verify_inputs(B + N + V, B, N, V, kind, drawn, dups=N > 3)
    sizes = None if B % 2 else np.random.default_rng(B).integers(-1, N + 2, B)
    got = check_verify(p, q, tokens, par, u, sizes)
    if B >= 40 and drawn:                             # (a chosen token has p(x), about 1 / V here, to be accepted)
        assert got[2].max() > 0                       # something is accepted
    check_verify(p, q, tokens, None, u, sizes)        # the same rows as chains


@pytest.mark.parametrize("kind", ["chain", "star", "tree"])
def test_verify_chosen_drafts_of_a_sharp_target(kind):
    """The likeliest tokens are proposed, some of them twice: branches are accepted several nodes deep, siblings refused."""
    rng = np.random.default_rng(2)
    B, N, V = 50, 12, 3001
    g = torch.Generator(device=DEV).manual_seed(77)
    p = torch.softmax(torch.randn((B, N, V), generator=g, device=DEV) * 6, -1)
    par = random_parents(rng, B, N, kind)
    top = p.topk(4, -1).indices.cpu().numpy()
    tokens = np.zeros((B, N), np.int64)
    for b in range(B):
        for i in range(1, N):
            tokens[b, i] = top[b, par[b, i], rng.integers(0, 4)]
    got = check_verify(p, None, tokens, par, rng.random((B, N)).astype(np.float32))
    assert got[2].max() >= (1 if kind == "star" else 3) and got[2].min() == 0


def test_verify_strided_rows_and_odd_tokens():
    p, q, tokens, par, u = verify_inputs(21, 6, 7, 999, "tree", True)
    wide = torch.zeros((6, 9, 1200), device=DEV)
    wide[:, 1:8, 101:1100] = p
    pv = wide[:, 1:8, 101:1100]
    assert not pv.is_contiguous()
    a = run_verify(p, q, tokens, par, u, None)
    assert all(np.array_equal(x, y) for x, y in zip(a, run_verify(pv, q, tokens, par, u, None)))
    tokens[0, 1:], tokens[1, 2], tokens[2, 1] = -1, 999, 2 ** 31 - 1   # never accepted
    check_verify(p, q, tokens, par, u)
    # one row shared by all nodes and sequences
    one = p[:1, :1].expand(6, 7, 999)
    check_verify(one, None, np.clip(tokens, 0, 998), par, u)


def test_verify_degenerate_distributions():
    V, N = 700, 4
    tokens, par = np.array([[0, 5, 5, 9]] * 6), np.array([[-1, 0, 0, 0]] * 6)
    u = np.full((6, N), 0.5, np.float32)
    p = torch.zeros((6, N, V), device=DEV)
    q = torch.zeros((6, N, V), device=DEV)
    p[0, :, 5], q[0, :, 5] = 1.0, 1.0                  # certain and accepted
    p[1, :, 6], q[1, :, 5] = 1.0, 1.0                  # certain and refused
    p[2, :, 300], q[2, :, :] = 1.0, 1.0 / V
    p[3], q[3] = 0.5 / V, 1.0 / V                      # the target has less everywhere: nothing is left after a refusal
    u[3] = 0.9
    p[4, :, 699], q[4, :, 699] = 1.0, 1.0              # the last index
    p[5], q[5, :, 5] = 0.0, 1.0                        # no mass at all
    u[4, 0] = np.nextafter(np.float32(1), np.float32(0))
    check_verify(p, q, tokens, par, u)
    check_verify(p, None, tokens, par, u)
    # no path out of the vocabulary with NaN or infinity among the probabilities
    p[0, 0, 3], p[1, 0, 3], q[2, 0, 300] = float("nan"), float("inf"), float("nan")
    for dq in (q, None):
        _, out, count = run_verify(p, dq, tokens, par, u, None)
        assert out.max() < V and out.min() >= -1 and all(out[b, count[b]] >= 0 for b in range(6))


# ------------------------------------------------------------------------------------------------ keep_path
@pytest.mark.parametrize("B,N,hkv,D,bs,layout", [(1, 1, 1, 64, 16, "head_major"), (3, 5, 2, 128, 16, "head_major"),
                                                 (17, 40, 8, 128, 32, "token_major"), (6, 256, 3, 64, 16, "head_major"),
                                                 (200, 12, 1, 128, 64, "head_major")])
@pytest.mark.parametrize("fp8", [False, True])
def test_keep_path(B, N, hkv, D, bs, layout, fp8):
    if fp8 and D != 128:
        pytest.skip("the 8-bit cache has head_dim 128")
    rng = np.random.default_rng(B * N)
    base = rng.integers(0, 70, B)
    nblk = -(-(base + N) // bs)
    NB, MB = int(nblk.sum()) + 2, int(nblk.max())
    perm, at = rng.permutation(NB), 0
    table = np.full((B, MB), -1)
    for b in range(B):
        table[b, : nblk[b]] = perm[at: at + nblk[b]]
        at += nblk[b]
    path = np.full((B, N), -1)
    acc = np.zeros(B, np.int64)
    for b in range(B):
        picks = np.concatenate([[0], 1 + np.flatnonzero(rng.random(N - 1) < rng.choice([0.2, 0.7, 1.0]))]) if b != 2 else np.array([], int)
        path[b, : len(picks)] = picks
        acc[b] = max(0, len(picks) - 1)
    if B > 5:
        path[3, 1] = 0                # does not increase: ends there
        acc[4] = N + 5                # clamped (the path ends at its -1)
        acc[5] = -2
        table[6 % B, 0] = NB          # a block outside the pool: its moves are skipped
    g = torch.Generator(device=DEV).manual_seed(1)
    caches = [torch.randint(0, 255, (NB, hkv, bs, D * (1 if fp8 else 2)), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    caches = [(c if layout == "head_major" else c.transpose(1, 2).contiguous()) for c in caches]
    want = [as_head_major(c, layout).cpu().numpy().copy() for c in caches]
    sh = pool_shape(B, hkv, hkv, D, bs, NB, MB, layout)
    ctx = torch.full((B,), -1, dtype=I32, device=DEV)
    views = caches if fp8 else [c.view(torch.bfloat16) for c in caches]
    (spec.kv_keep_path_fp8 if fp8 else spec.kv_keep_path)(sh, *views, gpu(table), gpu(base), gpu(path), gpu(acc), ctx)
    new = [so.keep_path(w, table, base, path, acc, bs) for w in want][0]
    assert np.array_equal(ctx.cpu().numpy(), new)
    for c, w in zip(caches, want):
        assert np.array_equal(as_head_major(c, layout).cpu().numpy(), w)


# ------------------------------------------------------------------------------------------------ together
class Loop:
    """A small serving loop: three requests, draft trees of up to 6 nodes, one layer, everything on the device."""

    def __init__(self, seed=0, steps=4):
        self.B, self.N, self.hq, self.hkv, self.D, self.bs, self.V, self.MB = 3, 6, 8, 2, 128, 16, 257, 6
        self.NB = 24
        B, N = self.B, self.N
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        self.shape = pool_shape(B, self.hq, self.hkv, self.D, self.bs, self.NB, self.MB)
        z = lambda *s: torch.zeros(s, dtype=I32, device=DEV)  # noqa: E731
        self.ctx, self.held, self.head, self.table = z(B), z(B), z(1), torch.full((B, self.MB), -1, dtype=I32, device=DEV)
        self.free = gpu(self.rng.permutation(self.NB))
        self.slot, self.pos, self.first, self.granted, self.total = z(B * N), z(B * N), z(B + 1), z(B), z(B)
        self.path, self.tokens, self.count, self.next_ctx, self.status = z(B, N), z(B, N), z(B), z(B), z(1)
        self.kc, self.vc = (torch.full((self.NB, self.hkv, self.bs, self.D), float("nan"), dtype=torch.bfloat16, device=DEV)
                            for _ in range(2))
        inv, _ = spec.rope_frequencies(128, 10000.0)
        self.rope = spec.Rope(128, False, inv.to(DEV))
        self.ws = torch.empty(spec.tree_workspace_bytes(self.shape, N), dtype=torch.uint8, device=DEV)
        self.ws_plan = torch.empty(spec.plan_slots_workspace_bytes(self.shape), dtype=torch.uint8, device=DEV)
        self.qkv = torch.zeros((B * N, (self.hq + 2 * self.hkv) * self.D), dtype=torch.bfloat16, device=DEV)
        self.q_rot = torch.zeros((B * N, self.hq, self.D), dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros((B, N, self.hq, self.D), dtype=torch.bfloat16, device=DEV)
        self.p, self.qd = (torch.zeros((B, N, self.V), device=DEV) for _ in range(2))
        self.par, self.drafts, self.sizes, self.u = z(B, N), z(B, N), z(B), torch.zeros((B, N), device=DEV)

    def feed(self, sizes=None):
        """New inputs for a step, in the same buffers."""
        B, N = self.B, self.N
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=self.g, device=DEV) * 0.7)
        self.par.copy_(gpu(random_parents(self.rng, B, N)))
        self.sizes.copy_(gpu(self.rng.integers(1, N + 1, B) if sizes is None else sizes))
        lg = torch.randn((B, N, self.V), generator=self.g, device=DEV)
        self.p.copy_(torch.softmax(lg, -1))
        self.qd.copy_(torch.softmax(lg + 0.2 * torch.randn(lg.shape, generator=self.g, device=DEV), -1))
        rows = self.qd[torch.arange(B, device=DEV)[:, None], self.par.clamp(min=0).long()].view(B * N, -1)
        self.drafts.copy_(torch.multinomial(rows, 1, generator=self.g).view(B, N).int())
        self.u.copy_(torch.rand((B, N), generator=self.g, device=DEV))

    def step(self, stream=None):
        hq, hkv, D = self.hq, self.hkv, self.D
        spec.plan_slots(self.shape, self.ctx, self.sizes, self.table, self.held, self.free, self.head, self.slot, self.pos,
                        self.first, self.granted, self.total, self.ws_plan, row_len=self.N, parents=self.par, status=self.status,
                        stream=stream)
        q, k, v = (self.qkv[:, a * D: b * D].unflatten(1, (b - a, D)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
        spec.rope_kv_append(self.shape, self.rope, q, k, v, self.pos, self.slot, self.q_rot, self.kc, self.vc, stream=stream)
        spec.tree_attention(self.shape, self.q_rot.view(self.out.shape), self.kc, self.vc, self.table, self.total, self.par, 0.09,
                            self.out, self.ws, tree_sizes=self.granted, stream=stream)
        spec.verify_drafts(self.p, self.qd, self.drafts, self.par, self.u, self.path, self.tokens, self.count,
                           tree_sizes=self.granted, stream=stream)
        spec.kv_keep_path(self.shape, self.kc, self.vc, self.table, self.ctx, self.path, self.count, self.next_ctx, stream=stream)

    def commit(self):
        self.ctx.copy_(self.next_ctx)

    def state(self):
        return [t.clone() for t in (self.slot, self.pos, self.table, self.held, self.head, self.total, self.out, self.path,
                                    self.tokens, self.count, self.next_ctx, self.kc, self.vc)]


def test_steps_together():
    """Several steps in a row against a shadow that keeps every sequence's keys and values in a plain list."""
    lp = Loop(seed=3)
    hq, hkv, D, N = lp.hq, lp.hkv, lp.D, lp.N
    inv = lp.rope.inv_freq.cpu().numpy()
    shadow = [([], []) for _ in range(lp.B)]
    kept = 0
    for step in range(5):
        lp.feed()
        lp.step()
        torch.cuda.synchronize()
        assert int(lp.status) == 0 and binding.workspace_status(lp.ws) == 0
        qkv = lp.qkv.cpu().double().numpy().reshape(lp.B, N, -1, D)
        par, sizes = lp.par.cpu().numpy(), lp.sizes.cpu().numpy()
        table, out = lp.table.cpu().numpy(), lp.out.cpu().double().numpy()
        for b in range(lp.B):
            n, base = int(sizes[b]), len(shadow[b][0])
            depth = [len(so.sees(par[b], i)) - 1 for i in range(n)]
            turned = so.rope(qkv[b, :n, : hq + hkv], [base + d for d in depth], inv, 128, False, 1.0)
            # what the operators store and read is rounded to bf16 (exactly the fp64 value's neighbour but for ties)
            as16 = lambda x: torch.as_tensor(x).to(torch.bfloat16).double().numpy()  # noqa: E731
            qr, kr, vr = as16(turned[:, :hq]), as16(turned[:, hq:]), qkv[b, :n, hq + hkv:]
            for h in range(hkv):
                k = np.array([r[h] for r in shadow[b][0]] + [kr[i, h] for i in range(n)])
                v = np.array([r[h] for r in shadow[b][1]] + [vr[i, h] for i in range(n)])
                G = hq // hkv
                want, mag, spread = so.tree_attention(qr[:, h * G:(h + 1) * G], k, v, par[b], n, 0.09)
                # bf16 weights and output, and q, k that may lie one bf16 step (2^-7) away where fp32 and fp64 round apart
                tol = (2.0 ** -7 + 2.0 ** -8 + 2 * 2.0 ** -7 * spread[..., None]) * mag + 1e-6
                assert np.all(np.abs(out[b, :n, h * G:(h + 1) * G] - want) <= tol)
            path, toks, count, _ = so.verify(lp.p[b].cpu().numpy(), lp.qd[b].cpu().numpy(), lp.drafts[b].cpu().numpy(), par[b], n,
                                             lp.u[b].cpu().numpy())
            assert np.array_equal(lp.path[b].cpu().numpy(), path) and np.array_equal(lp.tokens[b].cpu().numpy(), toks)
            for i in path[: count + 1]:
                shadow[b][0].append(kr[i])
                shadow[b][1].append(vr[i])
            kept += count
            assert int(lp.next_ctx[b]) == len(shadow[b][0])
            # the cache holds the kept tokens, in order
            T = len(shadow[b][0])
            ids = torch.as_tensor(table[b, : -(-T // lp.bs)], device=DEV).long()
            kk, vv = (c[ids].permute(0, 2, 1, 3).flatten(0, 1)[:T].cpu().double().numpy() for c in (lp.kc, lp.vc))
            assert np.array_equal(vv, np.array(shadow[b][1]))
            assert np.all(np.abs(kk - np.array(shadow[b][0])) <= 2.0 ** -7 * np.abs(kk) + 1e-6)
        lp.commit()
    assert kept > 5


def test_step_captured_and_replayed():
    """One captured step, replayed with other inputs in the same buffers, gives what eager steps give."""
    lp, ref = Loop(seed=8), Loop(seed=8)
    side = torch.cuda.Stream()
    lp.feed()
    ref.feed()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lp.step()                                        # warm-up; in place, so bring the state back
    torch.cuda.current_stream().wait_stream(side)
    lp.held.zero_(), lp.head.zero_(), lp.table.fill_(-1), lp.kc.fill_(float("nan")), lp.vc.fill_(float("nan")), lp.out.zero_()
    lp.q_rot.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lp.step()
    for i in range(4):
        graph.replay()
        ref.step()
        torch.cuda.synchronize()
        for a, b in zip(lp.state(), ref.state()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
        for x in (lp, ref):
            x.commit()
            x.feed()


def test_calls_on_two_streams():
    """Calls that overlap on two streams, with buffers of their own, give what they give alone."""
    loops = [Loop(seed=20 + i) for i in range(2)]
    alone = [Loop(seed=20 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for lp in loops + alone:
        lp.feed()
    torch.cuda.synchronize()
    for lp in alone:
        lp.step()
    torch.cuda.synchronize()
    for lp, st in zip(loops, streams):
        lp.step(stream=st)
    torch.cuda.synchronize()
    for a, b in zip(loops, alone):
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
