"""The continuous-batching operators on the GPU where a call leaves the usual: thousands of sequences, captured graphs, side streams,
large offsets, the checked build."""
import numpy as np
import pytest
import torch

import test_gpu_batch as t
from oracle import batch_oracle as bo
from paper_2511_21862_b200 import batch, binding, build, spec

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = torch.int32
gpu, host, pool_shape = t.gpu, t.host, t.pool_shape


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


@pytest.mark.parametrize("B,most,D,fp8", [(3000, 3, 64, False), (1500, 1, 128, False), (2000, 2, 128, True)])
def test_chunk_of_thousands_of_sequences(B, most, D, fp8):
    """More sequences and tiles than the plan keeps in registers and shared memory."""
    rng = np.random.default_rng(B)
    t.run_chunk(rng.integers(0, most + 1, B).tolist(), rng.integers(0, 40, B).tolist(), hq=2, hkv=1, D=D, fp8=fp8, bs=16, seed=B)


def test_chunk_of_many_tiles():
    """One prompt of more tiles than there are threads, behind a decode and before a short piece."""
    n, hq, hkv, D, bs = 9000, 16, 1, 64, 64
    ctx, new = [100, n, 50], [1, n, 30]
    out, _, _, _ = t.run_chunk(new, ctx, hq=hq, hkv=hkv, D=D, bs=bs, seed=1, check=False)
    again, _, _, _ = t.run_chunk(new, ctx, hq=hq, hkv=hkv, D=D, bs=bs, seed=1, check=False)
    assert torch.equal(out, again) and not out[: n + 31].isnan().any()
    # the whole prompt against plain attention in 64 bits on the GPU (the pool is rebuilt from the same seed)
    g = torch.Generator(device=DEV).manual_seed(1)
    held = [-(-c // bs) for c in ctx]
    NB = sum(held) + 7
    perm = np.random.default_rng(1).permutation(NB)
    k, v = (torch.randn((NB, hkv, bs, D), generator=g, device=DEV).to(torch.bfloat16).double() for _ in range(2))
    q = torch.randn((sum(new) + 3, hq, D), generator=g, device=DEV).to(torch.bfloat16).double()
    ids = torch.as_tensor(perm[held[0]: held[0] + held[1]], device=DEV)
    k, v = k[ids, 0].flatten(0, 1)[:n], v[ids, 0].flatten(0, 1)[:n]
    for lo in range(0, n, 1500):
        s = torch.einsum("nhd,td->hnt", q[1 + lo: 1 + lo + 1500], k) / D ** 0.5
        seen = torch.arange(n, device=DEV) <= torch.arange(lo, lo + s.shape[1], device=DEV)[:, None]
        w = torch.softmax(s.masked_fill(~seen, -torch.inf), -1)
        want, mag = torch.einsum("hnt,td->nhd", w, v), torch.einsum("hnt,td->nhd", w, v.abs())
        # weights and output rounded to bf16 (2^-8 each); scores of 64 dims, sums and exponentials: 2^-10 covers them here
        assert ((out[1 + lo: 1 + lo + 1500].double() - want).abs() <= (2 * 2.0 ** -8 + 2.0 ** -10) * mag).all()


def test_chunk_in_a_pool_beyond_32_bit_offsets():
    """Blocks at the end of a pool of more than 2^31 elements."""
    hq, hkv, D, bs, NB, MB = 8, 8, 128, 256, 8300, 3
    kc = torch.zeros((NB, hkv, bs, D), dtype=torch.bfloat16, device=DEV)
    vc = torch.zeros_like(kc)
    assert kc.numel() > 2 ** 31
    table = gpu([[NB - 1, NB - 3, NB - 2], [NB - 4, 0, 1]])
    for x in (kc, vc):
        x[NB - 4:].normal_(generator=torch.Generator(device=DEV).manual_seed(2))
    sh = pool_shape(2, hq, hkv, D, bs, NB, MB)
    q = torch.randn((41, hq, D), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).to(torch.bfloat16)
    out = torch.empty_like(q)
    ws = torch.empty(batch.chunk_workspace_bytes(sh, 41, 40), dtype=torch.uint8, device=DEV)
    batch.chunk_attention(sh, q, kc, vc, table, gpu([700, 200]), gpu([0, 40, 41]), 40, 0.1, out, ws)
    for b, (r0, n, T) in enumerate(((0, 40, 700), (40, 1, 200))):
        ids = table[b, : -(-T // bs)].long()
        k, v = (host(x[ids].transpose(1, 2).flatten(0, 1)[:T]) for x in (kc, vc))
        want, mag, spr = bo.chunk_attention(host(q[r0: r0 + n]), k, v, n, 0.1)
        tol = t.tolerance(host(q[r0: r0 + n]), k.reshape(T, -1), v, mag, spr, 0.1, False)
        assert (np.abs(host(out[r0: r0 + n]) - want) <= tol).all()


def test_page_operators_in_place_over_many_entries():
    """In place, on all SMs: a launch per phase must not read what a later one has updated."""
    rng = np.random.default_rng(21)
    for seed in range(3):
        ctx, held, table, free, head, shares, NB = t.shared_state(rng, 300, 16, 9000, 11)
        t.run_release(rng.permutation(300)[:290], None, ctx, table, held, free, head, shares, bs=16, NB=NB, in_place=True)
    ctx, held, table, free, NB = t.random_pool(rng, 400, 16, 9000, 400, extra_rows=300)
    t.run_fork(rng.integers(0, 100, 300), 100 + rng.permutation(300), None, ctx, table, held, free, 1, np.zeros(NB, np.int64), bs=16,
               NB=NB, in_place=True)


def test_page_operators_beyond_the_list_in_shared_memory():
    rng = np.random.default_rng(22)
    ctx, held, table, free, head, shares, NB = t.shared_state(rng, 6000, 16, 60, 5)
    t.run_release(rng.permutation(6000)[:5000], rng.integers(0, 60, 5000), ctx, table, held, free, head, shares, bs=16, NB=NB)
    ctx, held, table, free, NB = t.random_pool(rng, 6000, 16, 60, 4000, extra_rows=5000)
    t.run_fork(rng.integers(0, 1000, 5000), 1000 + rng.permutation(5000), rng.integers(0, 60, 5000), ctx, table, held, free, 0,
               np.zeros(NB, np.int64), bs=16, NB=NB)


def step(sh, s):
    """Everything of a step, on the current stream; out of place, so it can run again."""
    batch.fork_pages(sh, s["parents"], s["children"], s["ctx"], s["table"], s["held"], s["free"], s["head"], s["shares"], s["src"],
                     s["dst"], s["granted"], s["pages"], context_lens_out=s["ctx2"], blocks_held_out=s["held2"],
                     free_head_out=s["head2"], shares_out=s["shares2"])
    binding.kv_copy_blocks(sh, s["kc"], s["vc"], s["src"], s["dst"])
    batch.norm_rope_kv_append(sh, s["rope"], s["norm"], s["qkv"][:, :8], s["qkv"][:, 8:10], s["qkv"][:, 10:], s["pos"], s["slot"],
                              s["q"], s["kc"], s["vc"])
    batch.chunk_attention(sh, s["q"], s["kc"], s["vc"], s["table"], s["lens"], s["first"], 20, 0.1, s["out"], s["ws"])
    batch.shape_logits(s["logits"], probs=s["probs"], repetition=s["rep"], history=s["history"], history_lens=s["hlens"],
                       temperature=s["temp"])
    batch.release_pages(sh, s["children"], s["ctx2"], s["table"], s["held2"], s["free2"], s["head2"], s["shares2"], s["pages2"],
                        context_lens_out=s["ctx3"], blocks_held_out=s["held3"], free_head_out=s["head3"], shares_out=s["shares3"])


def step_state(seed):
    B, D, bs, MB, NB = 4, 128, 16, 8, 40
    g = torch.Generator(device=DEV).manual_seed(seed)
    sh = pool_shape(B, 8, 2, D, bs, NB, MB)
    table = np.full((B, MB), -1)
    table[0, :6], table[1, :4], table[2, :5] = range(6), range(6, 10), range(10, 15)
    i32 = lambda *n: torch.zeros(n, dtype=I32, device=DEV)  # noqa: E731
    s = dict(parents=gpu([0]), children=gpu([3]), ctx=gpu([70, 50, 75, 0]), table=gpu(table), held=gpu([6, 4, 5, 0]),
             free=gpu(np.arange(15, NB)), head=gpu([0]), shares=i32(NB), src=i32(1), dst=i32(1), granted=i32(1), ctx2=i32(B),
             held2=i32(B), head2=i32(1), shares2=i32(NB), ctx3=i32(B), held3=i32(B), head3=i32(1), shares3=i32(NB),
             free2=gpu(np.arange(15, NB)), kc=torch.randn((NB, 2, bs, D), generator=g, device=DEV).to(torch.bfloat16),
             vc=torch.randn((NB, 2, bs, D), generator=g, device=DEV).to(torch.bfloat16),
             qkv=torch.randn((22, 12, D), generator=g, device=DEV).to(torch.bfloat16), pos=gpu([70, 50] + list(range(55, 75))),
             slot=gpu([5 * 16, 9 * 16 + 2] + [(10 + p // 16) * 16 + p % 16 for p in range(55, 75)]),
             q=torch.empty((22, 8, D), dtype=torch.bfloat16, device=DEV), out=torch.zeros((22, 8, D), dtype=torch.bfloat16, device=DEV),
             lens=gpu([71, 51, 75, 0]), first=gpu([0, 1, 2, 22, 22]), logits=torch.randn((3, 5000), generator=g, device=DEV),
             probs=torch.zeros((3, 5000), device=DEV), rep=torch.full((3,), 1.2, device=DEV),
             history=torch.randint(0, 5000, (3, 64), generator=g, device=DEV, dtype=I32), hlens=gpu([64, 3, 0]),
             temp=torch.tensor([1.0, 0.0, 0.7], device=DEV), norm=batch.HeadNorm(1e-6),
             rope=spec.Rope(D, False, spec.rope_frequencies(D)[0].to(DEV)))
    s["pages"], s["pages2"] = (torch.empty(batch.pages_workspace_bytes(sh, 1), dtype=torch.uint8, device=DEV) for _ in range(2))
    s["ws"] = torch.empty(batch.chunk_workspace_bytes(sh, 22, 20), dtype=torch.uint8, device=DEV)
    return sh, s


RESULTS = ("out", "probs", "shares3", "head3", "free2", "ctx3", "held3", "kc", "vc", "q")


def test_a_step_captured_replayed_and_on_a_side_stream():
    sh, s = step_state(5)
    step(sh, s)
    torch.cuda.synchronize()
    want = {k: s[k].clone() for k in RESULTS}
    assert int(s["granted"]) == 1 and int(s["head3"]) == 0
    sh, r = step_state(5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(sh, r)
    side.synchronize()
    for k in RESULTS:
        assert torch.equal(r[k], want[k]), k
    sh, c = step_state(5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sh, c)
    for _ in range(3):
        c["out"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in RESULTS:
            assert torch.equal(c[k], want[k]), k


def test_two_chunk_calls_at_once_with_workspaces_of_their_own():
    runs = []
    for seed, new, ctx in ((1, [1, 300, 1], [900, 400, 50]), (2, [7, 1, 64], [2000, 30, 64])):
        first, call, ws, out = t.run_chunk(new, ctx, seed=seed)
        runs.append((first, call, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for _, call, _, stream in runs:
            with torch.cuda.stream(stream):
                call()
    torch.cuda.synchronize()
    for first, _, out, _ in runs:
        assert torch.equal(first, out)


def test_checked_build_agrees():
    build.build(checked=True)
    rooms = (0, 8192)   # one launch, and with a plan
    plain = [t.run_chunk([1, 40, 0, 200, 3], [900, 300, 7, 200, 64], seed=8, room=room)[0] for room in rooms]
    old = binding.use_library(build.LIB_CHECKED)
    try:
        for want, room in zip(plain, rooms):
            assert torch.equal(want, t.run_chunk([1, 40, 0, 200, 3], [900, 300, 7, 200, 64], seed=8, room=room)[0])
        t.run_chunk([1, 9, 1], [700, 80, 3000], fp8=True, seed=9)
        # a table entry outside the pool reads as zeros and is reported
        kc, vc = (torch.ones((5, 4, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        q, out = torch.ones((20, 4, 128), dtype=torch.bfloat16, device=DEV), torch.empty((20, 4, 128), dtype=torch.bfloat16, device=DEV)
        for width in (2, 512):
            sh = pool_shape(1, 4, 4, 128, 16, 5, width)
            ws = torch.empty(batch.chunk_workspace_bytes(sh, 20, 20), dtype=torch.uint8, device=DEV)
            batch.chunk_attention(sh, q, kc, vc, gpu([[99, 1] + [0] * (width - 2)]), gpu([20]), gpu([0, 20]), 20, 0.1, out, ws)
            assert binding.workspace_status(ws) & 8 and not out[:16].any()
    finally:
        binding.use_library(old if old != build.LIB_CHECKED else None)


def test_first_rows_that_overlap_or_run_over_are_harmless():
    """Rows outside the tensor do not exist, counts below zero are zero, and rows that several sequences claim stay inside it."""
    hq, hkv, D, bs = 4, 2, 128, 16
    kc, vc = (torch.randn((8, hkv, bs, D), device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((12, hq, D), device=DEV).to(torch.bfloat16)
    firsts = [-5, 3, 1, 9, 12], [0, 100, 2, 2 ** 31 - 1, 5], [0, 12, 0, 12, 0], [11, 12, 13, 14, 15], [5, 4, 3, 2, 1]
    for first, width in [(f, w) for f in firsts for w in (2, 512)]:
        sh, table = pool_shape(4, hq, hkv, D, bs, 8, width), gpu(np.pad(np.arange(8).reshape(4, 2), ((0, 0), (0, width - 2))))
        wide = torch.full((14, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(batch.chunk_workspace_bytes(sh, 12, 12), dtype=torch.uint8, device=DEV)
        batch.chunk_attention(sh, q, kc, vc, table, gpu([20, 32, 9, 1]), gpu(first), 12, 0.1, wide[1:13], ws)
        torch.cuda.synchronize()
        assert (wide[0] == 7).all() and (wide[13] == 7).all()


def test_logits_of_a_new_size_are_captured():
    """The first call of a size is the captured one; its replays read new logits."""
    x = torch.randn((50, 6, 70001), device=DEV)
    p = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        batch.shape_logits(x, probs=p, presence=torch.ones(50, device=DEV), history=torch.zeros((50, 4), dtype=torch.int32, device=DEV),
                           history_lens=torch.full((50,), 4, dtype=torch.int32, device=DEV))
    for _ in range(2):
        x.normal_()
        g.replay()
        want = x.double()
        want[..., 0] -= 1
        # exponents of up to 12 nats, two roundings of 2^-24 * 12 and the penalised logit's; exp, sum, quotient 2^-19
        assert torch.allclose(p.double(), torch.softmax(want, -1), rtol=1e-5, atol=0)
