"""Pools whose tokens, heads and blocks lie apart: the operators of a speculative step give what they give in a dense pool,
and leave the gaps alone (GPU)."""
import numpy as np
import pytest
import torch

from paper_2511_21862_b200 import binding, build, spec

import test_gpu_spec as base

pytestmark = pytest.mark.gpu
FP8 = (0.02, 0.03)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def spread(c, gap):
    """The case's pools with `gap` elements behind every token, head and block; (case, views as [NB, Hkv, bs, D])."""
    NB, hkv, bs, D = c["k"].shape
    ts, hs = D + gap, bs * (D + gap) + gap
    bst = hkv * hs + gap
    wide, views = {}, {}
    for name in "kv":
        flat = torch.full((NB * bst,), 0x7f if c["fp8"] else 77, dtype=c[name].dtype, device="cuda")
        views[name] = flat.as_strided((NB, hkv, bs, D), (bst, hs, ts, 1))
        views[name].copy_(c[name])
        wide[name] = flat
    sh = c["shape"]
    shape = binding.Shape(sh.batch, sh.num_q_heads, hkv, D, bs, NB, sh.max_blocks_per_seq, bst, hs, ts)
    return dict(c, shape=shape, **wide), views


@pytest.mark.parametrize("hq,D,N,fp8", [(16, 128, 2, None), (16, 128, 2, FP8), (32, 128, 4, None), (32, 128, 4, FP8),
                                        (40, 128, 8, None), (40, 128, 8, FP8), (32, 128, 16, None), (32, 128, 24, None),
                                        (32, 128, 24, FP8), (32, 128, 40, None), (32, 128, 40, FP8), (16, 64, 2, None),
                                        (32, 64, 4, None), (32, 64, 20, None)])
@pytest.mark.parametrize("gap", [16, 48])
def test_a_step_in_a_pool_with_gaps(hq, D, N, fp8, gap):
    hkv, bs = 8, 16
    c = base.tree_case([N, 60, 300, 700, 2500], hq, hkv, D, bs, N, seed=hq + N, fp8=fp8, sigma=0.7)
    wide, views = spread(c, gap)
    assert torch.equal(base.run_tree(c).view(torch.int16), base.run_tree(wide).view(torch.int16))
    # append the nodes' rows again, then keep the nodes 0, 1, 3, 4 ..
    B = len(c["lens"])
    rope = spec.Rope(D, False, torch.logspace(0, -3, D // 2, device="cuda"))
    rows = torch.arange(B, device="cuda").repeat_interleave(N)
    at = (base.gpu(c["lens"]) - N)[rows] + torch.arange(N, device="cuda", dtype=torch.int32).repeat(B)
    table = base.gpu(c["table"])
    slots = (table[rows, (at // bs).long()] * bs + at % bs).to(torch.int32)
    kept = [0] + [i for i in range(1, N) if i != 2]
    path = torch.full((B, N), -1, dtype=torch.int32, device="cuda")
    path[:, : len(kept)] = torch.tensor(kept, dtype=torch.int32, device="cuda")
    count = torch.full((B,), len(kept) - 1, dtype=torch.int32, device="cuda")
    qkv = torch.randn((B * N, hq + 2 * hkv, D), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(torch.bfloat16)
    for x in (c, wide):
        args = (x["shape"], rope, qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:], at.to(torch.int32), slots,
                torch.empty((B * N, hq, D), dtype=torch.bfloat16, device="cuda"), x["k"], x["v"])
        lens = torch.empty(B, dtype=torch.int32, device="cuda")
        if fp8:
            spec.rope_kv_append_fp8(*args, *fp8)
            spec.kv_keep_path_fp8(x["shape"], x["k"], x["v"], table, base.gpu(c["lens"] - N), path, count, lens)
        else:
            spec.rope_kv_append(*args)
            spec.kv_keep_path(x["shape"], x["k"], x["v"], table, base.gpu(c["lens"] - N), path, count, lens)
        assert np.array_equal(lens.cpu().numpy(), c["lens"] - N + len(kept))
    for name in "kv":
        assert torch.equal(views[name].contiguous().view(torch.uint8), c[name].view(torch.uint8))
        gaps = torch.ones(wide[name].numel(), dtype=torch.bool, device="cuda")
        gaps.as_strided(views[name].shape, views[name].stride()).fill_(False)
        assert bool((wide[name][gaps] == (0x7f if fp8 else 77)).all())
