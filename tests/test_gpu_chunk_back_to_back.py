"""Packed chunk attention, one call behind another in one workspace without a synchronisation: the kernels of a call that set out before
the one in front of them has ended must see this call's plan, not what an earlier call left in the workspace."""
import numpy as np
import pytest
import torch

import test_gpu_batch as t
from paper_2511_21862_b200 import batch, binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


@pytest.mark.parametrize("hq,hkv,D,fp8", [(32, 8, 128, False), (16, 1, 128, False), (8, 2, 64, False), (40, 8, 128, True)])
def test_calls_in_one_workspace(hq, hkv, D, fp8):
    rng = np.random.default_rng(hq + D)
    B, bs, MB, calls = 24, 16, 256, 60
    NB = 2000
    g = torch.Generator(device=DEV).manual_seed(1)
    kc, vc = (torch.randn((NB, hkv, bs, D), generator=g, device=DEV) for _ in range(2))
    kc, vc = ((x.to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else x.to(torch.bfloat16)) for x in (kc, vc))
    sh = t.pool_shape(B, hq, hkv, D, bs, NB, MB)
    rows, most = 1500, 400
    q = torch.randn((rows, hq, D), generator=g, device=DEV).to(torch.bfloat16)
    ws, ws2 = (torch.empty(batch.chunk_workspace_bytes(sh, rows, most), dtype=torch.uint8, device=DEV) for _ in range(2))
    table = torch.randint(0, NB, (B, MB), generator=g, device=DEV, dtype=torch.int32)
    steps = []
    for i in range(calls):   # few and many decodes, short pieces and long ones, rows without a context, in turn
        new = np.ones(B, np.int64)
        pieces = rng.integers(0, 5)
        new[rng.permutation(B)[:pieces]] = rng.integers(2, (20, 200, 400)[i % 3], pieces)
        new[rng.random(B) < (0.0, 0.5)[i % 2]] = 0
        while new.sum() > rows:
            new[new.argmax()] = 1
        ctx = np.where(rng.random(B) < 0.1, 0, rng.integers(1, (300, MB * bs)[i % 2], B))
        steps.append((t.gpu(ctx), t.gpu(np.concatenate([[0], np.cumsum(new)]))))
    outs, again = ([torch.zeros_like(q) for _ in range(calls)] for _ in range(2))

    def call(ctx, first, out, workspace):
        args = (sh, q, kc, vc, table, ctx, first, most, 0.1)
        if fp8:
            batch.chunk_attention_fp8(*args, 1.0, 1.0, out, workspace)
        else:
            batch.chunk_attention(*args, out, workspace)

    torch.cuda.synchronize()
    for (ctx, first), out in zip(steps, outs):
        call(ctx, first, out, ws)
    torch.cuda.synchronize()
    for (ctx, first), out in zip(steps, again):   # alone, in a workspace that is cleared before each
        ws2.zero_()
        torch.cuda.synchronize()
        call(ctx, first, out, ws2)
        torch.cuda.synchronize()
        assert binding.workspace_status(ws2) == 0
    for i in range(calls):
        assert torch.equal(outs[i], again[i]), i
