"""Packed chunk attention over the 8-bit cache with queries far outside the range of f16, in which its products are formed."""
import math

import numpy as np
import pytest
import torch

import test_gpu_batch as t
from oracle import batch_oracle as bo
from paper_2511_21862_b200 import batch, binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def run(new, ctx, base, *, hq, hkv, room, seed, odd=1.0):
    """Queries of magnitudes around `base` that differ from row to row and head to head, scores of ordinary size; one row in 20 is
    `odd` times as large."""
    rng = np.random.default_rng(seed)
    D, bs, B = 128, 16, len(new)
    held = [-(-c // bs) for c in ctx]
    MB, NB = max(max(held), room // bs), sum(held)
    table, at, perm = np.zeros((B, MB), np.int64), 0, rng.permutation(NB)
    for b in range(B):
        table[b, : held[b]] = perm[at: at + held[b]]
        at += held[b]
    g = torch.Generator(device=DEV).manual_seed(seed)
    kc, vc = ((torch.randn((NB, hkv, bs, D), generator=g, device=DEV) * 16).to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs, scale = 0.07, 0.11, 1 / (base * math.sqrt(D))
    first = np.concatenate([[0], np.cumsum(new)])
    rows = int(first[-1])
    size = base * 2.0 ** rng.integers(-7, 2, (rows, hq, 1))
    size[rng.random((rows, hq, 1)) < 0.05] = 0.0                       # rows of zeros among them
    size[rng.random((rows, hq, 1)) < 0.05] *= odd
    q = torch.as_tensor(rng.standard_normal((rows, hq, D)) * size).to(torch.bfloat16).to(DEV)
    out = torch.full_like(q, 5.0)
    sh = t.pool_shape(B, hq, hkv, D, bs, NB, MB)
    ws = torch.empty(batch.chunk_workspace_bytes(sh, rows, max(new)), dtype=torch.uint8, device=DEV)
    batch.chunk_attention_fp8(sh, q, kc.view(torch.uint8), vc.view(torch.uint8), t.gpu(table), t.gpu(ctx), t.gpu(first), max(new), scale,
                              ks, vs, out, ws)
    assert binding.workspace_status(ws) == 0
    got, qh, scale = t.host(out), t.host(q), float(np.float32(scale))
    for b in range(B):
        r0, n, T = int(first[b]), new[b], ctx[b]
        ids = torch.as_tensor(table[b, : held[b]], device=DEV)
        k, v = ((x[ids].transpose(1, 2).flatten(0, 1)[:T].double() * s).cpu().numpy() for x, s in ((kc, ks), (vc, vs)))
        want, mag, spread = bo.chunk_attention(qh[r0: r0 + n], k, v, n, scale)
        # As t.tolerance() over the 8-bit cache, but for the query's rounding: 2^-11 of a value, or 2^-40 of the largest of the rows.
        rows_of = np.abs(qh[r0: r0 + n]).reshape(n, hkv, -1).max((0, 2)).repeat(hq // hkv)
        q_err = 2.0 ** -11 * np.abs(qh[r0: r0 + n]).max(-1) + 2.0 ** -40 * rows_of
        k_sum = np.abs(k).sum(-1).max(0).repeat(hq // hkv)
        score = 2.0 ** -15.8 * spread + q_err * k_sum * scale
        score = np.minimum(score, 300.0)                                 # (rows with scores beyond that are only finite)
        rel = (1 + 2.0 ** -11) * (1 + 2.0 ** -8) - 1 + 2.0 ** -12 + np.expm1(2 * score)
        tol = rel[..., None] * mag + 2.0 ** -25 * T * np.abs(v).max()
        err = np.abs(got[r0: r0 + n] - want)
        assert (err <= tol).all(), (b, float((err / tol).max()))         # (a NaN fails, too)


@pytest.mark.parametrize("base", [1e5, 1e7, 1e30, 1.0, 1e-5, 1e-8, 1e-30])
def test_magnitudes(base):
    for room in (0, 8192):
        run([5, 1, 20, 2], [60, 200, 20, 333], base, hq=8, hkv=2, room=room, seed=1)


@pytest.mark.parametrize("base", [3e5, 2e-6])
def test_units_one_after_another(base):
    """Several (sequence, head) pairs a CTA, so that the next one's queries are loaded beside the last one's end; long and short ones."""
    rng = np.random.default_rng(5)
    run(rng.integers(2, 9, 36).tolist(), rng.integers(10, 120, 36).tolist(), base, hq=8, hkv=8, room=0, seed=2)
    run(rng.integers(2, 9, 70).tolist(), rng.integers(10, 400, 70).tolist(), base, hq=8, hkv=8, room=8192, seed=3)
    run([40, 3], [5000, 900], base, hq=16, hkv=1, room=8192, seed=4)


@pytest.mark.parametrize("base,odd", [(1.0, 2.0 ** 24), (1e-4, 2.0 ** 24), (1e8, 2.0 ** 20), (1e3, 2.0 ** -12)])
def test_rows_of_very_different_size(base, odd):
    """Small rows beside large ones keep their scores."""
    for room in (0, 8192):
        run([5, 1, 20, 2], [60, 200, 20, 333], base, hq=8, hkv=2, room=room, seed=6, odd=odd)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("fp8", [True, False])
def test_a_query_that_is_not_finite_stays_alone(bad, fp8):
    """Rows with one value that is not finite give what they give; every other row is as if they were zeros."""
    D, bs, hq, hkv, n, T = 128, 16, 8, 2, 20, 100
    g = torch.Generator(device=DEV).manual_seed(3)
    x = (torch.randn((2 * 7, hkv, bs, D), generator=g, device=DEV) for _ in range(2))
    kc, vc = ((t_ * 16).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else t_.to(torch.bfloat16) for t_ in x)
    q = torch.randn((2 * n, hq, D), generator=g, device=DEV).to(torch.bfloat16)
    hit = torch.zeros((2 * n, hq), dtype=torch.bool, device=DEV)
    hit[3, 1] = hit[9, 6] = hit[n + 1, 0] = True
    q[hit] = 0
    for room in (112, 8192):
        sh = t.pool_shape(2, hq, hkv, D, bs, 14, room // bs)
        table = torch.zeros((2, room // bs), dtype=torch.int32, device=DEV)
        table[:, :7] = torch.arange(14, dtype=torch.int32, device=DEV).view(2, 7)
        ws = torch.empty(batch.chunk_workspace_bytes(sh, 2 * n, n), dtype=torch.uint8, device=DEV)
        outs = []
        for value in (0.0, bad):
            q[hit, 70] = value
            out = torch.full_like(q, 5.0)
            args = (sh, q, kc, vc, table, t.gpu([T, T - 7]), t.gpu([0, n, 2 * n]), n, 0.05)
            if fp8:
                batch.chunk_attention_fp8(*args, 0.07, 0.11, out, ws)
            else:
                batch.chunk_attention(*args, out, ws)
            outs.append(out)
        assert torch.equal(outs[0][~hit], outs[1][~hit])
