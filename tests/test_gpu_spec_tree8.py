"""Tree attention over the 8-bit cache within the roundings that its kernels really have, and chains against the causal
operator where trees have a kernel of their own (9 to 64 score columns)."""
import math

import numpy as np
import pytest
import torch

from oracle import spec_oracle as so
from paper_2511_21862_b200 import binding, build
from util import fp32_output

import test_gpu_spec as base
from tree_tolerance import tolerance

pytestmark = pytest.mark.gpu
FP8 = (0.02, 0.03)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def check(c, seqs=None):
    with fp32_output():
        out = base.run_tree(c, f32=True).cpu().double().numpy()
    G, worst = c["hq"] // c["hkv"], 0.0
    q = c["q"].cpu().double().numpy()
    pools = [base.as_head_major(x, c["layout"]) for x in (c["k"], c["v"])]
    for b in range(len(c["lens"])):
        T = int(c["lens"][b])
        n = c["N"] if c["sizes"] is None else max(0, min(c["N"], int(c["sizes"][b])))
        if n == 0 or (seqs is not None and b not in seqs):
            continue
        ids = torch.as_tensor(c["table"][b, : -(-T // c["bs"])], device="cuda").long()
        k, v = (x[ids].view(base.E4M3).double().mul(s).permute(1, 0, 2, 3).flatten(1, 2)[:, :T].cpu().numpy()
                for x, s in zip(pools, c["fp8"]))
        for h in range(c["hkv"]):
            heads = slice(h * G, (h + 1) * G)
            want, mag, spread = so.tree_attention(q[b, :n, heads], k[h], v[h], c["par"][b], n, c["scale"])
            tol = tolerance(q[b, :n, heads], k[h], v[h], mag, spread, c["scale"]) + 1e-30
            ratio = np.abs(out[b, :n, heads] - want) / tol
            worst = max(worst, float(ratio.max()))
            assert np.all(ratio <= 1), (b, h, float(ratio.max()))
    return worst


@pytest.mark.parametrize("name", [n for n in base.TREE_CASES if base.TREE_CASES[n][-1].get("fp8")])
def test_listed_shapes(name):
    lens, hq, hkv, D, bs, N, opt = base.TREE_CASES[name]
    check(base.tree_case(lens, hq, hkv, D, bs, N, seed=sum(map(ord, name)), sigma=0.7, **opt))


@pytest.mark.parametrize("hq,N", [(16, 9), (40, 8), (32, 16), (48, 16)])
def test_many_short_units(hq, N):
    rng = np.random.default_rng(hq * N)
    lens = [int(x) for x in rng.integers(N, 385, 56)] + [128, 129, 256, 257, 384, 1, 0, 16]
    check(base.tree_case(lens, hq, 8, 128, 16, N, seed=N, fp8=FP8, sigma=0.7, sizes=[N if i % 3 else 1 + i % N for i in range(64)]),
          seqs=range(0, 64, 3))


@pytest.mark.parametrize("hq,N", [(16, 2), (32, 4), (16, 9), (48, 8), (48, 16), (64, 16), (64, 20)])
def test_scores_far_apart(hq, N):
    """References that are raised, and accumulators rescaled, again and again."""
    c = base.tree_case([N, 200, 700, 1500], hq, 8, 128, 16, N, seed=N + hq, fp8=FP8, sigma=1.0)
    c["q"].mul_(torch.logspace(-1, 1.3, hq, device="cuda")[None, None, :, None])
    ramp = torch.linspace(0.05, 1.0, c["k"].shape[0], device="cuda")[:, None, None, None]
    c["k"] = (c["k"].view(base.E4M3).float() * ramp).to(base.E4M3).view(torch.uint8)
    check(c)


@pytest.mark.parametrize("hq,N", [(16, 2), (32, 4), (16, 9), (40, 8), (32, 12), (48, 16)])
def test_rows_of_every_magnitude(hq, N):
    """Query rows from 2^-40 to 2^5, dims within a row down to 2^-20 of its largest."""
    c = base.tree_case([N, 130, 300, 520], hq, 8, 128, 16, N, seed=N * hq, fp8=FP8, sigma=0.7)
    c["q"].mul_(torch.logspace(-40, 5, hq, base=2.0, device="cuda").to(torch.bfloat16)[None, None, :, None])
    c["q"][:, :, ::2].mul_(torch.logspace(-20, 0, 128, base=2.0, device="cuda").to(torch.bfloat16))
    check(c)


@pytest.mark.parametrize("fp8", [None, FP8], ids=["bf16", "fp8"])
@pytest.mark.parametrize("hq,N", [(8, 9), (16, 5), (32, 4), (24, 6), (32, 8), (40, 8), (48, 8), (32, 16), (64, 8), (128, 4)])
def test_chains_against_the_causal_operator(hq, N, fp8):
    """Two kernels that differ in their roundings only: each within its own of the definition, so within twice that of one
    another.  (sum |weight * value| from the causal operator itself, over |v|: its 1 % are in the factor 2.1.)"""
    c = base.tree_case([N, 100, 300, 3000, 129], hq, 8, 128, 16, N, seed=N, kind="chain", fp8=fp8, sigma=0.7)
    with fp32_output():
        tree = base.run_tree(c, f32=True)
    ws = torch.empty(binding.workspace_bytes_mq(c["shape"], N), dtype=torch.uint8, device="cuda")
    table, lens = base.gpu(c["table"].astype(np.int32)), base.gpu(c["lens"])

    def causal(v):
        out = torch.empty(c["q"].shape, dtype=torch.float32, device="cuda")
        with fp32_output():
            if fp8:
                binding.decode_step_mq_fp8(c["shape"], c["q"], None, None, c["k"], v, table, torch.zeros_like(lens), lens,
                                           c["scale"], *fp8, out, ws)
            else:
                binding.decode_attention_mq(c["shape"], c["q"], c["k"], v, table, lens, c["scale"], out, ws)
        assert binding.workspace_status(ws) == 0
        return out

    want = causal(c["v"])
    mag = causal(c["v"] & 0x7f if fp8 else c["v"].abs())
    if fp8:
        k, v = (c[x].view(base.E4M3).float().nan_to_num() * s for x, s in zip("kv", fp8))
        largest = float((c["q"].float().abs().amax() * k.abs().sum(-1).amax()) * c["scale"])    # of any score's terms
        relative = 2.0 ** -10 + 2.0 ** -12 + math.expm1(2 * (2.0 ** -15.8 + 2.0 ** -17) * largest)
        floor = 2 * 2.0 ** -25 * 3000 * float(v.abs().amax())
    else:
        relative, floor = 2.0 ** -7 + 1e-4, 1e-6       # (weights in bf16, as in check_tree)
    assert bool(((tree - want).abs() <= 2.1 * (relative * mag + floor)).all())
    assert float(want.abs().max()) > 0.5
