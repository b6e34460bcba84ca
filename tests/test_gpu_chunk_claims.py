"""Packed chunk attention where the arrays on the device break the rule that rows of different sequences are distinct: what does not fit
the workspace, which was sized by the number of rows, is refused and nothing is written behind it."""
import pytest
import torch

import test_gpu_batch as t
from paper_2511_21862_b200 import batch, binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda"
GUARD = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


def claim_one_row(lens, room, *, hq, hkv, fp8, rows=1, extra=()):
    """Sequences of the given contexts, every second one with one new token in row 0 and the others with none; `extra`: first rows and
    lengths of sequences behind them.  Returns (status, output)."""
    bs, D, NB = 64, 128, -(-max(lens) // 64) + 1
    first, ctx = [], []
    for n in lens:                         # first_row 0, 1, 0, 1, ...: one token, then fewer than none
        first += [0, 1]
        ctx += [n, n]
    first, ctx = first + [f for f, _ in extra] + [rows], ctx + [n for _, n in extra]
    B = len(ctx)
    table = torch.zeros((B, room // bs), dtype=torch.int32, device=DEV)
    table[:, :NB] = torch.arange(NB, dtype=torch.int32, device=DEV)
    sh = t.pool_shape(B, hq, hkv, D, bs, NB, room // bs)
    g = torch.Generator(device=DEV).manual_seed(len(lens))
    kc, vc = (torch.randn((NB, hkv, bs, D), generator=g, device=DEV) for _ in range(2))
    kc, vc = ((x.to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else x.to(torch.bfloat16)) for x in (kc, vc))
    q = torch.randn((rows, hq, D), generator=g, device=DEV).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    need = batch.chunk_workspace_bytes(sh, rows, rows)
    whole = torch.full((need + GUARD,), 171, dtype=torch.uint8, device=DEV)
    ws = whole[:need]
    args = (sh, q, kc, vc, table, t.gpu(ctx), t.gpu(first), rows, 0.1)
    if fp8:
        batch.chunk_attention_fp8(*args, 1.0, 1.0, out, ws)
    else:
        batch.chunk_attention(*args, out, ws)
    torch.cuda.synchronize()
    assert (whole[need:] == 171).all()
    return binding.workspace_status(ws), out


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv", [(64, 8), (4, 4)])
def test_more_decodes_than_rows(hq, hkv, fp8):
    """Thousands of short contexts and, behind them, a long one that is cut into many pieces, all in one row."""
    status, out = claim_one_row([1] * 3000 + [8000], 8192, hq=hq, hkv=hkv, fp8=fp8)
    assert status == 1 and (out == 7).all()


def test_more_cut_decodes_than_rows():
    """Two long contexts in one row: their pieces would fit, the rows to be merged do not."""
    status, out = claim_one_row([9000, 9000], 1 << 16, hq=4, hkv=1, fp8=False)
    assert status == 1 and (out == 7).all()


def test_other_sequences_of_the_call_are_served():
    """Only the list of sequences with one new token is dropped."""
    status, out = claim_one_row([1] * 3000 + [8000], 8192, hq=8, hkv=2, fp8=False, rows=5, extra=[(1, 4), (5, 4)])
    assert status == 1 and (out[0] == 7).all()
    assert not (out[1:] == 7).all(-1).any() and torch.isfinite(out.float()).all()


def test_as_many_decodes_as_rows_fit():
    """The bound itself: one token a row, contexts as long as the table, every one cut."""
    t.run_chunk([1] * 40, [3000] * 40, hq=8, hkv=2, bs=16, pad=0, seed=3, max_chunk=1)
    t.run_chunk([1], [60000], hq=8, hkv=1, bs=64, pad=0, seed=4, max_chunk=1)
