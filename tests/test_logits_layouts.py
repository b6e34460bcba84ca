"""Shaped logits whose outputs lie node by node, not sequence by sequence: any strides with distinct rows are taken."""
import ctypes

import pytest
import torch

from paper_2511_21862_b200 import batch, binding, build

SHAPE = -2
STEP = 1 << 20   # (addresses on the CPU are never dereferenced)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def refused(B, N, V, seq, node):
    """Whether the C entry refuses outputs with these strides for their shape (without a GPU, what it accepts fails later)."""
    c = batch.ooco_logits_t(B, N, V, 1, 0, 0, N * V, V, seq, node, N * V, V, 0, 0)
    rc = batch._lib().ooco_shape_logits(ctypes.byref(c), STEP, *[None] * 13, 2 * STEP, None, None)
    assert rc != 0
    return rc == SHAPE


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses, for hosts without a GPU")
def test_strides():
    B, N, V = 3, 4, 100
    for seq, node in ((400, 100), (100, 300), (120, 360), (120, 341), (1 << 40, 100), (100, 1 << 40), (103, 307), ((1 << 62), 200)):
        assert not refused(B, N, V, seq, node), (seq, node)
    for seq, node in ((399, 100), (100, 299), (99, 1000), (1000, 99), (120, 339), (0, 100), (100, 0), (100, 100), (150, 120), (-400, 100)):
        assert refused(B, N, V, seq, node), (seq, node)
    assert not refused(1, N, V, 0, 100) and not refused(B, 1, V, 100, 0) and not refused(1, 1, V, 0, 0)
    assert refused(1, N, V, 0, 99) and refused(B, 1, V, 99, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [64, 1003, 50001])
def test_node_major_tables(V):
    """Views whose nodes are the outer dimension, in and out, in place too, give what contiguous tables give."""
    binding.lib()
    B, N = 3, 5
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((B, N, V), generator=g, device="cuda") * 3
    kw = dict(history=torch.randint(0, V, (B, 40), generator=g, device="cuda", dtype=torch.int32),
              history_lens=torch.full((B,), 40, dtype=torch.int32, device="cuda"), repetition=torch.full((B,), 1.3, device="cuda"),
              temperature=torch.tensor([0.7, 0.0, 1.1], device="cuda"))
    out, probs = torch.empty_like(x), torch.empty_like(x)
    batch.shape_logits(x, out=out, probs=probs, **kw)
    turned = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    o, p = torch.full((N, B, V), 9.0, device="cuda").transpose(0, 1), torch.full((N, B, V + 3), 9.0, device="cuda").transpose(0, 1)
    batch.shape_logits(turned(x), out=o, probs=p[..., :V], **kw)
    assert torch.equal(o, out) and (p[..., V:] == 9).all()
    # Rows of V + 3 values do not begin on boundaries of four, so another instantiation sums them, in another order: either result is
    # within expm1(3 * 2^-24 (d + 11.1)) + 2^-19 of the softmax (d = distance of the exponent to the largest: three roundings of an
    # exponent that may be taken beside a reference 11.1 away; exp, sum and quotient), their difference within twice that.
    d = -torch.log((probs / probs.amax(-1, keepdim=True)).clamp(min=1e-37)).double()
    rel = 2 * (torch.expm1(3 * 2.0 ** -24 * (d + 11.1)) + 2.0 ** -19)
    assert ((p[..., :V].double() - probs.double()).abs() <= rel * probs.double()).all()
    y = turned(x)
    batch.shape_logits(y, probs=y, **kw)
    assert torch.equal(y, probs)
