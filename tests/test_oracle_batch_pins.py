"""Pins of the continuous-batching oracle: closed forms, hand-worked cases, library counterparts (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import batch_oracle as bo


def test_fork_by_hand():
    # row 0: 20 tokens in blocks 5, 6 (block size 16); rows 2 and 3 become its children, 3 of its first 16 tokens alone
    table = np.array([[5, 6, -1], [7, -1, -1], [-1, -1, -1], [-1, -1, -1]])
    r = bo.fork_pages([0, 0], [2, 3], np.array([99, 16]), np.array([20, 3, 0, 0]), table, np.array([2, 1, 0, 0]), np.array([8, 9]),
                      0, np.zeros(10, int), block_size=16, num_blocks=10)
    assert r["table"].tolist() == [[5, 6, -1], [7, -1, -1], [5, 8, -1], [5, -1, -1]]
    assert r["ctx"].tolist() == [20, 3, 20, 16] and r["held"].tolist() == [2, 1, 2, 1]
    assert r["copy_src"].tolist() == [6, -1] and r["copy_dst"].tolist() == [8, -1] and r["head"] == 1
    assert r["shares"][5] == 2 and r["shares"].sum() == 2 and r["granted"].tolist() == [1, 1] and r["status"] == 0


def test_release_by_hand():
    # block 5 has three holders: two rows of the list give it back, the third keeps it; 6 and 8 become free in that order
    table = np.array([[5, 6], [5, 8], [5, 9]])
    free = np.array([-1, -1, -1, 3])
    r = bo.release_pages([1, 0], None, np.array([20, 30, 17]), table, np.array([2, 2, 2]), free, 3, np.array([0] * 5 + [2] + [0] * 4),
                         block_size=16, num_blocks=10)
    assert r["free"].tolist() == [-1, 8, 6, 3] and r["head"] == 1 and r["shares"].sum() == 0 and r["status"] == 0
    assert r["ctx"].tolist() == [0, 0, 17] and r["held"].tolist() == [0, 0, 2]


def test_release_is_the_inverse_of_fork():
    rng = np.random.default_rng(0)
    table, held, ctx = np.full((6, 5), -1), np.array([4, 2, 3, 0, 0, 0]), np.array([60, 32, 33, 0, 0, 0])
    ids = rng.permutation(20)
    table[0, :4], table[1, :2], table[2, :3] = ids[:4], ids[4:6], ids[6:9]
    free = ids[9:]
    f = bo.fork_pages([0, 2, 1], [3, 4, 5], None, ctx, table, held, free, 0, np.zeros(20, int), block_size=16, num_blocks=20)
    r = bo.release_pages([3, 4, 5], None, f["ctx"], f["table"], f["held"], free, f["head"], f["shares"], block_size=16, num_blocks=20)
    assert r["head"] == 0 and not r["shares"].any() and sorted(r["free"]) == sorted(free) and r["ctx"].tolist() == ctx.tolist()


def test_head_norm_against_torch():
    x, w = torch.randn(3, 2, 64, dtype=torch.float64), torch.randn(64, dtype=torch.float64)
    want = torch.nn.functional.rms_norm(x, (64,), w + 0.5, 1e-5)
    assert np.allclose(bo.head_norm(x.numpy(), w.numpy(), 1e-5, 0.5), want.numpy(), rtol=1e-13)
    assert np.allclose(np.square(bo.head_norm(x.numpy(), None, 0.0, 0.0)).mean(-1), 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_turn_keeps_lengths_and_relative_angles(interleaved):
    rng = np.random.default_rng(1)
    q, k, inv = rng.standard_normal((1, 1, 32)), rng.standard_normal((1, 1, 32)), 1e4 ** (-np.arange(8) / 8)
    t = lambda x, p: bo.turn(x, [p], inv, interleaved)  # noqa: E731
    assert np.isclose(np.linalg.norm(t(q, 77)), np.linalg.norm(q)) and np.array_equal(t(q, 5)[..., 16:], q[..., 16:])
    assert np.isclose((t(q, 12) * t(k, 9)).sum(), (t(q, 103) * t(k, 100)).sum())


def test_attention_against_torch():
    n, T, Hq, Hkv, D = 5, 9, 4, 2, 16
    q, k, v = (torch.randn(a, b, D, dtype=torch.float64) for a, b in ((n, Hq), (T, Hkv), (T, Hkv)))
    mask = torch.arange(T) <= torch.arange(T - n, T)[:, None]
    kk, vv = (x.transpose(0, 1).repeat_interleave(2, 0) for x in (k, v))
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), kk, vv, attn_mask=mask, scale=0.3).transpose(0, 1)
    out, mag, _ = bo.chunk_attention(q.numpy(), k.numpy(), v.numpy(), n, 0.3)
    assert np.allclose(out, want.numpy(), atol=1e-12) and (np.abs(out) <= mag + 1e-12).all()
    out, _, _ = bo.chunk_attention(q.numpy(), k.numpy()[:2], v.numpy()[:2], n, 0.3)       # the first three see nothing
    assert not out[:3].any() and np.allclose(out[3, 0], v.numpy()[0, 0])


def test_logits_by_hand():
    x = np.array([2.0, -2.0, 1.0, 0.5, 3.0])
    out, p = bo.shape_logits(x.copy(), repetition=2.0, frequency=0.25, presence=0.5, text=[0, 1, 1, 3], prompt=2, branch=[3],
                             bias=[(2, 1.0), (2, 0.5), (7, 9.0)], allowed=np.array([1, 1, 1, 1, 0], bool))
    # token 0: prompt only; 1: prompt and once generated; 3: once generated, once drafted
    assert out.tolist()[:4] == [1.0, -4.0 - 0.25 - 0.5, 2.5, 0.25 - 0.5 - 0.5] and out[4] == -math.inf
    e = np.exp(out - 2.5)
    assert np.allclose(p, e / e.sum())
    assert bo.shape_logits(x.copy(), temperature=0.0)[1].tolist() == [0, 0, 0, 0, 1]
    assert not bo.shape_logits(x.copy(), allowed=np.zeros(5, bool))[1].any()
    assert bo.shape_logits(np.array([np.nan, np.inf, np.inf]))[1].tolist() == [0, 0.5, 0.5]
