"""The tolerance of the 8-bit tree tests tells mistakes from rounding: mistakes are planted in the definition (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import spec_oracle as so

from tree_tolerance import tolerance

E4M3 = torch.float8_e4m3fn


def case(T, n, G, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    k, v = ((torch.randn((T, 128), generator=g) * 0.7 / s).clamp(-448, 448).to(E4M3).double().numpy() * s for s in (0.02, 0.03))
    q = (torch.randn((n, G, 128), generator=g) * 0.7 * gain).to(torch.bfloat16).double().numpy()
    par = [-1] + [(i - 1) // 2 for i in range(1, n)]
    return q, k, v, par


def high_term(q):
    """The larger of the two E4M3 terms of a query, alone."""
    exponent = np.floor(np.log2(np.abs(q).max(-1, keepdims=True)))
    a = 2.0 ** (7 - exponent)
    return torch.as_tensor(q * a).to(E4M3).double().numpy() / a


def wrong(T, n, G, seed, mistake, gain=1.0):
    """Largest error of the mistaken output in units of the tolerance."""
    q, k, v, par = case(T, n, G, seed, gain)
    scale = 1 / math.sqrt(128)
    want, mag, spread = so.tree_attention(q, k, v, par, n, scale)
    tol = tolerance(q, k, v, mag, spread, scale)
    return float((np.abs(mistake(q, k, v, par, n, scale, want) - want) / tol).max())


def attention(q, k, v, par, n, scale):
    return so.tree_attention(q, k, v, par, n, scale)[0]


@pytest.mark.parametrize("T,n,G", [(17, 9, 2), (40, 8, 5), (130, 16, 4), (300, 16, 4)])
def test_a_query_without_its_low_term(T, n, G):
    assert wrong(T, n, G, T, lambda q, k, v, par, n, s, want: attention(high_term(q), k, v, par, n, s)) > 2


@pytest.mark.parametrize("T,n,G,gain", [(300, 8, 5, 1.0), (1500, 16, 4, 1.0), (2500, 8, 5, 1.0), (2500, 16, 4, 10.0)])
def test_a_stage_left_out(T, n, G, gain):
    def mistake(q, k, v, par, n, s, want):
        keep = np.r_[0:64, 192:T]
        return attention(q, k[keep], v[keep], par, n, s)
    assert wrong(T, n, G, T, mistake, gain) > 5


@pytest.mark.parametrize("gain", [1.0, 10.0, 60.0])
def test_nothing_and_a_rescaling_left_out(gain):
    assert wrong(700, 8, 6, 1, lambda q, k, v, par, n, s, want: 0 * want, gain) > 20

    def unscaled(q, k, v, par, n, s, want):
        """The first half's part of the sums kept at a reference 14 (log2) below the second half's."""
        out = np.zeros_like(want)
        T = k.shape[0]
        for i in range(n):
            tok = [t for t in range(T - n)] + [T - n + j for j in so.sees(par, i)]
            x = (q[i] @ k[tok].T) * s
            w = np.exp(x - x.max(-1, keepdims=True)) * np.where(np.array(tok) < T // 2, 2.0 ** 14, 1.0)
            out[i] = (w / w.sum(-1, keepdims=True)) @ v[tok]
        return out
    assert wrong(700, 8, 6, 2, unscaled, gain) > 20


def test_rounding_alone_stays_within():
    """Weights rounded to f16 below a reference that is up to 2^14 too low, sums of the rounded weights, in 64 bits otherwise."""
    for T, n, G, gain in ((17, 9, 2, 1.0), (300, 8, 5, 1.0), (2500, 8, 5, 1.0), (700, 8, 6, 30.0)):
        q, k, v, par = case(T, n, G, T + 1, gain)
        scale = 1 / math.sqrt(128)
        want, mag, spread = so.tree_attention(q, k, v, par, n, scale)
        tol = tolerance(q, k, v, mag, spread, scale)
        for lag in (0.0, 7.3, 13.9):
            for i in range(n):
                tok = [t for t in range(T - n)] + [T - n + j for j in so.sees(par, i)]
                x = (q[i] @ k[tok].T) * scale / math.log(2)
                w = np.exp2(x - x.max(-1, keepdims=True) + lag).astype(np.float16).astype(np.float64)
                assert np.all(np.abs(w @ v[tok] / w.sum(-1, keepdims=True) - want[i]) <= tol[i])
