"""The `ramp` frequencies (scaled by index, between the indices that turn `high` and `low` times), from the published
definition and from what it promises (CPU)."""
import math

import numpy as np
import pytest
import torch

from paper_2511_21862_b200 import build, spec


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def published(rot, base, factor, length, low, high):
    """YaRN (Peng et al. 2023), "NTK-by-parts": correction range of whole indices, clamped to [0, rot - 1], and a linear ramp."""
    def dim_of(turns):
        return rot * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))

    first, last = max(math.floor(dim_of(high)), 0), min(math.ceil(dim_of(low)), rot - 1)
    j = torch.arange(rot // 2, dtype=torch.float64)
    inv = base ** -(2 * j / rot)
    kept = 1 - ((j - first) / ((last - first) or 1e-3)).clamp(0, 1)
    return (inv / factor * (1 - kept) + inv * kept).numpy()


CASES = [(rot, base, factor, length, 1.0, 32.0)
         for rot, base, factor in ((128, 1e4, 4.0), (64, 1e4, 8.0), (16, 1e4, 4.0), (128, 1e6, 4.0), (96, 5e5, 40.0))
         for length in (4096, 32768, 65536, 131072, 1 << 20)] + [(128, 1e4, 4.0, 65536, 0.5, 8.0), (32, 1e4, 2.0, 8192, 3.0, 4.0)]


@pytest.mark.parametrize("rot,base,factor,length,low,high", CASES)
def test_ramp_is_the_published_one(rot, base, factor, length, low, high):
    inv, mag = spec.rope_frequencies(rot, base, "ramp", factor=factor, original_len=length, low=low, high=high)
    want = published(rot, base, factor, length, low, high)
    # one rounding to fp32 beside differences of pow and log of a few 2^-53
    assert np.all(np.abs(inv.double().numpy() - want) <= 2.0 ** -24 * want * 1.001)
    assert abs(mag - (0.1 * math.log(factor) + 1)) <= 2.0 ** -24 * mag * 1.001


@pytest.mark.parametrize("rot,base,factor,length,low,high",
                         CASES + [(64, 1e4, 8.0, 4, 1.0, 2.0), (64, 1e4, 8.0, 6, 1.0, 32.0), (128, 1e4, 4.0, 64, 16.0, 32.0)])
def test_ramp_keeps_its_promises(rot, base, factor, length, low, high):
    """Frequencies that turn less than `low` times over `length` are divided by the whole factor, those that turn more than
    `low` times by less than it, those that turn more than `high` times (one index before that, the ramp's ends being whole
    indices) by nothing."""
    inv, _ = spec.rope_frequencies(rot, base, "ramp", factor=factor, original_len=length, low=low, high=high)
    ratio = spec.rope_frequencies(rot, base)[0].double() / inv.double()
    turns = np.array([length * base ** (-2 * j / rot) / (2 * math.pi) for j in range(rot // 2)])
    step = base ** (2 / rot)                                  # from one index to the next
    for j in range(rot // 2):
        if turns[j] < low * (1 - 1e-9):
            assert abs(float(ratio[j]) - factor) <= 1e-6 * factor, j
        if turns[j] > low * (1 + 1e-9):
            assert float(ratio[j]) < factor * (1 - 1e-6), j
        if turns[j] > high * step:
            assert abs(float(ratio[j]) - 1) <= 1e-6, j
