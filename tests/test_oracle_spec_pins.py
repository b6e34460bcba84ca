"""Pins of the plain definitions of the speculative-decoding operators, and of the host-side frequency table (CPU)."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import spec_oracle as so
from paper_2511_21862_b200 import build, spec


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def exact_distribution(p, q, tokens, parents, n):
    """Probability of every (accepted tokens, last token) outcome of one walk when the uniforms are uniform, by
    following the definition's branches with their probabilities (no random numbers)."""
    outcomes = {}

    def walk(cur, done, prob):
        w, mass = p[cur].astype(float).copy(), 1.0
        for c in range(cur + 1, n):
            if parents[c] != cur:
                continue
            x = tokens[c]
            take = min(1.0, w[x] / (mass * (1.0 if q is None else q[cur, x]))) if w[x] > 0 else 0.0
            walk_in = prob * take
            if walk_in > 0:
                walk(c, done + (x,), walk_in)
            prob *= 1 - take
            if q is None:
                mass -= w[x]
                w[x] = 0
            else:
                w = np.maximum(w - mass * q[cur], 0)
                mass = w.sum()
        if prob > 1e-15:
            for x in range(p.shape[1]):
                if w[x] > 0:
                    key = done + (x,)
                    outcomes[key] = outcomes.get(key, 0.0) + prob * w[x] / w.sum()

    walk(0, (), 1.0)
    return outcomes


def first_token_law(outcomes, V):
    law = np.zeros(V)
    for key, pr in outcomes.items():
        law[key[0]] += pr
    return law


@pytest.mark.parametrize("children", [1, 2, 3])
def test_drawn_drafts_leave_the_targets_distribution(children):
    """Averaged over the drafts (drawn from q), the first token of the outcome has the target's distribution."""
    rng = np.random.default_rng(children)
    V, n = 4, children + 1
    p, q = rng.dirichlet(np.ones(V), n), rng.dirichlet(np.ones(V), n)
    parents = [-1] + [0] * children
    law = np.zeros(V)
    for drafts in itertools.product(range(V), repeat=children):
        weight = np.prod([q[0, x] for x in drafts])
        law += weight * first_token_law(exact_distribution(p, q, [0, *drafts], parents, n), V)
    assert np.allclose(law, p[0], atol=1e-12)


def test_chosen_drafts_leave_the_targets_distribution():
    """Whatever tokens are proposed (repeated ones included), the first token has the target's distribution."""
    rng = np.random.default_rng(7)
    V = 5
    p = rng.dirichlet(np.ones(V), 4)
    for drafts in [(0, 1, 2), (3, 3, 1), (4, 4, 4)]:
        law = first_token_law(exact_distribution(p, None, [0, *drafts], [-1, 0, 0, 0], 4), V)
        assert np.allclose(law, p[0], atol=1e-12)


@pytest.mark.parametrize("drawn", [True, False])
def test_walk_follows_its_uniforms(drawn):
    """The walk with given uniforms, over a fine grid of them, spends on every outcome its probability."""
    rng = np.random.default_rng(11)
    V, n = 3, 3
    p = rng.dirichlet(np.ones(V), n).astype(np.float32)
    q = rng.dirichlet(np.ones(V), n).astype(np.float32) if drawn else None
    tokens, parents = np.array([0, 1, 2]), np.array([-1, 0, 0])
    want = exact_distribution(p, q, list(tokens), list(parents), n)
    grid = (np.arange(40) + 0.5) / 40
    got = {}
    for u in itertools.product(grid, repeat=3):
        path, out, count, _ = so.verify(p, q, tokens, parents, n, np.array(u, np.float32))
        got[tuple(out[: count + 1])] = got.get(tuple(out[: count + 1]), 0) + 40.0 ** -3
    # every outcome's region is a box per factor, so a grid of 40 points per axis misses each edge by at most 1/40
    for key in set(want) | set(got):
        assert abs(want.get(key, 0) - got.get(key, 0)) <= 3 / 40, key


def test_identical_distributions_accept_and_edges():
    p = np.array([[0.25, 0.75], [0.5, 0.5], [1.0, 0.0]], np.float32)
    path, out, count, _ = so.verify(p, p, np.array([0, 1, 0]), None, 3, np.array([0.0, 0.99, 0.99], np.float32))
    assert list(path) == [0, 1, 2] and list(out) == [1, 0, 0] and count == 2
    path, out, count, _ = so.verify(p, p, np.array([0, 1, 0]), None, 0, np.zeros(3, np.float32))
    assert list(path) == [-1] * 3 and list(out) == [-1] * 3 and count == 0


def test_slots_by_hand():
    table = np.full((3, 4), -1)
    table[0, :1], table[1, :2] = [7], [3, 5]
    r = so.plan_slots(np.array([2, 7, 0]), np.array([3, 2, 9]), table, np.array([1, 2, 0]), np.array([9, 8, 1, 0, 2]), 1,
                      block_size=4, num_blocks=10, row_len=0, num_rows=16)
    assert list(r["table"][0]) == [7, 8, -1, -1] and list(r["table"][1]) == [3, 5, 1, -1]
    assert list(r["slot_map"][:5]) == [30, 31, 32, 23, 4]
    assert list(r["positions"][:5]) == [2, 3, 4, 7, 8]
    # the third sequence needs three blocks and two are left: refused, nothing taken for it
    assert list(r["granted"]) == [3, 2, 0] and r["head"] == 3 and r["status"] == 128 and set(r["slot_map"][5:]) == {-1}
    assert list(r["total"]) == [5, 9, 0] and list(r["held"]) == [2, 3, 0] and list(r["first_token"]) == [0, 3, 5, 14]


def test_rope_keeps_relative_positions():
    """A rotated pair's length is magnitude times the old one, and q.k depends on the distance alone."""
    rng = np.random.default_rng(3)
    inv = 1 / 10000 ** (np.arange(8) / 8)
    for inter in (False, True):
        x, y = rng.standard_normal((1, 1, 24)), rng.standard_normal((1, 1, 24))
        dots = [float(np.sum(so.rope(x, [a], inv, 16, inter, 1.0) * so.rope(y, [a + 5], inv, 16, inter, 1.0)))
                for a in (0, 17, 4000)]
        assert np.allclose(dots, dots[0], atol=1e-9)
        z = so.rope(x, [12345], inv, 16, inter, 1.5)
        assert np.allclose(np.sum(z[..., :16] ** 2), 2.25 * np.sum(x[..., :16] ** 2)) and np.array_equal(z[..., 16:], x[..., 16:])


def test_keep_path_by_hand():
    pool = np.arange(4 * 1 * 2 * 1).reshape(4, 1, 2, 1).astype(float)
    table = np.array([[2, 0, 3, -1]])
    before = pool.copy()
    new = so.keep_path(pool, table, np.array([1]), np.array([[0, 2, 4, -1, -1]]), np.array([2]), 2)
    flat = lambda x, t: x[table[0, t // 2], 0, t % 2, 0]  # noqa: E731
    assert list(new) == [4]
    assert [flat(pool, t) for t in range(6)] == [flat(before, t) for t in (0, 1, 3, 5, 4, 5)]


def test_sees():
    par = [-1, 0, 0, 1, 3, 2]
    assert so.sees(par, 4) == {0, 1, 3, 4} and so.sees(par, 5) == {0, 2, 5} and so.sees([-1, -1, 1], 2) == {1, 2}


# ------------------------------------------------------------------------------------ frequencies (host code)
def frequencies(rot, base, kind, factor, length, low, high):
    """Written apart from the library: per index, from the definitions."""
    out, mag = [], 1.0
    for j in range(rot // 2):
        w = 1.0 / base ** (2 * j / rot)
        if kind == "linear":
            w = w / factor
        elif kind == "stretch":
            w = 1.0 / (base * factor ** (rot / (rot - 2))) ** (2 * j / rot)
        elif kind == "bands":
            wave = 2 * math.pi / w
            if wave > length / low:
                w /= factor
            elif wave >= length / high:
                smooth = (length / wave - low) / (high - low)
                w = (1 - smooth) * w / factor + smooth * w
        elif kind == "ramp":
            find = lambda turns: rot * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
            a, b = max(math.floor(find(high)), 0), min(math.ceil(find(low)), rot // 2 - 1)
            r = min(1.0, max(0.0, (j - a) / max(b - a, 1e-3)))
            w = w / factor * r + w * (1 - r)
            mag = 0.1 * math.log(factor) + 1
        out.append(w)
    return np.array(out), mag


@pytest.mark.parametrize("rot,base", [(128, 10000.0), (128, 5e5), (64, 1e6), (16, 10000.0)])
@pytest.mark.parametrize("kind,factor,length,low,high", [
    ("plain", 1.0, 0, 0.0, 0.0), ("linear", 4.0, 0, 0.0, 0.0), ("stretch", 8.0, 0, 0.0, 0.0),
    ("bands", 8.0, 8192, 1.0, 4.0), ("ramp", 32.0, 4096, 1.0, 32.0), ("ramp", 1.0, 4096, 1.0, 32.0)])
def test_frequencies(rot, base, kind, factor, length, low, high):
    inv, mag = spec.rope_frequencies(rot, base, kind, factor=factor, original_len=length, low=low, high=high)
    want, want_mag = frequencies(rot, base, kind, factor, length, low, high)
    assert inv.dtype == torch.float32
    # one rounding to fp32 (2^-24) beside pow / log differences of a few 2^-53
    assert np.all(np.abs(inv.double().numpy() - want) <= 2.0 ** -24 * want * 1.001)
    assert abs(mag - want_mag) <= 2.0 ** -24 * want_mag * 1.001
