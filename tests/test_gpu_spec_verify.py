"""Verification of drafts where the draft's probabilities hold values that are none (GPU), against the definition."""
import numpy as np
import pytest
import torch

from paper_2511_21862_b200 import binding, build

import test_gpu_spec as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.lib()


@pytest.mark.parametrize("odd", [float("nan"), -0.25], ids=["nan", "negative"])
@pytest.mark.parametrize("B,N,V", [(3, 6, 700), (6, 12, 5000), (40, 9, 1111), (4, 5, 40001)])
def test_draft_probabilities_that_are_none_count_as_zero(B, N, V, odd):
    """At drafted tokens (a child of such a probability is accepted where the target gives it any weight) and elsewhere (the
    token keeps its whole weight when others are refused)."""
    p, q, tokens, par, u = base.verify_inputs(B * N + V, B, N, V, "star" if B % 2 else "tree", True, noise=1.5)
    rng = np.random.default_rng(V)
    everywhere = rng.random((B, N, V)) < 0.05
    at_drafts = np.zeros((B, N, V), bool)
    for b in range(0, B, 2):                              # half of the sequences: at some drafted tokens, too
        for i in range(1, N, 2):
            at_drafts[b, max(0, int(par[b, i])), int(tokens[b, i])] = True
    for b in range(1, B, 2):                              # the others: not at them, so that they are refused now and then
        for i in range(1, N):
            everywhere[b, max(0, int(par[b, i])), int(tokens[b, i])] = False
    q[torch.as_tensor(everywhere | at_drafts, device="cuda")] = odd
    got = base.check_verify(p, q, tokens, par, u)
    assert got[2].max() > 0


@pytest.mark.parametrize("V", [300, 4000])
def test_a_row_without_any_draft_probability(V):
    """All of a row's draft probabilities NaN: every child with weight is accepted, and nothing leaves the weights."""
    B, N = 8, 5
    p, q, tokens, par, u = base.verify_inputs(5, B, N, V, "star", True)
    q[:, 0] = float("nan")
    p[1, 0, int(tokens[1, 1])] = 0.0                      # a child without weight, in one sequence
    path, out, count = base.check_verify(p, q, tokens, par, u)
    assert [int(c) for c in count] == [1] * B
    assert path[0, 1] == 1 and path[1, 1] == (2 if tokens[1, 2] != tokens[1, 1] else path[1, 1])


@pytest.mark.parametrize("drawn", [True, False])
def test_rows_of_nodes_not_reached_do_not_matter(drawn):
    """Whatever stands in the rows of nodes that the walk does not reach, and in the draft's rows of leaves."""
    B, N, V = 12, 10, 900
    p, q, tokens, par, u = base.verify_inputs(31, B, N, V, "tree", drawn)
    want = base.run_verify(p, q, tokens, par, u, None)
    for b in range(B):
        for i in range(N):
            if i not in want[0][b]:
                p[b, i] = float("nan") if i % 2 else float("inf")
            if drawn and (i not in want[0][b] or i not in par[b]):
                q[b, i] = float("inf") if i % 2 else float("nan")
    got = base.run_verify(p, q, tokens, par, u, None)
    assert all(np.array_equal(a, b) for a, b in zip(got, want))
