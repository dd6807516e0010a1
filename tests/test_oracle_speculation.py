"""Pins of oracle/speculation.py: trees against the multi-query oracle and brute force, the
verification against the distribution that it has to leave untouched."""
import itertools

import numpy as np
import pytest

from oracle import multi_query as OM
from oracle import speculation as OS


def rows(g, *shape):
    return g.standard_normal(shape)


@pytest.mark.parametrize("L,T", [(5, 3), (3, 3), (9, 1)])
def test_a_chain_is_the_causal_mask(L, T):
    g = np.random.default_rng(L)
    q, qp, C, K = rows(g, T, 2, 16), rows(g, T, 2, 4), rows(g, L, 16), rows(g, L, 4)
    out, lse, _ = OS.attend_tree(q, qp, C, K, np.arange(T) - 1, T, 0.3)
    want, want_lse = OM.attend_multi(q, qp, C, K, 0.3)
    assert np.allclose(out, want, atol=1e-13) and np.allclose(lse, want_lse, atol=1e-13)


def test_each_node_is_a_sequence_of_its_own_line():
    g = np.random.default_rng(1)
    parents = [-1, 0, 0, 1, 2, 1, -1, 6]
    T, ctx = len(parents), 4
    q, qp, C, K = rows(g, T, 3, 16), rows(g, T, 3, 4), rows(g, ctx + T, 16), rows(g, ctx + T, 4)
    out, lse, _ = OS.attend_tree(q, qp, C, K, parents, T, 0.3)
    for t in range(T):
        at = list(range(ctx)) + [ctx + i for i in sorted(OS.line_of(parents, t))]
        want, want_lse = OM.attend_multi(q[t:t + 1], qp[t:t + 1], C[at], K[at], 0.3)
        assert np.allclose(out[t], want[0], atol=1e-13) and np.allclose(lse[t], want_lse[0], atol=1e-13)


def test_bad_parents_and_nodes_behind_the_last_see_nothing():
    g = np.random.default_rng(2)
    q, qp, C, K = rows(g, 6, 1, 16), rows(g, 6, 1, 4), rows(g, 9, 16), rows(g, 9, 4)
    out, lse, _ = OS.attend_tree(q, qp, C, K, [-1, 1, 1, 0, -2, 0], 5, 0.3)
    assert np.isfinite(lse[[0, 3]]).all() and (lse[[1, 2, 4, 5]] == -np.inf).all() and (out[[1, 2, 4, 5]] == 0).all()


def first_tokens(target, draft, k, steps=400):
    """Distribution of the first emitted token for k children drawn from the draft (or, where it is
    None, the tokens 0 .. k - 1), the random numbers on a grid."""
    V = target.shape[1]
    got = np.zeros(V)
    grid = (np.arange(steps) + 0.5) / steps
    fine = (np.arange(4 * steps) + 0.5) / (4 * steps)
    choices = list(itertools.product(range(V), repeat=k)) if draft is not None else [tuple(range(k))]
    for xs in choices:
        weight = np.prod([draft[0, x] for x in xs]) if draft is not None else 1.0
        tokens = [0, *xs]
        for us in itertools.product(grid, repeat=k):
            path, _ = OS.verify_tree(target, draft, tokens, [-1] + [0] * k, k + 1, [0.5, *us])
            w = weight / steps ** k
            if len(path) > 1:
                got[tokens[path[1]]] += w
                continue
            # (the residual does not depend on which of the random numbers refused: integrate the draw)
            if us == tuple([grid[-1]] * k) or not hasattr(first_tokens, "memo") or (xs, "r") not in first_tokens.memo:
                r = np.zeros(V)
                for f in fine:
                    r[OS.verify_tree(target, draft, tokens, [-1] + [0] * k, k + 1, [f, *us])[1]] += 1 / len(fine)
                first_tokens.memo = {**getattr(first_tokens, "memo", {}), (xs, "r"): r}
            got += w * first_tokens.memo[(xs, "r")]
    return got


@pytest.mark.parametrize("k,steps", [(1, 400), (2, 40)])
@pytest.mark.parametrize("certain", [False, True])
def test_the_first_token_keeps_the_targets_distribution(k, steps, certain):
    p, q = np.array([0.5, 0.2, 0.3]), np.array([0.2, 0.5, 0.3])
    target = np.tile(p, (k + 1, 1))
    draft = None if certain else np.tile(q, (k + 1, 1))
    first_tokens.memo = {}
    got = first_tokens(target, draft, k, steps)
    # each random number's grid moves a border by half a cell at most: 3 borders a number
    assert np.abs(got - p).max() <= 3 * (k + 1) / steps


def test_walk_by_hand():
    p, q = np.array([[0.5, 0.5, 0.0]] * 4), np.array([[0.25, 0.25, 0.5]] * 4)
    parents = [-1, 0, 0, 2]
    # node 1 (token 2, p = 0) is refused; what is left is (p - q)+ = (.25, .25, 0) of sum .5, so the
    # next child, of token 0, has 0.5 left against q = .25: taken; then its child of token 1
    tokens = [9, 2, 0, 1]
    assert OS.verify_tree(p, q, tokens, parents, 4, [0.0, 0.0, 0.99, 0.99]) == ([0, 2, 3], 0)
    assert OS.verify_tree(p, q, tokens, parents, 2, [0.75, 0.0, 0.0, 0.0]) == ([0], 1)
    assert OS.verify_tree(p, None, tokens, parents, 3, [0.6, 0.0, 0.6, 0.0]) == ([0], 1)   # token 0 refused: only 1 is left
    assert OS.verify_tree(p, None, tokens, parents, 3, [0.6, 0.0, 0.49, 0.0]) == ([0, 2], 1)
    assert OS.verify_tree(p * 0, None, tokens, parents, 1, [0.6, 0, 0, 0]) == ([0], -1)
    assert OS.verify_tree(p, q, tokens, parents, 0, [0.6, 0, 0, 0]) == ([], -1)
