"""tree_verify's nodes: node 0, the committed token, is kept whatever its parent says, which is -1 or reported; drafts of
infinite probability or none are taken and refused as the numbers compare."""
import numpy as np
import pytest
import torch

import paper_2609_36760_gb300 as Q
from speculation_cases import distributions, drafted, trees
from test_gpu_verify import check, run, uniforms

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("parent", [0, 1, 5, -2, 1 << 30, -(1 << 31)])
@pytest.mark.parametrize("vocab", [100, 20001])
@pytest.mark.parametrize("certain", [False, True])
def test_a_parent_of_node_0_is_reported(parent, vocab, certain):
    target, draft = distributions(6, 6, vocab, 9)
    parents = trees("any", 6, 6)
    tokens, u = drafted(draft, parents, 5), uniforms(6, 6, 6)
    d = None if certain else draft
    want = run(target, d, tokens, parents, u)
    assert want[3] == 0
    parents[4, 0] = parent
    got = run(target, d, tokens, parents, u)
    assert got[3] == Q.DEVERR_BAD_TREE
    assert all(np.array_equal(a, b) for a, b in zip(want[:3], got[:3]))
    check(target, d, tokens, parents, u, got)
    # without a tree there is no node 0
    counts = torch.tensor([6, 6, 6, 6, 0, 6], dtype=torch.int32)
    got = run(target, d, tokens, parents, u, counts)
    assert got[3] == 0 and got[1][4] == 0


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("vocab", [100, 20001])
def test_an_infinite_probability_of_a_draft_accepts_it(vocab, certain):
    """More than anything that it is compared with; a NaN is not, and leaves nothing to draw from."""
    target, draft = distributions(6, 3, vocab, 9)
    parents = trees("star", 6, 3)
    tokens, u = drafted(draft, parents, 5), uniforms(6, 3, 6)
    tokens[:, 1], tokens[:, 2] = 7, 11
    u[:, 1] = 0.9
    target[:2, 0, 7], target[2:4, 0, 7] = float("inf"), float("nan")
    d = None if certain else draft
    path, kept, nxt, err = run(target, d, tokens, parents, u)
    assert (kept[:2] == 2).all() and (path[:2, 1] == 1).all() and ((0 <= nxt[:2]) & (nxt[:2] < vocab)).all()
    assert (path[2:4, 1] != 1).all()
    check(target, d, tokens, parents, u, (path, kept, nxt), only=[4, 5])
    if not certain:
        assert err == Q.DEVERR_BAD_PROBS and (kept[2:4] == 1).all() and (nxt[2:4] == -1).all()
