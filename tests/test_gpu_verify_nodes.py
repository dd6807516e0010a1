"""tree_verify's node 0: the committed token, kept whatever its parent says, which is -1 or reported."""
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
