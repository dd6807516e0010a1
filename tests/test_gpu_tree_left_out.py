"""mla_decode_tree without images where the row that its tiles leave out (a node's, with a value
that is not finite) is the first of a warp's 32: the row's block serves the other 31. Bounds as in
test_gpu_tree.py."""
import numpy as np
import pytest

import paper_2609_36760_gb300 as Q
from speculation_cases import KINDS, Cache, queries, trees
from test_gpu_tree import check, run

pytestmark = pytest.mark.gpu
NODES = 9


def seen_by(parents, counts, wrong):
    """[B, T]: nodes whose line has the node wrong[b] of their sequence."""
    seen = np.zeros(parents.shape, bool)
    for b, n in enumerate(counts):
        for t in range(n):
            up = t
            while up >= 0:
                seen[b, t] |= up == wrong[b]
                up = int(parents[b, up])
    return seen


@pytest.mark.parametrize("kind,protect", [(k, False) for k in KINDS] + [(4, True), ("c4r4", True)])
@pytest.mark.parametrize("heads", [1, 3, 7, 16])
@pytest.mark.parametrize("batch", [12, 210])
def test_a_warps_first_row_left_out(kind, protect, heads, batch):
    """Positions 0, 32, .. 352, each as another node; with 210 sequences several tiles a segment or
    CTA, so that such rows are met in a segment's first tile and in later ones."""
    wrong = [b % NODES if b % 12 else 0 for b in range(batch)]
    ctx = [32 * (b % 12) - t for b, t in enumerate(wrong)]
    counts = [NODES - (b % 5 == 4) * min(4, NODES - 1 - t) for b, t in enumerate(wrong)]
    c = Cache(kind, ctx, counts, protect=protect, seed=8)
    q, q_pe = queries(batch, NODES, heads, 8)
    p = trees("any", batch, NODES, 2)
    p[::2, 0::3] = -1  # (some with several roots)
    before = run(c, p, q, q_pe, False)
    check(c, p, q, q_pe, before, False)
    seen = seen_by(p, counts, wrong)
    bad = []
    for b, t in enumerate(wrong):
        row = c.rows[b][ctx[b] + t:ctx[b] + t + 1].clone()
        row[0, 20 + 50 * t] = float("inf")
        bad.append(row)
        if protect:
            c.drafts[b, t] = row[0].cuda()
    if not protect:
        c.write(bad, [a + t for a, t in zip(ctx, wrong)], None)
    out, lse = run(c, p, q, q_pe, False)
    assert Q.read_dev_err(c.err) == 0
    assert seen.any(1).all() and not seen[::2].all(1).any()
    assert np.isnan(out[seen]).all() and np.isnan(lse[seen]).all()
    out[seen], lse[seen] = before[0][seen], before[1][seen]
    check(c, p, q, q_pe, (out, lse), False)
