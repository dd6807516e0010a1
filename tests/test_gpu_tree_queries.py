"""mla_decode_tree's queries that are not finite in fp16: they cost their own row its result, and
no other. Bounds as in test_gpu_tree.py."""
import numpy as np
import pytest

import paper_2609_36760_gb300 as Q
from speculation_cases import Cache, queries, trees
from test_gpu_tree import check, images, run

pytestmark = pytest.mark.gpu


@images
@pytest.mark.parametrize("kind", [4, "bf16"])
@pytest.mark.parametrize("nodes,heads", [(9, 7), (9, 64)])
@pytest.mark.parametrize("value", ["nan", "inf", "-inf", "1e6"])
def test_a_query_that_is_not_finite_is_its_own_rows_alone(kind, nodes, heads, value, images):
    ctx, counts = [200, 0, 2000, 123], [9, 9, 9, 7]
    c = Cache(kind, ctx, counts, seed=8)
    q, q_pe = queries(len(ctx), nodes, heads, 8)
    p = trees("any", len(ctx), nodes, 2)
    before = run(c, p, q, q_pe, images)
    check(c, p, q, q_pe, before, images)
    wrong = np.zeros((len(ctx), nodes, heads), bool)
    bad_q, bad_pe = q.clone(), q_pe.clone()
    for b, t, h in ((0, 3, 0), (0, 8, heads - 1), (1, 0, 2), (2, 5, 5), (3, 6, heads - 1)):
        wrong[b, t, h] = True
        if (b + t) % 2:
            bad_q[b, t, h, 60 * t] = float(value)
        else:
            bad_pe[b, t, h, 7 * t] = float(value)
    out, lse = run(c, p, bad_q, bad_pe, images)
    assert Q.read_dev_err(c.err) == 0
    out[wrong], lse[wrong] = before[0][wrong], before[1][wrong]
    check(c, p, q, q_pe, (out, lse), images)
