"""mla_decode_tree against the 64-bit oracle on the values that its fp16 tiles hold, with the
least workspace and with room for the context's images (two main kernels).

Bounds, before the first run. Scores are fp32 sums of exact products: their error moves a weight
by less than 2^-15. Weights are rounded to fp16, 2^-11 of each (and by 2^-25 of the largest where
they are that small), in the numerator and in the sum, so that
    |out - exact| <= 2 (2^-11 + 2^-15) sum w |C| + 2^-25 L max|C| + 2^-8 |exact|,
the last for bf16; the sum alone gives lse within 2^-11 + 2^-15 + 2^-25 L. Over the images the sum
takes the weights before their rounding: lse within 2^-14; and where lse is asked for, the scores
are those of the values before their rounding to fp16."""
import numpy as np
import pytest
import torch

import paper_2609_36760_gb300 as Q
from oracle import speculation as OS
from speculation_cases import KINDS, TAU, Cache, queries, trees

pytestmark = pytest.mark.gpu
images = pytest.mark.parametrize("images", [False, True])


def run(c, parents, q, q_pe, images, counts=True, lse=True, max_len=0, fill=float("nan"), size=None):
    B, T, H, _ = q.shape
    out = torch.full((B, T, H, 512), fill, dtype=torch.bfloat16, device="cuda")
    z = torch.full((B, T, H), fill, device="cuda") if lse else None
    size = size or Q.tree_workspace_bytes(B, T, H, (max_len or 64 * c.table.size(1)) if images else 0)
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
    Q.mla_decode_tree(c.pool, c.kind, q.cuda(), q_pe.cuda(), c.table_d, c.lens_d, parents.cuda(), TAU, out, z, ws, c.err,
                      tree_lens=c.counts_d if counts else None, prot=c.prot, draft_rows=c.drafts, max_len=max_len)
    torch.cuda.synchronize()
    return out.cpu().double().numpy(), None if z is None else z.cpu().double().numpy()


def check(c, parents, q, q_pe, got, images, only=None):
    out, lse = got
    for b in range(len(c.lens)) if only is None else only:
        L, x = c.lens[b], c.seen(b)
        key = c.seen(b, exact=True) if images and lse is not None else x
        want, want_lse, mass = OS.attend_tree(q[b].double().numpy(), q_pe[b].double().numpy(), key[:, :512], key[:, 512:],
                                              parents[b].tolist(), c.counts[b], TAU, values=x[:, :512])
        top = np.abs(x[:, :512]).max() if L else 0.0
        tol = 2 * (2.0 ** -11 + 2.0 ** -15) * mass + 2.0 ** -25 * L * top + 2.0 ** -8 * np.abs(want)
        assert (np.abs(out[b] - want) <= tol).all(), (b, np.abs(out[b] - want).max())
        if lse is not None:
            none = np.isinf(want_lse)
            assert np.array_equal(none, np.isneginf(lse[b])), b
            off = np.abs(lse[b][~none] - want_lse[~none])
            assert (off <= (2.0 ** -14 if images else 2.0 ** -11 + 2.0 ** -15 + 2.0 ** -25 * L)).all(), (b, off.max())
            assert (out[b][none] == 0).all()


@images
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nodes,heads,shape", [(1, 16, "chain"), (5, 1, "any"), (8, 16, "any"), (13, 20, "star"),
                                               (64, 1, "any"), (7, 100, "any"), (4, 128, "forest"), (64, 16, "chain")])
def test_trees_over_short_contexts(kind, nodes, heads, shape, images):
    ctx = [0, 1, 63, 64, 65, 127, 128, 190]
    counts = [nodes, 1, nodes, max(1, nodes - 1), nodes, (nodes + 1) // 2, nodes, nodes]
    c = Cache(kind, ctx, counts, seed=nodes)
    q, q_pe = queries(len(ctx), nodes, heads, nodes)
    p = trees(shape, len(ctx), nodes, heads)
    check(c, p, q, q_pe, run(c, p, q, q_pe, images), images)
    assert Q.read_dev_err(c.err) == 0


@images
@pytest.mark.parametrize("kind", [4, 2, "c4r4"])
@pytest.mark.parametrize("nodes,heads", [(1, 16), (9, 20), (26, 128), (64, 64)])
def test_protected_rows_and_the_nodes_own(kind, nodes, heads, images):
    ctx = [0, 3, 4, 5, 100, 127, 131, 132, 133, 300]
    counts = [nodes] * 9 + [max(1, nodes // 2)]
    c = Cache(kind, ctx, counts, protect=True, seed=nodes)
    q, q_pe = queries(len(ctx), nodes, heads, nodes)
    p = trees("any", len(ctx), nodes, heads)
    check(c, p, q, q_pe, run(c, p, q, q_pe, images), images)
    assert Q.read_dev_err(c.err) == 0


@images
@pytest.mark.parametrize("kind,protect", [(4, False), (2, True), ("c4r4", True), ("bf16", False)])
@pytest.mark.parametrize("ctx,nodes,heads", [([5000], 8, 16), ([1900, 700], 16, 128), ([9001], 2, 64), ([2500, 1], 3, 64),
                                             ([4000, 3900, 20], 32, 16), ([70000], 3, 32)])
def test_long_contexts_are_split_and_merged(kind, protect, ctx, nodes, heads, images):
    c = Cache(kind, ctx, [nodes] * len(ctx), protect=protect, seed=nodes)
    q, q_pe = queries(len(ctx), nodes, heads, nodes)
    p = trees("any", len(ctx), nodes, heads)
    check(c, p, q, q_pe, run(c, p, q, q_pe, images, max_len=max(c.lens)), images)
    assert Q.read_dev_err(c.err) == 0


@images
@pytest.mark.parametrize("kind", KINDS)
def test_sequences_without_a_tree_and_padding(kind, images):
    """Counts of zero (an idle place of a batch, with a context and without), padded nodes whose
    parents hold anything."""
    ctx, counts = [70, 0, 200, 5], [0, 0, 3, 2]
    c = Cache(kind, ctx, counts, seed=4)
    q, q_pe = queries(4, 5, 16)
    p = trees("chain", 4, 5)
    p[2, 3:], p[3, 2:] = 99, -7
    check(c, p, q, q_pe, run(c, p, q, q_pe, images), images)
    assert Q.read_dev_err(c.err) == 0


@pytest.mark.parametrize("kind,protect", [(4, False), ("c4r4", True), ("bf16", False)])
@pytest.mark.parametrize("nodes,heads", [(8, 32), (12, 32), (5, 100), (26, 32), (26, 64)])
def test_images_beyond_l2_and_groups_without_nodes(kind, protect, nodes, heads):
    """A table so wide that the images take more than L2: the plan goes group by group (2, 3, 4 and 7
    groups of 128 rows), or some sequences at a time (13), with trees that leave whole groups without a node."""
    ctx = [0, 1, 127, 128, 500, 900, 129, 64, 3, 1300, 256, 700]
    counts = [max(0, nodes - 3 * i) for i in range(len(ctx))]
    counts[5], counts[9] = nodes, nodes
    c = Cache(kind, ctx, counts, protect=protect, seed=nodes, extra=118)
    q, q_pe = queries(len(ctx), nodes, heads, nodes)
    p = trees("any", len(ctx), nodes, heads)
    check(c, p, q, q_pe, run(c, p, q, q_pe, True), True)
    assert Q.read_dev_err(c.err) == 0


@pytest.mark.parametrize("kind,protect", [(4, False), (2, True), ("c4r4", False), ("bf16", False)])
@pytest.mark.parametrize("heads", [4, 32])
def test_lse_where_a_few_keys_have_the_weight(kind, protect, heads):
    """Scores so far apart that the roundings of the cached values do not average out (4e-4 of a score: lse would
    be off by more than it may). With what they left off, a score is off by its 72 steps of accumulation,
    each 2^-24 of a sum below 14: 2^-14."""
    ctx = [300, 1016, 1100, 4000]
    c = Cache(kind, ctx, [8] * 4, protect=protect, seed=1)
    q, q_pe = queries(4, 8, heads, 1, spread=1.0)
    p = trees("any", 4, 8)
    check(c, p, q, q_pe, run(c, p, q, q_pe, True), True)


def test_room_for_some_of_the_sequences():
    """A workspace for the images of one, two or all but one sequence: the others go after them."""
    ctx, nodes = [700, 90, 0, 1300, 257], 9
    for kind, protect, heads in ((4, True, 32), ("bf16", False, 16), (2, False, 4)):
        c = Cache(kind, ctx, [9, 4, 9, 9, 0], protect=protect, seed=3)
        q, q_pe = queries(5, nodes, heads, 3)
        p = trees("any", 5, nodes)
        least, full = (Q.tree_workspace_bytes(5, nodes, heads, n) for n in (0, 64 * c.table.size(1)))
        for share in (1, 2, 4):
            got = run(c, p, q, q_pe, True, size=least + (full - least) * share // 5)
            check(c, p, q, q_pe, got, True)
        assert Q.read_dev_err(c.err) == 0


@images
def test_no_sequence_has_a_tree(images):
    c = Cache(4, [70, 0, 200], [0, 0, 0], seed=4)
    q, q_pe = queries(3, 5, 32)
    out, lse = run(c, trees("chain", 3, 5), q, q_pe, images)
    assert Q.read_dev_err(c.err) == 0 and (out == 0).all() and np.isneginf(lse).all()


@pytest.mark.parametrize("nodes", [1, 5])
def test_more_sequences_than_the_plan_holds_on_chip(nodes):
    B = 4200
    ctx, counts = [(7 * i) % 90 for i in range(B)], [nodes] * B
    c = Cache(4, ctx, counts, seed=2)
    q, q_pe = (x.repeat(70, 1, 1, 1) for x in queries(60, nodes, 16, 2))
    p = trees("any", B, nodes)
    for images in (False, True):
        got = run(c, p, q, q_pe, images)
        check(c, p, q, q_pe, got, images, only=[0, 1, 13, 2000, 4095, 4096, 4199])
    assert Q.read_dev_err(c.err) == 0


@images
def test_scores_that_grow_raise_the_reference(images):
    """Contexts whose scores rise by more than 2^8 from tile to tile, and nodes above them."""
    c = Cache("bf16", [700, 300], [20, 20], seed=2)
    q, q_pe = queries(2, 20, 32, spread=0.02)
    for b in range(2):
        n = c.lens[b]
        c.rows[b][:, 512] = (torch.arange(n) * (90.0 / n)).bfloat16()
    q_pe[..., 0] = 20.0
    c.write(c.rows, [0, 0], None)
    p = trees("any", 2, 20)
    check(c, p, q, q_pe, run(c, p, q, q_pe, images), images)


@images
def test_bad_trees_are_reported_and_see_nothing(images):
    c = Cache(4, [100, 100, 100], [6, 6, 6], seed=3)
    q, q_pe = queries(3, 6, 16)
    p = trees("chain", 3, 6)
    p[1, 2], p[1, 4], p[2, 0] = 2, 0, -2  # a node its own parent, and a root that is not one
    got = run(c, p, q, q_pe, images)
    assert Q.read_dev_err(c.err) == Q.DEVERR_BAD_TREE
    check(c, p, q, q_pe, got, images)
    assert np.isneginf(got[1][1, [2, 3]]).all() and np.isfinite(got[1][1, [0, 1, 4, 5]]).all() and np.isneginf(got[1][2]).all()


@images
@pytest.mark.parametrize("kind,protect,value", [(4, False, "inf"), (2, False, "1e30"), ("c4r4", False, "inf"), (4, True, "nan"),
                                                ("c4r4", True, "1e30"), ("bf16", False, "nan"), ("bf16", False, "inf"),
                                                ("bf16", False, "1e30")])
@pytest.mark.parametrize("nodes,heads", [(9, 7), (9, 64)])
def test_values_that_are_not_finite_reach_the_nodes_that_see_them(kind, protect, value, nodes, heads, images):
    """In rows of nodes: NaN for those that see them, the same results as before for the others."""
    ctx, counts, bad = [200, 0, 5000, 123, 60], [9, 9, 9, 7, 4], [[3], [1, 8], [8], [2, 6], [0]]
    c = Cache(kind, ctx, counts, protect=protect, seed=8)
    q, q_pe = queries(len(ctx), nodes, heads, 8)
    p = trees("any", len(ctx), nodes, 2)
    p[:, 0] = -1
    before = run(c, p, q, q_pe, images)
    check(c, p, q, q_pe, before, images)
    seen = np.zeros((len(ctx), nodes), bool)
    for b, wrong in enumerate(bad):
        for t in range(counts[b]):
            up = t
            while up >= 0:
                seen[b, t] |= up in wrong
                up = int(p[b, up])
        for t in wrong:
            row = c.rows[b][ctx[b] + t:ctx[b] + t + 1].clone()
            row[0, 20 + 69 * t] = float(value)
            if protect:
                c.drafts[b, t] = row[0].cuda()
            else:
                c.write([row if i == b else row[:0] for i in range(len(ctx))], [ctx[b] + t] * len(ctx), None)
    assert not seen.all(1)[[0, 1, 2, 3]].any() and seen.any(1).all()
    out, lse = run(c, p, q, q_pe, images)
    assert Q.read_dev_err(c.err) == 0
    assert np.isnan(out[seen]).all() and np.isnan(lse[seen]).all()
    out[seen], lse[seen] = before[0][seen], before[1][seen]
    check(c, p, q, q_pe, (out, lse), images)


@images
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ctx,at", [(300, 40), (5000, 4700)])
def test_a_context_that_is_not_finite_leaves_rows_without_a_node_zero(kind, ctx, at, images):
    c = Cache(kind, [ctx, 70], [3, 5], seed=8)
    q, q_pe = queries(2, 5, 16, 8)
    p = trees("chain", 2, 5)
    row = c.rows[0][at:at + 1].clone()
    row[0, 7] = float("inf")
    c.write([row, row[:0]], [at, 0], None)
    out, lse = run(c, p, q, q_pe, images)
    assert np.isnan(out[0, :3]).any(-1).all()
    assert (out[0, 3:] == 0).all() and np.isneginf(lse[0, 3:]).all()
    check(c, p, q, q_pe, (out, lse), images, only=[1])


@pytest.mark.parametrize("images", [False, True])
def test_queries_behind_the_last_node_are_not_used(images):
    c = Cache(4, [300, 0, 70], [3, 5, 0], seed=8)
    q, q_pe = queries(3, 5, 16, 8)
    p = trees("chain", 3, 5)
    want = run(c, p, q, q_pe, images)
    q[0, 3:], q_pe[0, 4:], q[2] = float("nan"), float("inf"), float("nan")
    got = run(c, p, q, q_pe, images)
    assert all(np.array_equal(x, y) for x, y in zip(got, want))
    check(c, p, q, q_pe, got, images, only=[1])


@images
@pytest.mark.parametrize("count", [-1, 7, 1 << 30])
def test_bad_counts_leave_the_sequence_without_rows(count, images):
    c = Cache(4, [100, 3], [6, 6], seed=3)
    q, q_pe = queries(2, 6, 16)
    p = trees("chain", 2, 6)
    c.counts_d[0] = count
    out, lse = run(c, p, q, q_pe, images)
    assert Q.read_dev_err(c.err) == Q.DEVERR_BAD_TREE
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all()
    check(c, p, q, q_pe, (out, lse), images, only=[1])


@images
def test_more_nodes_than_tokens_and_bad_lengths(images):
    c = Cache(4, [0, 30], [6, 6], seed=3)
    q, q_pe = queries(2, 6, 16)
    p = trees("chain", 2, 6)
    c.lens_d[0] = 5
    out, lse = run(c, p, q, q_pe, images, counts=False)
    assert Q.read_dev_err(c.err) == Q.DEVERR_BAD_TREE and (out[0] == 0).all() and np.isneginf(lse[0]).all()
    check(c, p, q, q_pe, (out, lse), images, only=[1])
    for bad in (-1, 1 << 20):
        c.err.zero_()
        c.lens_d[0] = bad
        out, lse = run(c, p, q, q_pe, images)
        assert Q.read_dev_err(c.err) & Q.DEVERR_BAD_POSITION and (out[0] == 0).all() and np.isneginf(lse[0]).all()
        check(c, p, q, q_pe, (out, lse), images, only=[1])


@images
def test_bad_blocks_are_reported(images):
    c = Cache(4, [100, 40], [3, 3])
    q, q_pe = queries(2, 3, 16)
    p = trees("chain", 2, 3)
    c.table_d[0, 0] = 1 << 20
    out, lse = run(c, p, q, q_pe, images)
    assert Q.read_dev_err(c.err) == Q.DEVERR_BAD_BLOCK and np.isfinite(out).all()
    check(c, p, q, q_pe, (out, lse), images, only=[1])


def test_a_chain_is_the_multi_token_decode():
    c = Cache(4, [500, 64, 1000], [4, 4, 4], seed=9)
    q, q_pe = queries(3, 4, 32)
    out, lse = run(c, trees("chain", 3, 4), q, q_pe, False, counts=False)
    want = torch.empty((3, 4, 32, 512), device="cuda")
    z = torch.empty((3, 4, 32), device="cuda")
    Q.mla_decode_multi(c.pool, 4, q.cuda(), q_pe.cuda(), c.table_d, c.lens_d, TAU, want, z, Q.workspace_for(3, 128), c.err)
    torch.cuda.synchronize()
    assert np.array_equal(out, want.bfloat16().double().cpu().numpy())
    assert np.array_equal(lse, z.double().cpu().numpy())


@images
def test_without_lse_and_with_the_least_workspace(images):
    c = Cache("c4r4", [300, 40], [9, 9], protect=True)
    q, q_pe = queries(2, 9, 16)
    p = trees("any", 2, 9)
    for lse in (False, True):
        check(c, p, q, q_pe, run(c, p, q, q_pe, images, lse=lse), images)
    need = Q.tree_workspace_bytes(2, 9, 16)
    assert np.array_equal(run(c, p, q, q_pe, images, size=need)[0], run(c, p, q, q_pe, False)[0])
    with pytest.raises(Q.QmlaError, match="workspace"):
        run(c, p, q, q_pe, images, size=need - 1)


@images
def test_lengths_beyond_the_bound_are_bad(images):
    c = Cache(4, [300, 40], [9, 9])
    q, q_pe = queries(2, 9, 16)
    p = trees("any", 2, 9)
    out, lse = run(c, p, q, q_pe, images, max_len=308)
    assert Q.read_dev_err(c.err) == Q.DEVERR_BAD_POSITION and (out[0] == 0).all() and np.isneginf(lse[0]).all()
    check(c, p, q, q_pe, (out, lse), images, only=[1])


@images
def test_two_captured_steps_of_one_workspace(images):
    """Two graphs that share a workspace, replayed in turn with new lengths and trees in place."""
    c = Cache(4, [2000, 700], [8, 8], seed=5)
    q, q_pe = (x.cuda() for x in queries(2, 8, 64))
    p = trees("any", 2, 8).cuda()
    ws = torch.empty(Q.tree_workspace_bytes(2, 8, 64, 64 * c.table.size(1) if images else 0), dtype=torch.uint8, device="cuda")
    outs = [torch.empty((2, 8, 64, 512), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens = [c.lens_d.clone(), (c.lens_d - 3).contiguous()]

    def call(i):
        Q.mla_decode_tree(c.pool, 4, q, q_pe, c.table_d, lens[i], p, TAU, outs[i], None, ws, c.err)

    call(0), call(1)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o.fill_(float("nan"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    lens[0].copy_(lens[1])
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[1])


def test_on_another_stream_than_the_current_one():
    c = Cache("bf16", [900], [5], seed=6)
    q, q_pe = queries(1, 5, 16)
    p = trees("any", 1, 5)
    want = run(c, p, q, q_pe, False)
    s = torch.cuda.Stream()
    out = torch.zeros((1, 5, 16, 512), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(Q.tree_workspace_bytes(1, 5, 16), dtype=torch.uint8, device="cuda")
    args = (q.cuda(), q_pe.cuda(), c.table_d, c.lens_d, p.cuda())
    s.wait_stream(torch.cuda.current_stream())
    Q.mla_decode_tree(c.pool, "bf16", *args, TAU, out, None, ws, c.err, stream=s)
    s.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want[0])
