"""tree_verify against the 64-bit oracle: whole numbers, all equal. The oracle normalises its
residuals at every step and sums in another order, so its borders are a few 2^-50 off; the
random numbers are on 24 bits, so a decision within that of a border is met once in 10^9."""
import numpy as np
import pytest
import torch

import paper_2609_36760_gb300 as Q
from oracle import speculation as OS
from speculation_cases import distributions, drafted, trees

pytestmark = pytest.mark.gpu


def run(target, draft, tokens, parents, u, counts=None, err=None):
    B, T, _ = target.shape
    path = torch.full((B, T), 77, dtype=torch.int32, device="cuda")
    kept, nxt = (torch.full((B,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    err = torch.zeros(1, dtype=torch.int32, device="cuda") if err is None else err
    Q.tree_verify(dev(target), dev(draft), dev(tokens), dev(parents), dev(u), path, kept, nxt, err, tree_lens=dev(counts))
    return path.cpu().numpy(), kept.cpu().numpy(), nxt.cpu().numpy(), Q.read_dev_err(err)


def check(target, draft, tokens, parents, u, got, counts=None, only=None):
    B, T, _ = target.shape
    for b in range(B) if only is None else only:
        n = T if counts is None else int(counts[b])
        path, nxt = OS.verify_tree(target[b].double().numpy(), None if draft is None else draft[b].double().numpy(),
                                   tokens[b].tolist(), parents[b].tolist(), n, u[b].double().numpy())
        assert got[1][b] == len(path) and got[0][b].tolist() == path + [-1] * (T - len(path)) and got[2][b] == nxt, b


def uniforms(batch, nodes, seed=0):
    return torch.rand(batch, nodes, generator=torch.Generator().manual_seed(seed + 31))


@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 1000, 4097, 32001])
@pytest.mark.parametrize("shape,nodes", [("chain", 1), ("chain", 8), ("star", 12), ("any", 33), ("any", 64)])
@pytest.mark.parametrize("certain", [False, True])
def test_walks(vocab, shape, nodes, certain):
    B = 12 if vocab > 4000 else 40
    target, draft = distributions(B, nodes, vocab, vocab)
    parents = trees(shape, B, nodes, 1)
    tokens = drafted(draft, parents, 1)
    u = uniforms(B, nodes, nodes)
    if certain:
        draft = None
    got = run(target, draft, tokens, parents, u)
    assert got[3] == 0
    check(target, draft, tokens, parents, u, got)


@pytest.mark.parametrize("vocab", [50001, 131072])
@pytest.mark.parametrize("certain", [False, True])
def test_large_vocabularies(vocab, certain):
    target, draft = distributions(6, 5, vocab, 3)
    parents = trees("star", 6, 5)
    tokens = drafted(draft, parents, 4)
    u = uniforms(6, 5, 8)
    u[:, 1:] = u[:, 1:].sqrt()  # more refusals
    d = None if certain else draft
    got = run(target, d, tokens, parents, u)
    check(target, d, tokens, parents, u, got)


@pytest.mark.parametrize("apart", [0.0, 0.01, 3.0])
def test_drafts_near_and_far(apart):
    """Equal distributions (everything is accepted), nearly equal ones (residuals of cancelled
    differences) and unlike ones (refusal after refusal)."""
    target, draft = distributions(64, 9, 777, 1, apart)
    parents = trees("star", 64, 9)
    tokens = drafted(draft, parents, 2)
    u = uniforms(64, 9, 3)
    got = run(target, draft, tokens, parents, u)
    check(target, draft, tokens, parents, u, got)
    if apart == 0.0:
        assert (got[1] == 2).all()


@pytest.mark.parametrize("certain", [False, True])
def test_bf16_probabilities(certain):
    target, draft = distributions(24, 16, 5003, 7, dtype=torch.bfloat16)
    parents = trees("any", 24, 16, 2)
    tokens = drafted(draft.float(), parents, 5)
    u = uniforms(24, 16, 6)
    d = None if certain else draft
    check(target, d, tokens, parents, u, run(target, d, tokens, parents, u))


def test_strides_and_rows_off_any_boundary():
    target, draft = distributions(7, 6, 1001, 9)
    parents = trees("any", 7, 6, 2)
    tokens, u = drafted(draft, parents, 5), uniforms(7, 6, 6)
    want = run(target, draft, tokens, parents, u)
    wide = torch.full((7, 9, 1003), 0.5, device="cuda")
    wide[:, 1:7, 2:1003] = target.cuda()
    turned = draft.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    got = run(wide[:, 1:7, 2:], turned, tokens, parents, u)
    assert all(np.array_equal(a, b) for a, b in zip(want[:3], got[:3]))
    shared = target[:1].cuda().expand(7, -1, -1)  # one row for all sequences
    check(target[:1].expand(7, -1, -1), draft, tokens, parents, u, run(shared, draft, tokens, parents, u))


def test_counts_and_what_lies_behind_them():
    counts = torch.tensor([0, 1, 3, 6, 0], dtype=torch.int32)
    target, draft = distributions(5, 6, 300, 9)
    parents = trees("any", 5, 6, 2)
    tokens, u = drafted(draft, parents, 5), uniforms(5, 6, 6)
    parents[2, 3:], tokens[2, 3:] = 1000, -5
    got = run(target, draft, tokens, parents, u, counts)
    assert got[3] == 0
    check(target, draft, tokens, parents, u, got, counts)
    for bad in (-1, 7):
        counts[3] = bad
        got = run(target, draft, tokens, parents, u, counts)
        assert got[3] == Q.DEVERR_BAD_TREE and got[1][3] == 0 and got[2][3] == -1 and (got[0][3] == -1).all()
        check(target, draft, tokens, parents, u, got, counts, only=[0, 1, 2, 4])


def test_bad_nodes_are_passed_over():
    target, draft = distributions(30, 6, 100, 9)
    parents = trees("star", 30, 6)
    tokens, u = drafted(draft, parents, 5), uniforms(30, 6, 6)
    tokens[:, 1], tokens[:, 3], parents[:, 2], parents[:, 4] = 100, -1, 2, 5
    got = run(target, draft, tokens, parents, u)
    assert got[3] == Q.DEVERR_BAD_TREE
    check(target, draft, tokens, parents, u, got)


def test_the_edges_of_the_random_numbers():
    """0, the largest below 1, and what is no number of that range; rows with empty beginnings and ends."""
    vals = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, float("inf"), float("nan"), 0.5])
    p = torch.zeros(8, 1, 640)
    p[:, 0, 100:108] = 0.125
    got = run(p, None, torch.zeros(8, 1, dtype=torch.int32), torch.full((8, 1), -1, dtype=torch.int32), vals[:, None])
    assert got[2].tolist() == [100, 107, 107, 107, 100, 107, 100, 104]
    q = torch.full((8, 1, 640), 1 / 1024)  # sums of whole steps: every border is exact
    got = run(q, None, torch.zeros(8, 1, dtype=torch.int32), torch.full((8, 1), -1, dtype=torch.int32), torch.arange(8)[:, None] / 8.0)
    assert got[2].tolist() == [80 * i for i in range(8)]


def test_rows_with_nothing_to_draw_from():
    for value, certain in ((0.0, True), (float("nan"), True), (float("inf"), True), (float("nan"), False)):
        target = torch.full((2, 2, 50), 0.02)
        target[0] = value
        draft = None if certain else torch.full((2, 2, 50), 0.02)
        tokens, parents = torch.tensor([[0, 3]] * 2).int(), torch.tensor([[-1, 0]] * 2).int()
        u = torch.full((2, 2), 0.999)
        u[1, 1] = 0.0
        got = run(target, draft, tokens, parents, u)
        assert got[3] == Q.DEVERR_BAD_PROBS and got[2][0] == -1 and 0 <= got[2][1] < 50
    # negative values count as nothing
    target = torch.full((1, 1, 50), -1.0)
    target[0, 0, 17] = 0.25
    assert run(target, None, torch.zeros(1, 1).int(), torch.full((1, 1), -1).int(), torch.full((1, 1), 0.9))[2].tolist() == [17]


def test_refused_tokens_are_not_drawn_and_a_token_twice():
    target = torch.full((16, 4, 4), 0.25)
    tokens = torch.tensor([[0, 2, 2, 1]] * 16).int()
    parents = trees("star", 16, 4)
    u = uniforms(16, 4, 3)
    u[:, 1:] = 0.97
    got = run(target, None, tokens, parents, u)
    check(target, None, tokens, parents, u, got)
    assert set(got[2][got[1] == 1]) <= {0, 3}


def test_captured_and_replayed_with_new_inputs():
    target, draft = distributions(9, 7, 3001, 9)
    parents = trees("any", 9, 7, 2)
    tokens = drafted(draft, parents, 5)
    us = [uniforms(9, 7, s) for s in (1, 2)]
    d = [x.cuda() for x in (target, draft, tokens, parents, us[0].clone())]
    path = torch.zeros((9, 7), dtype=torch.int32, device="cuda")
    kept, nxt = torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")
    Q.tree_verify(*d, path, kept, nxt, None)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Q.tree_verify(*d, path, kept, nxt, None)
    for u in (us[1], us[0]):
        d[4].copy_(u)
        g.replay()
        torch.cuda.synchronize()
        check(target, draft, tokens, parents, u, (path.cpu().numpy(), kept.cpu().numpy(), nxt.cpu().numpy()))
