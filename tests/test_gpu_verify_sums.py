"""tree_verify's sums where their rounding shows: nothing or next to nothing left of a row."""
import pytest
import torch

import paper_2609_36760_gb300 as Q
from speculation_cases import trees
from test_gpu_verify import check, run

pytestmark = pytest.mark.gpu


def refused_rows(batch, vocab, drafts, dtype, seed):
    """Rows of a half in all, on `drafts` tokens of unlike size, and a tree that drafts each of them. Random
    numbers of almost 1 refuse all: a token has at most half of what is not refused yet."""
    g = torch.Generator().manual_seed(seed)
    target = torch.zeros(batch, drafts + 1, vocab, dtype=dtype)
    tokens = torch.zeros(batch, drafts + 1, dtype=torch.int32)
    for b in range(batch):
        at = torch.randperm(vocab, generator=g)[:drafts]
        p = torch.exp(-20 * torch.rand(drafts, generator=g))
        target[b, 0, at] = (p / (2.02 * p.sum())).to(dtype)
        tokens[b, 1:] = at.int()
    u = torch.full((batch, drafts + 1), 1 - 2.0 ** -24)
    u[:, 0] = torch.rand(batch, generator=g)
    return target, tokens, trees("star", batch, drafts + 1), u


@pytest.mark.parametrize("vocab,drafts", [(64, 10), (64, 30), (70, 63), (1000, 3), (1001, 40), (32000, 20), (40001, 63)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nothing_is_left_when_every_token_was_refused(vocab, drafts, dtype):
    target, tokens, parents, u = refused_rows(100, vocab, drafts, dtype, vocab)
    path, kept, nxt, err = run(target, None, tokens, parents, u)
    assert err == Q.DEVERR_BAD_PROBS
    assert (kept == 1).all() and (nxt == -1).all() and (path[:, 1:] == -1).all()
    for b in range(40):  # each alone: as many CTAs a row as there are, and its own report
        got = run(target[b:b + 1], None, tokens[b:b + 1], parents[b:b + 1], u[b:b + 1])
        assert got[3] == Q.DEVERR_BAD_PROBS and got[2][0] == -1, b


@pytest.mark.parametrize("vocab,drafts", [(70, 30), (1001, 40), (32000, 20), (40001, 62)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_token_that_is_left_is_drawn_however_small(vocab, drafts, dtype):
    target, tokens, parents, u = refused_rows(100, vocab, drafts, dtype, vocab + 1)
    left = []
    for b in range(100):
        free = (target[b, 0] == 0).nonzero()[:, 0]
        left.append(int(free[(37 * b) % len(free)]))
        target[b, 0, left[-1]] = 2.0 ** -90
    got = run(target, None, tokens, parents, u)
    assert got[3] == 0 and (got[1] == 1).all() and got[2].tolist() == left
    check(target, None, tokens, parents, u, got)
