"""tree_verify's sums where their rounding shows: nothing left of a row, next to nothing left, and
a row of millions of tokens whose draw lies next to a border."""
import numpy as np
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


def exact_sum(x):
    """Sum of float32 values in units of 2^-149."""
    mantissa, exponent = np.frexp(x.astype(np.float64))
    whole = (mantissa * (1 << 24)).astype(np.int64)
    return sum(int(whole[exponent == e].sum()) << int(e - 24 + 149) for e in np.unique(exponent[x > 0]))


def parts(whole):
    """The same as float32 values that add up to it."""
    out = []
    while whole:
        low = max(whole.bit_length() - 24, 0)
        top = whole >> low
        out.append(np.float32(np.ldexp(float(top), low - 149)))
        whole -= top << low
    return out


@pytest.mark.parametrize("batch", [1, 320])
def test_a_border_in_a_row_of_millions(batch):
    """The number 0.5 on a row of two equal halves and a token between them of 2^-42 of a half: that token
    is drawn if the sums before it and in all are within 2^-43 of a half. The first half is
    millions of tokens, the other a few, so that errors of the sums do not cancel. (An emulation of a lane's sums
    in fp32 pairs is 2^-46 off for 2^20 tokens a warp, which is one CTA a row, if the pairs are kept
    normal, and 2^-41 if they are not.)"""
    vocab = 1 << 24
    first = vocab - 1000
    z = np.exp(2.5 * np.random.default_rng(7).standard_normal(first))
    t = np.zeros(vocab, np.float32)
    t[:first] = z / (2 * z.sum())
    half = exact_sum(t[:first])
    t[first] = np.float32(2.0 ** -42 * np.ldexp(float(half), -149))
    rest = parts(half)
    t[first + 500:first + 500 + len(rest)] = rest
    assert exact_sum(t[first + 1:]) == half
    shared = torch.from_numpy(t).cuda().view(1, 1, vocab).expand(batch, 1, vocab)
    none = torch.full((batch, 1), -1, dtype=torch.int32)
    got = run(shared, None, torch.zeros_like(none), none, torch.full((batch, 1), 0.5))
    assert got[3] == 0 and got[2].tolist() == [first] * batch
