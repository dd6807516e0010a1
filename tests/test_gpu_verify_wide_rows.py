"""tree_verify over rows on 16-byte borders, whose values are read eight (bf16) or four (float32)
at a time, against the 64-bit oracle and against the same rows off such borders."""
import numpy as np
import pytest
import torch

from speculation_cases import distributions, drafted, trees
from test_gpu_verify import check, run, uniforms

pytestmark = pytest.mark.gpu
dtypes = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


def placed(x, lead, end):
    """The same rows `lead` elements behind a 16-byte border, padded by `end` elements of another value."""
    B, T, V = x.shape
    wide = torch.full((B, T, lead + V + end), 0.5, dtype=x.dtype, device="cuda")
    wide[..., lead:lead + V] = x.cuda()
    return wide[..., lead:lead + V]


@dtypes
@pytest.mark.parametrize("vocab", [8, 16, 64, 72, 1000, 4104, 32000])
@pytest.mark.parametrize("shape,nodes", [("chain", 5), ("star", 12), ("any", 33)])
@pytest.mark.parametrize("certain", [False, True])
def test_walks(dtype, vocab, shape, nodes, certain):
    B = 6 if vocab > 4200 else 24
    target, draft = distributions(B, nodes, vocab, vocab + 1, dtype=dtype)
    parents = trees(shape, B, nodes, 1)
    tokens = drafted(draft.float(), parents, 1)
    u = uniforms(B, nodes, nodes + 1)
    u[::2, 1:] = u[::2, 1:].sqrt()  # more refusals: sums of what two and more left
    d = None if certain else draft
    got = run(target, d, tokens, parents, u)
    assert got[3] == 0
    check(target, d, tokens, parents, u, got)


@dtypes
@pytest.mark.parametrize("vocab,batch", [(131072, 3), (128256, 5)])
@pytest.mark.parametrize("certain", [False, True])
def test_large_vocabularies(dtype, vocab, batch, certain):
    target, draft = distributions(batch, 4, vocab, 3, dtype=dtype)
    parents = trees("star", batch, 4)
    tokens = drafted(draft.float(), parents, 4)
    u = uniforms(batch, 4, 8)
    u[:, 1:] = 1 - (1 - u[:, 1:]) / 8  # nearly all are refused
    d = None if certain else draft
    got = run(target, d, tokens, parents, u)
    assert got[3] == 0
    check(target, d, tokens, parents, u, got)


@dtypes
@pytest.mark.parametrize("certain", [False, True])
def test_one_cta_a_row(dtype, certain):
    """So many sequences that each row has one: the longest pieces."""
    B, vocab = 320, 9000
    target, draft = distributions(4, 3, vocab, 5, dtype=dtype)
    target, draft = target.repeat(80, 1, 1), draft.repeat(80, 1, 1)
    parents = trees("star", B, 3)
    tokens = drafted(draft.float(), parents, 2)
    u = uniforms(B, 3, 4)
    u[:, 1:] = u[:, 1:].sqrt()
    d = None if certain else draft
    got = run(target, d, tokens, parents, u)
    assert got[3] == 0
    check(target, d, tokens, parents, u, got)


@dtypes
@pytest.mark.parametrize("certain", [False, True])
def test_on_and_off_the_borders(dtype, certain):
    """Padded rows on borders, one of both off its border, a stride that is no multiple, an odd vocabulary."""
    B, nodes = 16, 9
    for vocab in (2000, 2001):
        target, draft = distributions(B, nodes, vocab, 7, dtype=dtype)
        parents = trees("any", B, nodes, 2)
        tokens, u = drafted(draft.float(), parents, 5), uniforms(B, nodes, 6)
        want = run(target, None if certain else draft, tokens, parents, u)
        check(target, None if certain else draft, tokens, parents, u, want)
        for tl, te, dl, de in ((0, 8, 0, 16), (8, 8, 16, 0), (1, 7, 0, 8), (0, 8, 3, 5), (0, 1, 0, 0), (0, 0, 0, 3)):
            got = run(placed(target, tl, te), None if certain else placed(draft, dl, de), tokens, parents, u)
            assert got[3] == 0
            assert all(np.array_equal(a, b) for a, b in zip(want[:3], got[:3])), (vocab, tl, te, dl, de)
