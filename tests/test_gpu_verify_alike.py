"""tree_verify where the draft is nearly the target: what refusals leave is made of units of the
probabilities' last places, and every number of it is a difference of those."""
import numpy as np
import pytest
import torch

import paper_2609_36760_gb300 as Q
from speculation_cases import trees
from test_gpu_verify import check, run

pytestmark = pytest.mark.gpu


def alike(batch, children, vocab, steps, dtype, seed, empty=0.0):
    """A draft q, the target up to `steps` units of q's last place beside it (0 in a share `empty` of the
    tokens), and a star of children that are refused by the largest number below 1: their tokens have p < q."""
    g = torch.Generator().manual_seed(seed)
    q = torch.softmax(0.5 * torch.randn(batch, 1, vocab, generator=g), -1).to(dtype)
    unit = q.float() * torch.finfo(dtype).eps
    p = (q.float() + unit * torch.randint(-steps, steps + 1, q.shape, generator=g)).to(dtype)
    if empty:
        p[torch.rand(p.shape, generator=g) < empty] = 0
    less = (p.double() <= q.double() * (1 - 2.0 ** -24))[:, 0]
    tokens = torch.zeros(batch, children + 1, dtype=torch.int32)
    tokens[:, 1:] = torch.multinomial(less.float(), children, replacement=True, generator=g).int()
    u = torch.full((batch, children + 1), 1 - 2.0 ** -24)
    u[:, 0] = torch.rand(batch, generator=g)
    rows = lambda x: x.expand(-1, children + 1, -1).contiguous()  # noqa: E731
    return rows(p), rows(q), tokens, trees("star", batch, children + 1), u


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("children", [1, 2, 3, 9])
@pytest.mark.parametrize("vocab", [40, 1001, 20000, 60045])
@pytest.mark.parametrize("steps,empty", [(1, 0.0), (3, 0.0), (3, 0.5)])
def test_refusals_of_a_draft_that_is_nearly_the_target(dtype, children, vocab, steps, empty):
    batch = 60 if vocab < 2000 else 12
    target, draft, tokens, parents, u = alike(batch, children, vocab, steps, dtype, vocab + children + steps, empty)
    got = run(target, draft, tokens, parents, u)
    assert got[3] == 0 and (got[1] == 1).all()
    check(target, draft, tokens, parents, u, got)


@pytest.mark.parametrize("children", [2, 5])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_drafts_value_that_is_no_number_leaves_nothing_of_its_token(children, value):
    """An infinity is more than any probability; a NaN counts as one."""
    target, draft, tokens, parents, u = alike(30, children, 500, 3, torch.float32, 5)
    want = run(target, draft, tokens, parents, u)
    used = set(tokens[:, 1:].flatten().tolist()) | set(want[2].tolist())
    at = next(v for v in range(500) if v not in used)
    draft[..., at] = value
    got = run(target, draft, tokens, parents, u)
    target[..., at] = 0
    draft[..., at] = 0.5
    assert got[3] == 0
    check(target, draft, tokens, parents, u, got)
