"""mla_prefill's bundles (planned calls of many pairs put four items of a sequence side by side,
head by head) and the two forms of the fused writer at their border. The bounds are those of
test_gpu_prefill.py; bytes are compared as in test_gpu_rows.py."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_36760_gb300 as Q
import plan_model as P
from test_gpu_prefill import Prompt
from test_gpu_rows import KINDS, Cache, check_append

pytestmark = pytest.mark.gpu


def offsets(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def planned(p, causal):
    """The model's plan of this call, rows and keys of padding among those given."""
    return P.plan(offsets(p.lq), offsets(p.lk), p.q.size(0), p.kv.size(0), p.H, causal, Q.num_sms())


@pytest.mark.parametrize("heads", [100, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_batches_with_a_plan(heads, causal):
    lq, lk = [5, 0, 300, 128, 1, 77, 257, 600], [5, 9, 300, 500, 0, 78, 1000, 700]
    p = Prompt(lq, lk, heads, seed=heads, pad_q=700, pad_kv=3000)
    plan = planned(p, causal)
    assert plan["size"] == 4 and max(len(b) for b in plan["bundles"]) > 1
    p.kv[sum(lk):], p.rows[sum(lk):] = math.nan, math.inf
    assert p.run(causal) == 0
    p.check(causal)


@pytest.mark.parametrize("n,m", [(1100, 1100), (1124, 2400), (1300, 1290), (2300, 2300)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts_of_five_to_nine_items(n, m, causal):
    """Bundles of four and of what is left, the last item with one tile or two; fewer keys than queries."""
    p = Prompt([n, 40], [m, 2100], 128, seed=n, pad_q=1500)
    plan = planned(p, causal)
    assert plan["size"] == 4 and sorted(len(b) for b in plan["bundles"])[-1] == 4
    assert p.run(causal) == 0
    p.check(causal)


@pytest.mark.parametrize("n,heads", [(1124, 4), (600, 7)])
@pytest.mark.parametrize("causal", [True, False])
def test_bundles_that_hold_items_cut_into_parts(n, heads, causal):
    short = 300
    p = Prompt([1] * short + [n], [1] * short + [30000], heads, seed=n)
    plan = planned(p, causal)
    assert plan["size"] == 4 and plan["joins"] and max(len(b) for b in plan["bundles"]) > 4
    assert p.run(causal) == 0
    p.check(causal, sequences={0, 1, 150, short - 1, short})


def test_bundles_give_what_single_items_give():
    """The same sequence among so many rows that bundles are made, and alone: the same bits (nothing is cut up)."""
    n = 1300
    a = Prompt([n], [n], 32, seed=3, pad_kv=2000)
    b = Prompt([n], [n], 32, seed=3, pad_q=10000, pad_kv=2000)
    b.q[:n], b.kv[:], b.rows[:] = a.q, a.kv, a.rows
    assert planned(a, True)["size"] == 1 and planned(b, True)["size"] == 4
    assert not planned(a, True)["joins"] and not planned(b, True)["joins"]
    assert a.run() == 0 and b.run() == 0
    a.check()
    assert torch.equal(a.out, b.out[:n]) and torch.equal(a.lse, b.lse[:n])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("norm,weight", [(True, False), (False, False)])
@pytest.mark.parametrize("n", [3040, 3041, 4256, 4257, 4299])
def test_the_writer_of_many_tokens_without_norm_or_weights(kind, norm, weight, n):
    c = Cache(kind, [n - 700, 700], protect=kind in (2, "c4r4"), seed=n)
    check_append(c, norm, weight, n % 2 == 0, torch.arange(n), strided=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("offset", [2, 8])
def test_many_tokens_off_a_16_byte_boundary(kind, offset):
    """Rows in 4-byte pieces (2 elements off) take the form of few tokens at any length."""
    c = Cache(kind, [4300], protect=kind == 4, seed=offset)
    check_append(c, True, True, False, torch.arange(4300), strided=True, offset=offset)
