"""Offsets that decrease or overlap: which sequences mla_prefill computes, in short calls (which
have no plan) and long ones alike. The results of those are what the same sequence gives alone,
and no row of the others is touched. (Values of a sequence do not depend on its neighbours, but
its keys can be cut into parts in one call and not in the other; the sequences here are short.)"""
from __future__ import annotations

import math
import random

import pytest
import torch

import paper_2609_36760_gb300 as Q

pytestmark = pytest.mark.gpu
TAU = 1.0 / math.sqrt(192.0)


def kept(cu_q, cu_kv, n_q, n_kv):
    """The sequences that are computed: offsets in order and in range, queries behind the ends of all
    earlier sequences whose offsets are."""
    out, reach = [], 0
    for b in range(len(cu_q) - 1):
        if 0 <= cu_q[b] <= cu_q[b + 1] <= n_q and 0 <= cu_kv[b] <= cu_kv[b + 1] <= n_kv:
            if cu_q[b] >= reach:
                out.append(b)
            reach = max(reach, cu_q[b + 1])
    return out


def call(t, cu_q, cu_kv, out, lse, causal, n_kv):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(Q.prefill_workspace_bytes(len(cu_q) - 1, out.size(0)), dtype=torch.uint8, device="cuda")
    kv, pe = t["kv"][:n_kv], t["pe"][:n_kv]
    Q.mla_prefill(t["q"], kv[..., :128], kv[..., 128:], pe, i32(cu_q), i32(cu_kv), TAU, out, lse, ws, err, causal=causal)
    return Q.read_dev_err(err)


def check(cu_q, cu_kv, n_q, n_kv, heads=2, causal=True, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    t = {"q": rnd(n_q, heads, 192), "kv": rnd(max(n_kv, 9000), heads, 256), "pe": rnd(max(n_kv, 9000), 64)}
    want = torch.full((n_q, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    want_lse = torch.full((n_q, heads), 7.0, device="cuda")
    good = kept(cu_q, cu_kv, n_q, n_kv)
    for b in good:
        assert call(t, cu_q[b:b + 2], cu_kv[b:b + 2], want, want_lse, causal, n_kv) == 0
    out, lse = torch.full_like(want, 7.0), torch.full_like(want_lse, 7.0)
    err = call(t, cu_q, cu_kv, out, lse, causal, n_kv)
    assert err == (0 if len(good) == len(cu_q) - 1 else Q.DEVERR_BAD_OFFSETS)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    return good


@pytest.mark.parametrize("n_kv", [700, 9000])
@pytest.mark.parametrize("cu_q,good", [
    ([0, 300, 100, 400, 350, 600, 700], [0, 5]),  # 100 .. 400 begins inside 0 .. 300, 350 .. 600 inside that
    ([0, 50, 40, 180, 260], [0, 3]),
    ([50, 10, 60, 60, 700], [1, 2, 3]),  # (nothing before 10 .. 60 has good offsets)
    ([0, 701, 50, 100, 700], [2, 3]),  # (an end beyond n_q reaches nowhere)
    ([-5, 20, 300, 260, 700], [1]),
])
def test_which_sequences_are_left_out(cu_q, good, n_kv):
    cu_kv = [min(40 * b, 400) for b in range(len(cu_q))]
    assert check(cu_q, cu_kv, 700, n_kv) == good


@pytest.mark.parametrize("n", [260, 2560])
@pytest.mark.parametrize("batch", [8, 64, 70])
def test_the_same_rows_many_times(n, batch):
    """0, n, 0, n, ..: half of the sequences go over all rows; together they would have several
    times the items that the workspace has room for. The first is computed, the others are not."""
    cu = [n * (b & 1) for b in range(batch + 1)]
    assert check(cu, cu, n, n) == [0]


@pytest.mark.parametrize("batch,n_kv", [(20, 2000), (64, 2000), (64, 9000), (90, 9000), (1030, 9000), (2500, 9000)])
def test_random_steps_backwards(batch, n_kv):
    """Offsets that mostly grow, in one and in several rounds of the plan's block."""
    rnd = random.Random(batch)
    n_q, cu_q, cu_kv = 4 * batch + 50, [0], [0]
    for b in range(batch):
        step = rnd.choice([0, 1, 2, 3, 5])
        if rnd.random() < 4 / batch or b in (31, 32, 1023, 1024):
            step = -rnd.randint(1, 9)
        cu_q.append(min(n_q, max(0, cu_q[-1] + step)))
        cu_kv.append(min(n_kv, max(0, cu_kv[-1] + (-3 if rnd.random() < 1 / batch else rnd.choice([0, 1, 2])))))
    good = kept(cu_q, cu_kv, n_q, n_kv)
    assert 0 < len(good) < batch
    g = torch.Generator(device="cuda").manual_seed(batch)
    rnd_t = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    t = {"q": rnd_t(n_q, 1, 192), "kv": rnd_t(n_kv, 1, 256), "pe": rnd_t(n_kv, 64)}
    out = torch.full((n_q, 1, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_q, 1), 7.0, device="cuda")
    assert call(t, cu_q, cu_kv, out, lse, True, n_kv) == Q.DEVERR_BAD_OFFSETS
    # The good ones alone, in one call whose other sequences are empty.
    only_q, only_kv = [], []
    for b in good:
        only_q.append((cu_q[b], cu_q[b + 1]))
        only_kv.append((cu_kv[b], cu_kv[b + 1]))
    want, want_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    for (a, z), (c, d) in zip(only_q, only_kv):
        if z > a:
            want[a:z] = 0
            want_lse[a:z] = -math.inf
    touched = (out[:, 0, 0] != 7) | (lse[:, 0] != 7)
    assert torch.equal(touched, want_lse[:, 0] != 7)
    some = [i for i, (a, z) in enumerate(only_q) if z > a]
    for i in random.Random(1).sample(some, min(40, len(some))):
        assert call(t, list(only_q[i]), list(only_kv[i]), want, want_lse, True, n_kv) == 0
        a, z = only_q[i]
        assert torch.equal(out[a:z], want[a:z]) and torch.equal(lse[a:z], want_lse[a:z])
