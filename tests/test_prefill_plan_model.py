"""Bounds that mla_prefill's workspace relies on, from a model of its plan, over random calls and
extreme ones; every key step of every item lies in one part."""
from __future__ import annotations

import random

import pytest

import plan_model as P


def random_call(rnd):
    batch = rnd.choice([1, 1, 2, 5, 40, 300])
    big = rnd.choice([300, 3000, 60000, 3000000]) // (1 if batch < 40 else 20)
    cu_q, cu_kv = [0], [0]
    for _ in range(batch):
        a = rnd.choice([0, 1, 17, 100, 128, 129, 256, 300, 700, 2000])
        cu_q.append(cu_q[-1] + a)
        cu_kv.append(cu_kv[-1] + rnd.choice([0, 1, a, a, a + rnd.randint(0, big), rnd.randint(0, big)]))
    return cu_q, cu_kv, rnd.choice([1, 2, 7, 16, 18, 64, 100, 128, 1024]), rnd.random() < 0.7, rnd.choice([1, 148, 152, 152])


def check(cu_q, cu_kv, heads, causal, sms):
    n_q, n_kv = max(cu_q[-1], 1), cu_kv[-1]
    p = P.plan(cu_q, cu_kv, n_q, n_kv, heads, causal, sms)
    entries = [e for b in p["bundles"] for e in b]
    assert len(entries) <= p["max_items"] + P.SLOTS
    assert p["slots"] <= P.SLOTS and len(p["joins"]) <= P.SHARES
    assert all(0 <= min(k, p["longest"]) >> p["shift"] < p["threads"] for k in p["keys"])
    of = {}
    for e in entries:
        of.setdefault(e["q_row"], []).append(e)
    for b in range(len(cu_q) - 1):
        lq, lk = cu_q[b + 1] - cu_q[b], cu_kv[b + 1] - cu_kv[b]
        for r0 in range(0, lq, P.ROWS):
            it = P.item(cu_q[b], lq, cu_kv[b], lk, r0, causal)
            parts = sorted(of[it["q_row"]], key=lambda e: e["part"])
            assert [e["part"] for e in parts] == list(range(parts[0]["parts"]))
            for name in ("n0", "n1"):  # the parts' key steps, one after the other
                at = it["kv_start"]
                for e in parts:
                    if e[name]:
                        assert e["kv_start"] == at and at < cu_kv[b + 1]
                        assert e["kv_start"] + e["kv_len"] == cu_kv[b + 1]
                    at += e[name] * P.TILE
                assert at == it["kv_start"] + it[name] * P.TILE
    return p


@pytest.mark.parametrize("block", range(6))
def test_parts_and_bounds(block):
    cut = 0
    for seed in range(block * 60, block * 60 + 60):
        cut += bool(check(*random_call(random.Random(seed)))["joins"])
    assert cut > 5


@pytest.mark.parametrize("lk", [4 * 128, 2 ** 20 - 1, 2 ** 26])
@pytest.mark.parametrize("lq,heads", [(1, 1), (128, 1), (129, 1), (256, 1), (300, 1), (5, 150), (5000, 1), (64, 160)])
def test_extreme_calls(lq, lk, heads):
    for causal in (True, False):
        for sms in (1, 152):
            check([0, lq], [0, lk], heads, causal, sms)
