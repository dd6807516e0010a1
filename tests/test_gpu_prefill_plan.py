"""The list that mla_prefill's plan leaves in the workspace against the model of the plan: the
same items and parts, the longest bundles first. (The list is the library's own; nothing outside
of it relies on its form.)"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2609_36760_gb300 as Q
import plan_model as P

pytestmark = pytest.mark.gpu
TAU = 1.0 / math.sqrt(192.0)
FIELDS = ["q_row", "rows", "kv_start", "kv_len", "vis0", "step", "n0", "n1", "first", "bundle", "head", "dealt", "part",
          "parts", "slot", "unused"]


def cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(int).tolist()


def listed(lq, lk, heads, causal):
    """(the model's plan, the entries of the list, the joins) of a call of these lengths."""
    n_q, n_kv, batch = sum(lq), sum(lk), len(lq)
    q = torch.zeros(n_q, heads, 192, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(n_kv, heads, 128, dtype=torch.bfloat16, device="cuda")
    pe = torch.zeros(n_kv, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(n_q, heads, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(Q.prefill_workspace_bytes(batch, n_q), dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    Q.mla_prefill(q, kv, kv, pe, i32(cu(lq)), i32(cu(lk)), TAU, out, None, ws, err, causal=causal)
    assert Q.read_dev_err(err) == 0
    p = P.plan(cu(lq), cu(lk), n_q, n_kv, heads, causal, Q.num_sms())
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    words = ws.cpu().numpy().view(np.int32)
    entries, cut = int(words[0]), int(words[2])
    items = up(256 + 4 * (batch + 1)) // 4
    join = items + 16 * (p["max_items"] + P.SLOTS)
    return (p, [dict(zip(FIELDS, words[items + 16 * i:items + 16 * i + 16].tolist())) for i in range(entries)],
            [tuple(words[join + 4 * i:join + 4 * i + 4].tolist()) for i in range(cut)])


# Lengths of queries and keys, heads: bundles of four whose last item has one tile; the same with
# keys in parts; items that the SMs' fair share alone would cut up, into more parts than SMs, and
# that the weighing leaves whole (the longest is the second of its bundle); single items.
CALLS = {
    "one_tile_last": ([1100, 1300, 700, 90, 1124], [1100, 1300, 700, 900, 2300], 128),
    "ragged": ([5, 0, 300, 128, 1, 77, 257, 1500, 2000], [5, 9, 300, 500, 0, 78, 1000, 1500, 4000], 100),
    "cut_in_bundles": ([1] * 300 + [1124], [1] * 300 + [30000], 4),
    "whole_after_all": ([1] * 64 + [1124], [1] * 64 + [60000], 20),
    "few_rows": ([50], [9050], 16),
    "two_long": ([512, 3], [16896, 5000], 16),
    "one_head": ([600, 1], [40000, 20000], 1),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", CALLS)
def test_the_list_is_the_models(name, causal):
    lq, lk, heads = CALLS[name]
    p, got, joins = listed(lq, lk, heads, causal)
    keys = ["q_row", "rows", "kv_start", "kv_len", "vis0", "step", "n0", "n1", "dealt", "part", "parts"]
    whole = lambda e: tuple(e[k] for k in keys)  # noqa: E731
    at, lengths, want = 0, [], {tuple(whole(e) for e in b): min(k, p["longest"]) >> p["shift"]
                                for b, k in zip(p["bundles"], p["keys"])}
    while at < len(got):
        n = got[at]["bundle"]
        bundle = got[at:at + n]
        assert all(e["first"] == at and e["bundle"] == n and e["head"] == 0 for e in bundle)
        lengths.append(want.pop(tuple(whole(e) for e in bundle)))
        at += n
    assert not want
    assert lengths == sorted(lengths, reverse=True)
    # joins: the items cut up, each with a place of its own for heads x parts results
    assert sorted((q, r, n) for q, r, _, n in joins) == sorted(p["joins"])
    slots = {e["q_row"]: e["slot"] for e in got if e["parts"] > 1}
    assert all(slots[q] == s for q, _, s, _ in joins)
    ends = sorted((s, s + n * heads) for _, _, s, n in joins)
    assert all(b <= c for (_, b), (c, _) in zip(ends, ends[1:])) and (not ends or ends[-1][1] == p["slots"] <= P.SLOTS)
