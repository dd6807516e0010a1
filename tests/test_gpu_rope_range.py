"""rope_append's rotation at the ends of bf16's range: k' = RN_bf16(RN_f32(a c - b s)),
infinite where that leaves fp32 or a value is infinite, NaN where infinities meet as inf - inf
or 0 x inf, channel by channel."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_36760_gb300 as Q
from test_gpu_rows import Cache

pytestmark = pytest.mark.gpu
LARGEST = 3.3895313892515355e38  # of bf16


@pytest.mark.parametrize("n", [5, 4300])
@pytest.mark.parametrize("interleaved", [False, True])
def test_large_and_infinite_keys(n, interleaved):
    c = Cache("bf16", [n], seed=n)
    rows = c.rows.clone()
    rows[:, 512:] = rows[:, 512:].sign() * LARGEST
    rows[1, 512:] = math.inf
    rows[3, 512:544] = -math.inf
    rows[4, 520] = math.nan
    pool, _, err = c.fresh()
    dev = rows.cuda()
    Q.rope_append(pool, "bf16", dev[:, :512], dev[:, 512:], c.seq.cuda(), c.pos.cuda(), c.table.cuda(), c.cs.cuda(), err,
                  interleaved=interleaved)
    assert Q.read_dev_err(err) == 0
    blocks = c.table[c.seq.long(), (c.pos // 64).long()].long()
    got = pool.cpu().view(torch.bfloat16).view(c.total, 64, 576)[blocks, (c.pos % 64).long()]
    assert torch.equal(got[:, :512], rows[:, :512])
    t, k = c.cs[c.pos.long()].double(), rows[:, 512:].double()
    a, b = (k[:, 0::2], k[:, 1::2]) if interleaved else (k[:, :32], k[:, 32:])
    u, v = a * t[:, :32] - b * t[:, 32:], a * t[:, 32:] + b * t[:, :32]
    want = (torch.stack([u, v], -1).flatten(1) if interleaved else torch.cat([u, v], 1)).float().bfloat16()
    assert bool(want.isinf().any()) and bool(want.isnan().any()) and bool(want.isfinite().any())
    assert torch.equal(got[:, 512:].isnan(), want.isnan())
    assert torch.equal(got[:, 512:].nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
