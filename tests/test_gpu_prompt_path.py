"""The prompt operators as a serving program uses them, chunk by chunk: rope_append,
cache_read, the up-projection (a plain matrix product), rope_query and mla_prefill;
and the decode of the last token in the absorbed form over the same cache.

Tolerances. mla_prefill sees the up-projected keys and values rounded to bf16, so the
reference takes those values too and the bounds of test_gpu_prefill.py apply:
|out - exact| <= (2^-8 + 2 e + 2^-18) sum w |v| + 2^-8 |exact|. The absorbed decode
rounds in other places: its query to bf16, its tiles and weights to fp16 (2^-11), where
the expanded form has rounded keys and values (bf16). A rounding of 2^-8 of every term of
a score moves it by at most 2^-8 of the sum of the terms' sizes. With d that bound for
the terms of both forms together (the fp16 tiles add an eighth), the two scores of a key
differ by at most 1.125 d, the normalised weights by a factor exp(2.25 d), and
|expanded - absorbed| <= (exp(2.25 d) - 1 + 2^-7) sum w |v| + 2^-9 sum w |c| |W_v| + 2^-8 |out|
(values and weights in bf16; tiles and weights in fp16; the result in bf16)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_36760_gb300 as Q

pytestmark = pytest.mark.gpu
TAU = 1.0 / math.sqrt(192.0)
WIDTH = {4: 20736, 2: 12544, "c4r4": 20480, "bf16": 73728}


def table_of(n):
    freq = 10000.0 ** (-torch.arange(32, dtype=torch.float64, device="cuda") / 32.0)
    ang = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([torch.cos(ang), torch.sin(ang)], 1).float()


@pytest.mark.parametrize("kind,protect", [(4, True), (2, False), ("c4r4", True), ("bf16", False)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_chunked_prompts_and_the_decode_behind_them(kind, protect, interleaved):
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    H, chunks = 6, [[150, 1, 64], [131, 300, 0], [1, 1, 1]]  # the last one: a decode step's tokens
    B, ends = 3, [282, 302, 65]
    blocks = [-(-n // 64) for n in ends]
    table = torch.full((B, max(blocks)), -1, dtype=torch.int32, device="cuda")
    perm = torch.randperm(sum(blocks), generator=torch.Generator().manual_seed(1)).int().cuda()
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = perm[at:at + n]
        at += n
    pool = torch.zeros(sum(blocks), WIDTH[kind], dtype=torch.uint8, device="cuda")
    prot = torch.zeros(B, 132, 576, dtype=torch.bfloat16, device="cuda") if protect else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    cs, weight = table_of(400), (1 + 0.2 * rnd(512)).bfloat16()
    w_kv = (rnd(512, H * 256) / math.sqrt(512)).bfloat16()
    ws = torch.empty(Q.prefill_workspace_bytes(B, 512), dtype=torch.uint8, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    done = [0, 0, 0]
    for new in chunks:
        total = [d + n for d, n in zip(done, new)]
        lens, n = i32(total), sum(new)
        seq = i32([b for b in range(B) for _ in range(new[b])])
        pos = i32([done[b] + t for b in range(B) for t in range(new[b])])
        proj, q = (2 * rnd(n, 576)).bfloat16(), rnd(n, H, 192).bfloat16()
        extra = dict(seq_lens=lens, prot=prot) if protect else {}
        Q.rope_append(pool, kind, proj[:, :512], proj[:, 512:], seq, pos, table, cs, err, norm_weight=weight,
                      interleaved=interleaved, **extra)
        whole_seq = i32([b for b in range(B) for _ in range(total[b])])
        whole_pos = i32([t for b in range(B) for t in range(total[b])])
        rows = torch.empty(sum(total), 576, dtype=torch.bfloat16, device="cuda")
        Q.cache_read(pool, kind, whole_seq, whole_pos, table, rows, err, **extra)
        kv = (rows[:, :512] @ w_kv).view(-1, H, 256)
        Q.rope_query(q[..., 128:], pos, cs, q[..., 128:], err, interleaved=interleaved)
        out = torch.empty(n, H, 128, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(n, H, device="cuda")
        cu = lambda x: i32([sum(x[:i]) for i in range(B + 1)])  # noqa: E731
        Q.mla_prefill(q, kv[..., :128], kv[..., 128:], rows[:, 512:], cu(new), cu(total), TAU, out, lse, ws, err)
        assert Q.read_dev_err(err) == 0
        aq = ak = 0
        for a, m in zip(new, total):
            if a:
                k = torch.cat([kv[ak:ak + m, :, :128], rows[ak:ak + m, None, 512:].expand(m, H, 64)], -1).double()
                s = TAU * torch.einsum("qhc,khc->hqk", q[aq:aq + a].double(), k)
                e = 192 * 2.0 ** -24 * float(TAU * torch.einsum("qhc,khc->hqk", q[aq:aq + a].double().abs(), k.abs()).max())
                late = torch.arange(m, device="cuda")[None] > torch.arange(a, device="cuda")[:, None] + m - a
                p = torch.softmax(s.masked_fill(late, -math.inf), -1)
                v = kv[ak:ak + m, :, 128:].double()
                want, size = torch.einsum("hqk,khc->qhc", p, v), torch.einsum("hqk,khc->qhc", p, v.abs())
                gap = (out[aq:aq + a].double() - want).abs()
                assert bool((gap <= (2.0 ** -8 + 2 * e + 2.0 ** -18) * size + 2.0 ** -8 * want.abs()).all())
            aq, ak = aq + a, ak + m
        done = total
    assert done == ends
    # The same tokens by the decode, which attends to the cached latents themselves.
    w_k, w_v = w_kv.view(512, H, 256)[..., :128].double(), w_kv.view(512, H, 256)[..., 128:].double()
    q_lat = torch.einsum("bhc,dhc->bhd", q[..., :128].double(), w_k).bfloat16().contiguous()
    q_pe = q[..., 128:].contiguous()
    o = torch.empty(B, H, 512, device="cuda")
    dlse = torch.empty(B, H, device="cuda")
    Q.mla_decode_ex(pool, kind, q_lat, q_pe, table, i32(ends), TAU, o, dlse, Q.workspace_for(B, H), err, prot=prot)
    assert Q.read_dev_err(err) == 0
    absorbed = torch.einsum("bhd,dhc->bhc", o.double(), w_v)
    ak = 0
    for b, m in enumerate(ends):
        c, pe = rows[ak:ak + m, :512].double(), rows[ak:ak + m, 512:].double()
        key = torch.einsum("kd,dhc->khc", c, w_k)
        val = torch.einsum("kd,dhc->khc", c, w_v)
        qc, qr = q[b, :, :128].double(), q[b, :, 128:].double()
        s = TAU * (torch.einsum("hc,khc->hk", qc, key) + torch.einsum("hc,kc->hk", qr, pe))
        # channels by which either form's rounded scores are made
        near = TAU * (torch.einsum("hc,khc->hk", qc.abs(), key.abs())
                      + torch.einsum("hd,kd->hk", torch.einsum("hc,dhc->hd", qc, w_k).abs(), c.abs())
                      + 2 * torch.einsum("hc,kc->hk", qr.abs(), pe.abs()))
        d = 2.0 ** -8 * float(near.max())
        p = torch.softmax(s, -1)
        size = torch.einsum("hk,khc->hc", p, val.abs())
        # (the decode's weights and tiles: fp16; summed over the latents before W_v)
        wide = torch.einsum("hd,dhc->hc", torch.einsum("hk,kd->hd", p, c.abs()), w_v.abs())
        bound = (math.exp(2.25 * d) - 1 + 2.0 ** -7) * size + 2.0 ** -9 * wide + 2.0 ** -8 * absorbed[b].abs()
        gap = (out[b].double() - absorbed[b]).abs()
        assert bool((gap <= bound).all()), (b, float((gap - bound).max()))
        assert float((lse[b].double() - dlse[b].double()).abs().max()) <= 1.25 * d
        ak += m
