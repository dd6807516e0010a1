"""Caches, trees and probabilities for the tests of the tree operators."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2609_36760_gb300 as Q

TAU = 1.0 / math.sqrt(192.0)
KINDS = [4, 2, "c4r4", "bf16"]
WIDTH = {4: 20736, 2: 12544, "c4r4": 20480, "bf16": 73728}
POISON = 0xAB


def trees(shape: str, batch: int, nodes: int, seed: int = 0) -> torch.Tensor:
    g = torch.Generator().manual_seed(seed)
    t = torch.arange(nodes).expand(batch, -1)
    if shape == "chain":
        p = t - 1
    elif shape == "star":
        p = torch.where(t == 0, -1, 0)
    elif shape == "forest":  # every third node a root
        p = torch.where(t % 3 == 0, -1, t - 1)
    else:
        p = torch.where(t == 0, -1, (torch.rand(batch, nodes, generator=g) * t).long().clamp_max(nodes))
    return p.int().contiguous()


def tile_values(x: torch.Tensor, kind, exact: bool = False) -> np.ndarray:
    """What the attention's fp16 tiles hold of rows x [n, 576]: RN_f16(s (q - z)), or the bf16 values;
    exact: before that rounding."""
    if kind == "bf16":
        return (x if exact else x.half()).double().numpy()
    out = []
    for a, b, content in ((0, 512, True), (512, 576, False)):
        g = x[:, a:b].float().reshape(x.size(0), (b - a) // 64, 64)
        m = 3.0 if kind == 2 and content else 15.0
        lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
        s = ((hi - lo).clamp_min(1e-8).double() / m).float()
        if kind == "c4r4":
            s = s.bfloat16().float() if content else s
            z = (-lo.double() / s.double()).float().round().clamp(0, m)
            q = ((g.double() / s.double()).float() + z).round().clamp(0, m)
        else:
            s = s.half().float().clamp(2.0 ** -24, 65504.0)
            z = (-lo.double() / s.double()).round().clamp(0, m).float()
            q = (g.double() / s.double() + z).round().clamp(0, m).float()
        out.append((s * (q - z)).flatten(1))
    out = torch.cat(out, 1)
    return (out if exact else out.half()).double().numpy()


class Cache:
    """Sequences of ctx[b] context tokens and counts[b] nodes in a poisoned pool, written by the
    library's plain writers (checked against the oracle elsewhere)."""

    def __init__(self, kind, ctx, counts, protect=False, seed=0, extra=1):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.ctx, self.counts, self.protect = kind, ctx, counts, protect
        self.lens = [a + b for a, b in zip(ctx, counts)]
        nblk = [max(1, -(-n // 64)) for n in self.lens]
        perm = torch.randperm(sum(nblk) + 2, generator=g).int()
        self.table = torch.full((len(ctx), max(nblk) + extra), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(nblk):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.pool = torch.full((sum(nblk) + 2, WIDTH[kind]), POISON, dtype=torch.uint8, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.prot = torch.full((len(ctx), 132, 576), float("nan"), dtype=torch.bfloat16, device="cuda") if protect else None
        self.drafts = torch.full((len(ctx), 64, 576), float("nan"), dtype=torch.bfloat16, device="cuda") if protect else None
        gain = torch.exp(0.5 * torch.randn(512, generator=g))
        gain[:2] *= 8
        self.rows = [torch.cat([torch.randn(n, 512, generator=g) * gain, torch.randn(n, 64, generator=g)], 1).bfloat16()
                     for n in self.lens]
        self.table_d = self.table.cuda()
        self.write([x[:c] for x, c in zip(self.rows, ctx)], [0] * len(ctx), ctx)
        self.write([x[c:] for x, c in zip(self.rows, ctx)], ctx, None)
        if protect:
            for b, (c, n) in enumerate(zip(ctx, counts)):
                self.drafts[b, :n] = self.rows[b][c:].cuda()
        self.lens_d = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.counts_d = torch.tensor(counts, dtype=torch.int32, device="cuda")

    def write(self, rows, first, lens_after):
        """Appends rows[b] from position first[b] on; with lens_after the protection rows too."""
        x = torch.cat(rows).cuda()
        if not x.size(0):
            return
        seq = torch.cat([torch.full((len(r),), b, dtype=torch.int32) for b, r in enumerate(rows)]).cuda()
        pos = torch.cat([torch.arange(f, f + len(r), dtype=torch.int32) for f, r in zip(first, rows)]).cuda()
        lat, kpe = x[:, :512].contiguous(), x[:, 512:].contiguous()
        prot = self.prot if lens_after is not None else None
        after = None if prot is None else torch.tensor(lens_after, dtype=torch.int32, device="cuda")
        if self.kind == "bf16":
            Q.bf16_append(self.pool, lat, kpe, seq, pos, self.table_d, self.err)
        elif self.kind == "c4r4":
            Q.quant_append_c4r4(self.pool, lat, kpe, seq, pos, self.table_d, self.err, seq_lens=after, prot=prot)
        elif prot is not None:
            Q.quant_append_protected(self.pool, self.kind, lat, kpe, seq, pos, self.table_d, after, prot, self.err)
        else:
            Q.quant_append(self.pool, self.kind, lat, kpe, seq, pos, self.table_d, self.err)

    def seen(self, b, exact=False) -> np.ndarray:
        """Rows of sequence b as attention sees them, in its tiles or before their rounding."""
        x = tile_values(self.rows[b], self.kind, exact)
        if self.protect:
            c, own = self.ctx[b], (self.rows[b] if exact else self.rows[b].half()).double().numpy()
            for p in range(c):
                if p < 4 or p >= c - 128:
                    x[p] = own[p]
            x[c:] = own[c:]
        return x


def queries(batch, nodes, heads, seed=0, spread=0.5):
    g = torch.Generator().manual_seed(seed + 77)
    return ((torch.randn(batch, nodes, heads, 512, generator=g) * spread).bfloat16(),
            torch.randn(batch, nodes, heads, 64, generator=g).bfloat16())


def distributions(batch, nodes, vocab, seed=0, apart=0.7, dtype=torch.float32):
    """(target, draft) probabilities, the tokens of each tree drawn from the draft later on."""
    g = torch.Generator().manual_seed(seed + 5)
    d = 2.5 * torch.randn(batch, nodes, vocab, generator=g)
    t = d + apart * torch.randn(batch, nodes, vocab, generator=g)
    return torch.softmax(t, -1).to(dtype), torch.softmax(d, -1).to(dtype)


def drafted(draft, parents, seed=0):
    """A token for every node, drawn from its parent's row."""
    g = torch.Generator().manual_seed(seed + 9)
    B, T, V = draft.shape
    at = parents.long().clamp(0, T - 1)
    rows = torch.gather(draft.double(), 1, at[..., None].expand(B, T, V)).reshape(B * T, V)
    return torch.multinomial(rows, 1, generator=g).view(B, T).int()
