"""rope_append, cache_read and rope_query against plain 64-bit forms.

The writer's and the reader's results are defined as RN_bf16(RN_f32(exact)), which
64-bit arithmetic rounded through fp32 gives except where it lands within 2^-46 of a
border; so rows and cache bytes are compared for equality. The bytes of a transformed
row are those that the plain writers (checked against the oracle elsewhere) store for it.

A rotated query a c + b s is a rounded product, an FMA (2^-24 of its own result each)
and a rounding to bf16 (2^-8): |got - exact| <= 2^-8 |exact| + 2^-22 (|a c| + |b s|)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_36760_gb300 as Q

pytestmark = pytest.mark.gpu
POISON = 0xAB
KINDS = [4, 2, "c4r4", "bf16"]
WIDTH = {4: 20736, 2: 12544, "c4r4": 20480, "bf16": 73728}


def table_of(rope_len):
    freq = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32.0)
    ang = torch.arange(rope_len, dtype=torch.float64)[:, None] * freq
    return torch.cat([torch.cos(ang), torch.sin(ang)], 1).float()


def rotated(x, cs, pos, interleaved):
    t = cs[pos.long()].double().view(-1, *([1] * (x.dim() - 2)), 64)
    c, s, x = t[..., :32], t[..., 32:], x.double()
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :32], x[..., 32:])
    u, v = a * c - b * s, a * s + b * c
    return (torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)).float().bfloat16()


def turned_right(got, x, cs, pos, interleaved):
    """Whether got is x turned, within the bound above."""
    t = cs[pos.long()].double().view(-1, *([1] * (x.dim() - 2)), 64)
    c, s, x = t[..., :32], t[..., 32:], x.double()
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :32], x[..., 32:])
    g = got.double()
    ga, gb = (g[..., 0::2], g[..., 1::2]) if interleaved else (g[..., :32], g[..., 32:])
    return all(bool(((u - (p + q)).abs() <= 2.0 ** -8 * (p + q).abs() + 2.0 ** -22 * (p.abs() + q.abs())).all())
               for u, p, q in ((ga, a * c, -b * s), (gb, a * s, b * c)))


def normed(x, w, eps):
    d = x.double()
    return (d * (1.0 if w is None else w.double()) / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)).float().bfloat16()


class Cache:
    """Sequences of the given lengths in a poisoned pool, their tokens drawn on the host."""

    def __init__(self, kind, lens, protect=False, seed=0, spare=2):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.lens, self.protect = kind, lens, protect
        nblk = [max(1, -(-n // 64)) for n in lens]
        total = sum(nblk) + spare
        perm = torch.randperm(total, generator=g).int()
        self.table = torch.full((len(lens), max(nblk) + 1), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(nblk):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.total = total
        self.seq = torch.cat([torch.full((n,), b) for b, n in enumerate(lens)]).int()
        self.pos = torch.cat([torch.arange(n) for n in lens]).int()
        gain = torch.exp(0.5 * torch.randn(512, generator=g))
        gain[:2] *= 8
        n = sum(lens)
        self.rows = torch.cat([torch.randn(n, 512, generator=g) * gain * 3, torch.randn(n, 64, generator=g)], 1).bfloat16()
        self.weight = (1 + 0.2 * torch.randn(512, generator=g)).bfloat16()
        self.cs = table_of(max(lens) + 3)

    def fresh(self):
        pool = torch.full((self.total, WIDTH[self.kind]), POISON, dtype=torch.uint8, device="cuda")
        prot = (torch.full((len(self.lens), 132, 576), -1.5, dtype=torch.bfloat16, device="cuda") if self.protect else None)
        return pool, prot, torch.zeros(1, dtype=torch.int32, device="cuda")

    def plain(self, x, lens_dev, pick):
        """Bytes that the plain writers leave for the transformed rows x."""
        pool, prot, err = self.fresh()
        lat, kpe = x[:, :512].contiguous().cuda(), x[:, 512:].contiguous().cuda()
        seq, pos, table = self.seq[pick].cuda(), self.pos[pick].cuda(), self.table.cuda()
        if self.kind == "bf16":
            Q.bf16_append(pool, lat, kpe, seq, pos, table, err)
        elif self.kind == "c4r4":
            Q.quant_append_c4r4(pool, lat, kpe, seq, pos, table, err, seq_lens=lens_dev if self.protect else None, prot=prot)
        elif self.protect:
            Q.quant_append_protected(pool, self.kind, lat, kpe, seq, pos, table, lens_dev, prot, err)
        else:
            Q.quant_append(pool, self.kind, lat, kpe, seq, pos, table, err)
        assert Q.read_dev_err(err) == 0
        return pool, prot


def check_append(c, norm, weight, interleaved, pick, strided, offset=0):
    """offset: elements by which the rows are moved off a 16-byte boundary."""
    lens_dev = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    rows = c.rows[pick]
    x = torch.cat([normed(rows[:, :512], c.weight if weight else None, 1e-6) if norm else rows[:, :512],
                   rotated(rows[:, 512:], c.cs, c.pos[pick], interleaved)], 1)
    want, want_prot = c.plain(x, lens_dev, pick)
    if strided:
        wide = torch.zeros(rows.size(0), 600 + offset, dtype=torch.bfloat16, device="cuda")
        wide[:, offset:576 + offset] = rows.cuda()
        lat, kpe = wide[:, offset:512 + offset], wide[:, 512 + offset:576 + offset]
    else:
        lat, kpe = rows[:, :512].contiguous().cuda(), rows[:, 512:].contiguous().cuda()
    pool, prot, err = c.fresh()
    Q.rope_append(pool, c.kind, lat, kpe, c.seq[pick].cuda(), c.pos[pick].cuda(), c.table.cuda(), c.cs.cuda(), err,
                  norm_weight=c.weight.cuda() if weight else None, norm=norm, interleaved=interleaved,
                  seq_lens=lens_dev if c.protect else None, prot=prot)
    assert Q.read_dev_err(err) == 0
    if c.kind == "c4r4":  # (the page's padding is never written)
        assert torch.equal(pool[:, :20288], want[:, :20288])
    assert torch.equal(pool, want)
    if c.protect:
        assert torch.equal(prot, want_prot)
    return pool, prot, x, lens_dev


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm,weight", [(True, True), (True, False), (False, False)])
def test_rope_append_equals_the_plain_writers(kind, interleaved, norm, weight):
    c = Cache(kind, [1, 130, 64, 77])
    check_append(c, norm, weight, interleaved, torch.arange(sum(c.lens)), strided=interleaved)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("offset", [2, 4, 8])
def test_rope_append_rows_off_a_16_byte_boundary(kind, offset):
    c = Cache(kind, [37, 3], seed=offset)
    check_append(c, True, True, False, torch.arange(40), strided=True, offset=offset)


@pytest.mark.parametrize("kind", KINDS)
def test_rope_append_single_tokens_and_long_calls(kind):
    c = Cache(kind, [8300, 1], seed=3)  # four tokens a lane from 8,192 on
    check_append(c, True, True, True, torch.arange(8301), strided=True)
    for n in (1, 2, 5):
        check_append(c, True, True, False, torch.arange(8301)[torch.linspace(0, 8300, n).long()], strided=False)


@pytest.mark.parametrize("kind", [4, 2, "c4r4"])
@pytest.mark.parametrize("lens", [[3, 131, 132, 133], [300, 1, 4, 129], [9000]])
def test_protected_write_and_read(kind, lens):
    c = Cache(kind, lens, protect=True, seed=5)
    pool, prot, x, lens_dev = check_append(c, True, True, False, torch.arange(sum(lens)), strided=True)
    got = torch.full((sum(lens), 576), 7.0, dtype=torch.bfloat16, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    Q.cache_read(pool, kind, c.seq.cuda(), c.pos.cuda(), c.table.cuda(), got, err, seq_lens=lens_dev, prot=prot)
    packed = torch.empty_like(got)
    Q.cache_read(pool, kind, c.seq.cuda(), c.pos.cuda(), c.table.cuda(), packed, err)
    assert Q.read_dev_err(err) == 0
    end = torch.tensor(lens)[c.seq.long()]
    kept = (c.pos < 4) | (c.pos >= end - 128)
    assert torch.equal(got.cpu()[kept], x[kept])
    assert torch.equal(got.cpu()[~kept], packed.cpu()[~kept])
    # a position behind its sequence has no protection row: refused, its row left as it was
    last = torch.tensor([lens[0]], dtype=torch.int32, device="cuda")
    one = torch.full((1, 576), 7.0, dtype=torch.bfloat16, device="cuda")
    Q.cache_read(pool, kind, None, last, c.table.cuda()[:1], one, err, seq_lens=lens_dev[:1].clone(), prot=prot[:1])
    assert Q.read_dev_err(err) == Q.DEVERR_BAD_POSITION and bool((one == 7).all())


def dequantised(x, kind):
    """s (q - z) in fp32 (products of a stored scale and a small integer), rounded to bf16."""
    out = []
    for a, b, content in ((0, 512, True), (512, 576, False)):
        g = x[:, a:b].float().reshape(x.size(0), -1, 64)
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
        out.append((s * (q - z)).reshape(x.size(0), -1))
    return torch.cat(out, 1).bfloat16()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 3, 4, 331, 8300])
@pytest.mark.parametrize("stride", [576, 584])
def test_cache_read_values(kind, n, stride):
    c = Cache(kind, [max(1, n - n // 3), n // 3] if n > 2 else [n], seed=n)
    pool, prot, x, _ = check_append(c, True, True, False, torch.arange(sum(c.lens)), strided=False)
    wide = torch.full((n, stride), 7.0, dtype=torch.bfloat16, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    order = torch.randperm(n, generator=torch.Generator().manual_seed(1))
    Q.cache_read(pool, kind, c.seq[order].cuda(), c.pos[order].cuda(), c.table.cuda(), wide[:, :576], err)
    assert Q.read_dev_err(err) == 0
    want = x if kind == "bf16" else dequantised(x, kind)
    assert torch.equal(wide[:, :576].cpu(), want[order])
    assert bool((wide[:, 576:] == 7).all())


@pytest.mark.parametrize("kind", KINDS)
def test_bad_tokens_are_left_out(kind):
    """Bad sequence ids, positions, angles and blocks: reported, nothing written for them."""
    c = Cache(kind, [70, 70], seed=9)
    table = c.table.clone()
    table[1, 1] = c.total + 5
    seq = torch.tensor([0, 2, -1, 0, 0, 1, 0, 1], dtype=torch.int32)
    pos = torch.tensor([5, 5, 5, -1, 64 * 3, 65, 72, 6], dtype=torch.int32)  # the table has 3 blocks, the angles 73
    good = torch.tensor([0, 7])
    bits = Q.DEVERR_BAD_SEQ | Q.DEVERR_BAD_POSITION | Q.DEVERR_BAD_BLOCK
    pool, _, err = c.fresh()
    rows = c.rows[:8].cuda()
    cs = c.cs[:72].contiguous()
    Q.rope_append(pool, kind, rows[:, :512], rows[:, 512:], seq.cuda(), pos.cuda(), table.cuda(), cs.cuda(), err, norm=True)
    assert Q.read_dev_err(err) == bits
    want, _, err2 = c.fresh()
    Q.rope_append(want, kind, rows[:, :512][good.cuda()], rows[:, 512:][good.cuda()], seq[good].cuda(), pos[good].cuda(),
                  table.cuda(), cs.cuda(), err2, norm=True)
    assert Q.read_dev_err(err2) == 0 and torch.equal(pool, want)
    assert int((pool != POISON).any(1).sum()) == 2
    err.zero_()
    out = torch.full((8, 576), 7.0, dtype=torch.bfloat16, device="cuda")
    pos[6] = 6
    Q.cache_read(pool, kind, seq.cuda(), pos.cuda(), table.cuda(), out, err)
    assert Q.read_dev_err(err) == bits
    assert bool((out[[1, 2, 3, 4, 5]] == 7).all()) and not bool((out[[0, 7]] == 7).all())


@pytest.mark.parametrize("n,heads", [(1, 1), (1, 16), (7, 20), (33, 128), (1000, 3)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_query(n, heads, interleaved):
    g = torch.Generator().manual_seed(n)
    q = torch.randn(n, heads, 192, generator=g).bfloat16()
    pos = torch.randint(0, 5000, (n,), generator=g).int()
    cs = table_of(5000)
    right = lambda got: turned_right(got.cpu(), q[..., 128:], cs, pos, interleaved)  # noqa: E731
    qd, err = q.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty(n, heads, 64, dtype=torch.bfloat16, device="cuda")
    Q.rope_query(qd[..., 128:], pos.cuda(), cs.cuda(), out, err, interleaved=interleaved)
    assert right(out)
    # heads outermost, then in place: the content part stays as it was
    turned = torch.empty(heads, n, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    Q.rope_query(qd[..., 128:], pos.cuda(), cs.cuda(), turned, err, interleaved=interleaved)
    assert torch.equal(turned, out)
    Q.rope_query(qd[..., 128:], pos.cuda(), cs.cuda(), qd[..., 128:], err, interleaved=interleaved)
    assert torch.equal(qd, torch.cat([q[..., :128].cuda(), out], -1)) and Q.read_dev_err(err) == 0


@pytest.mark.parametrize("kind", KINDS)
def test_strides_of_a_single_row_are_not_used(kind):
    """One token, one head: any stride may stand in the axes of one element."""
    c = Cache(kind, [3])
    one = lambda t, last: t.cuda().as_strided((1, last), (last + 1, 1))  # noqa: E731
    lens_dev = torch.tensor([3], dtype=torch.int32, device="cuda")
    at = torch.tensor([2])
    x = torch.cat([normed(c.rows[at, :512], c.weight, 1e-6), rotated(c.rows[at, 512:], c.cs, c.pos[at], False)], 1)
    want, want_prot = c.plain(x, lens_dev, at)
    pool, prot, err = c.fresh()
    seq, pos, table, cs = c.seq[at].cuda(), c.pos[at].cuda(), c.table.cuda(), c.cs.cuda()
    Q.rope_append(pool, c.kind, one(c.rows[2, :512].contiguous(), 512), one(c.rows[2, 512:].contiguous(), 64), seq, pos, table,
                  cs, err, norm_weight=c.weight.cuda(), seq_lens=lens_dev if c.protect else None, prot=prot)
    assert torch.equal(pool, want) and (not c.protect or torch.equal(prot, want_prot))
    keep = dict(seq_lens=lens_dev if c.protect else None, prot=prot)
    rows = [torch.zeros(1, 576, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    Q.cache_read(pool, c.kind, seq, pos, table, rows[0], err, **keep)
    Q.cache_read(pool, c.kind, seq, pos, table, rows[1].as_strided((1, 576), (577, 1)), err, **keep)
    assert torch.equal(*rows) and bool(rows[0].any())
    q = torch.randn(1, 1, 64).bfloat16().cuda()
    out = [torch.zeros_like(q) for _ in range(2)]
    Q.rope_query(q, pos, cs, out[0], err)
    Q.rope_query(q.as_strided((1, 1, 64), (3, 5, 1)), pos, cs, out[1].as_strided((1, 1, 64), (65, 1, 1)), err)
    assert torch.equal(*out) and bool(out[0].any()) and Q.read_dev_err(err) == 0


def test_rope_query_broadcast_heads_and_bad_positions():
    g = torch.Generator().manual_seed(4)
    q = torch.randn(6, 1, 64, generator=g).bfloat16().cuda().expand(6, 5, 64)  # head stride 0: one row for all heads
    pos = torch.tensor([0, 9, -1, 10, 3, 1 << 30], dtype=torch.int32)
    cs, err = table_of(10), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((6, 5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    Q.rope_query(q, pos.cuda(), cs.cuda(), out, err)
    assert Q.read_dev_err(err) == Q.DEVERR_BAD_POSITION
    good = [0, 1, 4]
    assert turned_right(out[good].cpu(), q.cpu()[good], cs, pos[good], False)
    assert bool((out[[2, 3, 5]] == 7).all())


def test_blocks_and_rows_past_32_bits():
    """A pool of over 4 GB, its last block, and rows that lie behind 4 GB of others."""
    blocks = (1 << 32) // WIDTH[4] + 40
    pool = torch.zeros(blocks, WIDTH[4], dtype=torch.uint8, device="cuda")
    table = torch.tensor([[blocks - 1, blocks - 2]], dtype=torch.int32, device="cuda")
    c = Cache(4, [100], seed=21)
    seq, pos = c.seq.cuda(), c.pos.cuda()
    wide = torch.zeros(3_730_000, 576, dtype=torch.bfloat16, device="cuda")[-100:]  # 4.3 GB before them
    wide.copy_(c.rows)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    Q.rope_append(pool, 4, wide[:, :512], wide[:, 512:], seq, pos, table, c.cs.cuda(), err, norm_weight=c.weight.cuda())
    Q.cache_read(pool, 4, seq, pos, table, wide, err)
    assert Q.read_dev_err(err) == 0
    x = torch.cat([normed(c.rows[:, :512], c.weight, 1e-6), rotated(c.rows[:, 512:], c.cs, c.pos, False)], 1)
    assert torch.equal(wide.cpu(), dequantised(x, 4))
    assert not bool(pool[:-2].any())


def test_a_zero_row_and_large_values():
    """eps keeps a row of zeros finite; without it the row is NaN, as 0 / 0 is. Large and
    small rows (2^40, 2^-40) normalise like any other."""
    c = Cache("bf16", [4], seed=2)
    c.rows[0, :512] = 0
    c.rows[1, :512] *= 2.0 ** 40
    c.rows[2, :512] *= 2.0 ** -40
    check_append(c, True, True, False, torch.arange(4), strided=False)
    pool, _, err = c.fresh()
    rows = c.rows.cuda()
    Q.rope_append(pool, "bf16", rows[:, :512], rows[:, 512:], None, torch.zeros(1, dtype=torch.int32, device="cuda").expand(4).contiguous(),
                  torch.tensor([[0], [1], [2], [-1]], dtype=torch.int32, device="cuda"), c.cs.cuda(), err, norm=True, eps=0.0)
    first = pool.view(torch.bfloat16).view(c.total, 64, 576)[0, 0]
    assert bool(first[:512].isnan().all()) and bool(first[512:].isfinite().all())
    assert Q.read_dev_err(err) == Q.DEVERR_BAD_BLOCK


def test_on_another_stream_and_replayed():
    """A captured step (write, read back, rotate) replays on new inputs in the same buffers."""
    c = Cache(4, [40, 25], seed=8)
    n = 65
    pool, _, err = c.fresh()
    rows, seq, pos, table, cs = c.rows.cuda(), c.seq.cuda(), c.pos.cuda(), c.table.cuda(), c.cs.cuda()
    q = torch.randn(n, 4, 192, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    out = torch.empty(n, 576, dtype=torch.bfloat16, device="cuda")
    qo = torch.empty(n, 4, 64, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()

    def step():
        Q.rope_append(pool, 4, rows[:, :512], rows[:, 512:], seq, pos, table, cs, err, norm=True)
        Q.cache_read(pool, 4, seq, pos, table, out, err)
        Q.rope_query(q[..., 128:], pos, cs, qo, err)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rows.mul_(-1)
    graph.replay()
    torch.cuda.synchronize()
    x = torch.cat([normed(-c.rows[:, :512], None, 1e-6), rotated(-c.rows[:, 512:], c.cs, c.pos, False)], 1)
    assert torch.equal(out.cpu(), dequantised(x, 4)) and not torch.equal(out, first)
    assert turned_right(qo.cpu(), q.cpu()[..., 128:], c.cs, c.pos, False)
    assert Q.read_dev_err(err) == 0 and math.isfinite(float(out.float().sum()))
