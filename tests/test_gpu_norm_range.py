"""rope_append's norm over the whole range of bf16: rows whose squares, or the sum of them,
lie outside the range of fp32, with and without eps, in both forms of the fused writer.

x' = RN_bf16(RN_f32(w x / sqrt(mean x^2 + eps))) from 64-bit arithmetic, whose squares of
bf16 values neither overflow (3.4e38^2 = 1.2e77) nor underflow (9e-41^2 = 8e-81). Rows are
compared for equality, as the plain writers store x', except where a result lies below
2^-100: there the product's own rounding (2^-24) is not carried along, which can move the
rounding to bf16 by one step, |got - exact| <= 2^-8 (1 + 2^-15) |exact| + 2^-134 (half
a step of a subnormal)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_36760_gb300 as Q
from test_gpu_rows import KINDS, Cache, rotated

pytestmark = pytest.mark.gpu
LARGEST = 3.3895313892515355e38  # of bf16
FORMS = [7, 4300]  # tokens: a warp per group; a token in eight lanes


def exact(x, w, eps):
    d = x.double()
    eps = float(torch.tensor(eps, dtype=torch.float32))  # (as the call takes it)
    return d * (1.0 if w is None else w.double()) / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)


def write(c, rows, weight, eps, strided=False):
    """The cache of the rows (its own copy), and the plain writers' of x'."""
    pool, prot, err = c.fresh()
    dev = rows.cuda()
    lat, kpe = dev[:, :512], dev[:, 512:]
    if not strided:
        lat, kpe = lat.contiguous(), kpe.contiguous()
    Q.rope_append(pool, c.kind, lat, kpe, c.seq.cuda(), c.pos.cuda(), c.table.cuda(), c.cs.cuda(), err,
                  norm_weight=None if weight is None else weight.cuda(), norm=True, eps=eps)
    assert Q.read_dev_err(err) == 0
    return pool


def stored(c, pool):
    """The rows of a BF16 cache, in the order of the tokens."""
    blocks = c.table[c.seq.long(), (c.pos // 64).long()].long()
    return pool.cpu().view(torch.bfloat16).view(c.total, 64, 576)[blocks, (c.pos % 64).long()]


# (eps, factor of the rows): the squares' sum overflows; they underflow; eps against both.
FAR = [(1e-6, 2.0 ** 58), (1e-6, 2.0 ** 62), (0.0, 2.0 ** 100), (1e-6, 2.0 ** 120), (1e30, 2.0 ** 62), (0.0, 2.0 ** -46),
       (0.0, 2.0 ** -62), (0.0, 2.0 ** -75), (0.0, 2.0 ** -110), (1e-38, 2.0 ** -62), (1e-44, 2.0 ** -75), (1e-30, 2.0 ** -50)]


@pytest.mark.parametrize("n", FORMS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("weighted", [True, False])
def test_rows_far_from_one(n, kind, weighted):
    """Every third row far, of another factor than its neighbours; the others as ever."""
    c = Cache(kind, [n], seed=n)
    w = c.weight if weighted else None
    for eps in sorted({e for e, _ in FAR}):
        factors = [f for e, f in FAR if e == eps]
        rows = c.rows.clone()
        for i in range(0, n, 3):
            rows[i, :512] = (c.rows[i, :512].double() * factors[(i // 3) % len(factors)]).bfloat16()
        assert bool(rows.isfinite().all())
        x = torch.cat([exact(rows[:, :512], w, eps).float().bfloat16(), rotated(rows[:, 512:], c.cs, c.pos, False)], 1)
        assert torch.equal(write(c, rows, w, eps), c.plain(x, None, torch.arange(n))[0]), eps


@pytest.mark.parametrize("n", FORMS)
def test_the_ends_of_the_range(n):
    """The largest bf16 throughout, 1.5 x 2^59 throughout, the smallest normal and subnormal ones,
    one large value among small ones, a zero row, each with and without eps."""
    c = Cache("bf16", [n], seed=1)
    rows = c.rows.clone()
    rows[:, :512] = rows[:, :512].sign()
    sizes = [LARGEST, 1.5 * 2.0 ** 59, 2.0 ** -126, 2.0 ** -133, 3 * 2.0 ** -133]
    for i in range(n):
        rows[i, :512] = (rows[i, :512].double() * sizes[i % len(sizes)]).bfloat16()
    rows[5, :512] = 1.0
    rows[5, 100] = LARGEST
    rows[6, :512] = 0
    for eps in (0.0, 1e-6, 1e-44, 1e30):
        got = stored(c, write(c, rows, c.weight, eps))[:, :512].double()
        want = exact(rows[:, :512], c.weight, eps)
        plain = want.float().bfloat16().double()
        if eps == 0.0:
            assert bool(got[6].isnan().all())
            got[6] = want[6] = plain[6] = 0
        assert bool(((got - want).abs() <= 2.0 ** -8 * (1 + 2.0 ** -15) * want.abs() + 2.0 ** -134).all()), eps
        assert torch.equal(got[want.abs() >= 2.0 ** -100], plain[want.abs() >= 2.0 ** -100]), eps


@pytest.mark.parametrize("n", FORMS)
def test_infinite_and_nan_rows(n):
    """x / inf is 0, inf / inf is NaN; a NaN reaches its whole row and no other one."""
    c = Cache("bf16", [n], seed=2)
    clean = stored(c, write(c, c.rows, c.weight, 1e-6))
    rows = c.rows.clone()
    rows[1, 7], rows[1, 300], rows[1, 301] = math.inf, -math.inf, LARGEST
    rows[4, 511] = math.nan
    rows[5, 0], rows[5, 64] = math.nan, math.inf
    got = stored(c, write(c, rows, c.weight, 1e-6))
    special = torch.tensor([1, 4, 5])
    same = torch.ones(n, dtype=torch.bool)
    same[special] = False
    assert torch.equal(got[same], clean[same])
    infinite = torch.zeros(512, dtype=torch.bool)
    infinite[[7, 300]] = True
    assert bool(got[1, :512][infinite].isnan().all()) and bool((got[1, :512][~infinite] == 0).all())
    assert bool(got[[4, 5], :512].isnan().all())
    assert torch.equal(got[:, 512:], clean[:, 512:])


def test_far_rows_off_a_16_byte_boundary():
    """The form for rows in 4-byte pieces, over the wide form's border."""
    c = Cache(4, [4300], seed=3)
    rows = c.rows.clone()
    rows[::5, :512] = (rows[::5, :512].double() * 2.0 ** 70).bfloat16()
    rows[2::5, :512] = (rows[2::5, :512].double() * 2.0 ** -70).bfloat16()
    wide = torch.zeros(4300, 600, dtype=torch.bfloat16)
    wide[:, 2:578] = rows
    x = torch.cat([exact(rows[:, :512], c.weight, 0.0).float().bfloat16(), rotated(rows[:, 512:], c.cs, c.pos, False)], 1)
    assert torch.equal(write(c, wide[:, 2:578], c.weight, 0.0, strided=True), c.plain(x, None, torch.arange(4300))[0])


@pytest.mark.parametrize("n", FORMS)
@pytest.mark.parametrize("kind", [4, 2, "c4r4"])
def test_far_rows_among_protected_and_bad_ones(kind, n):
    """Sink and recent rows of far tokens; a far token without a place is not written."""
    c = Cache(kind, [n], protect=True, seed=4)
    c.rows[::2, :512] = (c.rows[::2, :512].double() * 2.0 ** 65).bfloat16()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    x = torch.cat([exact(c.rows[:, :512], c.weight, 1e-6).float().bfloat16(), rotated(c.rows[:, 512:], c.cs, c.pos, True)], 1)
    good = torch.arange(n)[torch.arange(n) != 2]
    want, want_prot = c.plain(x[good], lens, good)
    seq = c.seq.clone()
    seq[2] = 1  # (there is one sequence)
    pool, prot, err = c.fresh()
    rows = c.rows.cuda()
    Q.rope_append(pool, kind, rows[:, :512], rows[:, 512:], seq.cuda(), c.pos.cuda(), c.table.cuda(), c.cs.cuda(), err,
                  norm_weight=c.weight.cuda(), interleaved=True, seq_lens=lens, prot=prot)
    assert Q.read_dev_err(err) == Q.DEVERR_BAD_SEQ
    assert torch.equal(pool, want) and torch.equal(prot, want_prot)
