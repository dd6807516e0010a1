"""cache_keep: bytes moved, none changed."""
import numpy as np
import pytest
import torch

import paper_2609_36760_gb300 as Q
from speculation_cases import KINDS, Cache

pytestmark = pytest.mark.gpu


def slot_bytes(pool, kind, blk, slot):
    """Every byte of one token slot, as a flat array."""
    p = pool[blk]
    if kind == "bf16":
        return p[slot * 1152:(slot + 1) * 1152]
    cb = 16 if kind == 2 else 32
    regions = [(0, 8, cb), (512 * cb, 1, 32)] + ([(18432, 8, 2), (19456, 1, 4), (19712, 9, 1)] if kind == "c4r4"
                                                 else [(512 * cb + 2048, 9, 4)])
    return np.concatenate([p[o + (g * 64 + slot) * w:o + (g * 64 + slot + 1) * w] for o, n, w in regions for g in range(n)])


def put(pool, kind, blk, slot, data):
    p = pool[blk]
    if kind == "bf16":
        p[slot * 1152:(slot + 1) * 1152] = data
        return
    cb = 16 if kind == 2 else 32
    regions = [(0, 8, cb), (512 * cb, 1, 32)] + ([(18432, 8, 2), (19456, 1, 4), (19712, 9, 1)] if kind == "c4r4"
                                                 else [(512 * cb + 2048, 9, 4)])
    i = 0
    for o, n, w in regions:
        for g in range(n):
            p[o + (g * 64 + slot) * w:o + (g * 64 + slot + 1) * w] = data[i:i + w]
            i += w


def plain(c, paths):
    pool = c.pool.cpu().numpy().copy()
    old = pool.copy()
    t = c.table.numpy()
    for b, path in enumerate(paths):
        for i, node in enumerate(path):
            s, d = c.ctx[b] + node, c.ctx[b] + i
            put(pool, c.kind, t[b, d // 64], d % 64, slot_bytes(old, c.kind, t[b, s // 64], s % 64))
    return pool


def call(c, paths, nodes, alias=False, counts=True):
    path = torch.full((len(paths), nodes), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    kept = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    new = c.lens_d if alias else torch.full((len(paths),), 77, dtype=torch.int32, device="cuda")
    Q.cache_keep(c.pool, c.kind, c.table_d, c.lens_d, path.cuda(), kept, new, c.err, tree_lens=c.counts_d if counts else None,
                 prot=c.prot, draft_rows=c.drafts)
    return new.tolist()


PATHS = [[0], [0, 1, 2, 3], [0, 2, 5, 9], [0, 15], [], list(range(16)), [1, 3, 4, 6, 7, 8, 12, 14, 15]]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ctx", [0, 50, 57, 63, 64, 120, 1000])
def test_rows_move_and_nothing_else(kind, ctx):
    c = Cache(kind, [ctx + i for i in range(len(PATHS))], [16] * len(PATHS), seed=ctx)
    want = plain(c, PATHS)
    assert call(c, PATHS, 16, alias=ctx == 63, counts=ctx != 57) == [x + len(p) for x, p in zip(c.ctx, PATHS)]
    assert np.array_equal(c.pool.cpu().numpy(), want) and Q.read_dev_err(c.err) == 0


@pytest.mark.parametrize("kind", KINDS)
def test_the_largest_tree(kind):
    paths = [list(range(1, 64)), list(range(0, 64, 2)), list(range(64)), [63]]
    c = Cache(kind, [30, 64, 1, 127], [64] * 4, seed=1)
    want = plain(c, paths)
    call(c, paths, 64)
    assert np.array_equal(c.pool.cpu().numpy(), want) and Q.read_dev_err(c.err) == 0


@pytest.mark.parametrize("kind", [4, 2, "c4r4"])
@pytest.mark.parametrize("ctx", [0, 1, 3, 4, 60, 125, 128, 131, 400])
def test_protection_rows_are_those_of_the_new_length(kind, ctx):
    paths = [[0, 2, 3, 7, 8], [0, 1], [], [0, 4, 5, 6]]
    c = Cache(kind, [ctx, ctx + 1, ctx + 2, ctx + 3], [9] * 4, protect=True, seed=ctx)
    before = c.prot.clone()
    new = call(c, paths, 9)
    got = c.prot.cpu()
    for b, path in enumerate(paths):
        x = torch.cat([c.rows[b][:c.ctx[b]], c.rows[b][c.ctx[b]:][path]])
        L = new[b]
        want = before[b].cpu()
        for p in range(c.ctx[b], L):
            want[4 + p % 128] = x[p]
            if p < 4:
                want[p] = x[p]
        assert torch.equal(torch.nan_to_num(got[b], nan=-9.0), torch.nan_to_num(want, nan=-9.0))
        for p in range(L):  # every protected position of the new length
            if p < 4:
                assert torch.equal(got[b, p], x[p])
            elif p >= L - 128:
                assert torch.equal(got[b, 4 + p % 128], x[p])


def test_bad_paths_counts_and_lengths_leave_the_sequence_alone():
    def fresh():
        return Cache(4, [100, 20], [8, 8], seed=3)

    for path, kept in (([0, 2, 2], 3), ([0, 5, 3], 3), ([-1, 2], 2), ([0, 8], 2), ([0], 9), ([0], -1), ([0, 1 << 30], 2)):
        c = fresh()
        before = c.pool.clone()
        p = torch.full((2, 8), -1, dtype=torch.int32)
        p[0, :len(path)] = torch.tensor(path, dtype=torch.int32)
        p[1, :2] = torch.tensor([0, 5], dtype=torch.int32)
        new = torch.zeros(2, dtype=torch.int32, device="cuda")
        Q.cache_keep(c.pool, 4, c.table_d, c.lens_d, p.cuda(), torch.tensor([kept, 2], dtype=torch.int32, device="cuda"), new,
                     c.err, tree_lens=c.counts_d)
        assert Q.read_dev_err(c.err) == Q.DEVERR_BAD_TREE and new.tolist() == [108, 22]
        c2 = fresh()
        want = plain(c2, [[], [0, 5]])
        assert np.array_equal(c.pool.cpu().numpy(), want) and torch.equal(before, c2.pool)
    for n, ln, bit in ((9, 108, Q.DEVERR_BAD_TREE), (-1, 108, Q.DEVERR_BAD_TREE), (8, 7, Q.DEVERR_BAD_TREE),
                       (8, -1, Q.DEVERR_BAD_POSITION), (8, 1 << 20, Q.DEVERR_BAD_POSITION)):
        c = fresh()
        before = c.pool.clone()
        c.counts_d[0], c.lens_d[0] = n, ln
        assert call(c, [[0, 4], []], 8) == [ln, 20]
        assert Q.read_dev_err(c.err) == bit and torch.equal(c.pool, before)


def test_bad_blocks_are_not_touched():
    c = Cache("bf16", [60], [16], seed=3)
    want = plain(c, [[0, 2]])  # 60 -> 60, 62 -> 61: the second block is not needed
    c.table_d[0, 1] = 99
    call(c, [[0, 2]], 16)
    assert Q.read_dev_err(c.err) == 0 and np.array_equal(c.pool.cpu().numpy(), want)
    before = c.pool.clone()
    assert call(c, [[0, 9]], 16) == [62]  # 69 lies in it
    assert Q.read_dev_err(c.err) == Q.DEVERR_BAD_BLOCK and torch.equal(c.pool, before)
