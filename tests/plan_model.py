"""The plan of mla_prefill (plan_kernel in prefill.cu) in plain Python, for good offsets: which
items a call has, which of their keys go in parts, and in what order of length the bundles
stand. Times of bundles of equal length are in no order."""
from __future__ import annotations

import numpy as np

TILE, ROWS, SHARES, LEAST, LENGTHS = 128, 256, 160, 4, (1.0, 1.15, 1.35, 1.7)
SLOTS, SMALL, THREADS = 2 * SHARES, 64, 1024


def item(q0, lq, k0, lk, r0, causal):
    rows = min(lq - r0, ROWS)
    vis0, step = (r0 + lk - lq + 1, 1) if causal else (lk, 0)
    steps = lambda last: -(-max(min(lk, vis0 + step * last), 0) // TILE)  # noqa: E731
    n0, n1 = steps(min(rows, TILE) - 1), steps(rows - 1) if rows > TILE else 0
    return dict(q_row=q0 + r0, rows=rows, kv_start=k0, kv_len=lk, vis0=vis0, step=step, n0=n0, n1=n1)


def rounds(it):
    return (3 * it["n0"] + 3) >> 2 if it["rows"] <= TILE else max(it["n0"], it["n1"])


def parts_at(r, length):
    return -(-r // length) if r - length > length >> 1 else 1


def plan(cu_q, cu_kv, n_q, n_kv, heads, causal, sms=152):
    batch = len(cu_q) - 1
    max_items = n_q // ROWS + batch
    size = 4 if max_items * heads >= 8 * sms else 1
    bundles = []
    for b in range(batch):
        q0, lq, k0, lk = cu_q[b], cu_q[b + 1] - cu_q[b], cu_kv[b], cu_kv[b + 1] - cu_kv[b]
        tiles = -(-lq // ROWS)
        for t0 in range(0, tiles, size):
            k = min(size, tiles - t0)
            bundles.append([item(q0, lq, k0, lk, (t0 + k - 1 - x) * ROWS, causal) for x in range(k)])
    items = [it for bundle in bundles for it in bundle]
    total = sum(rounds(it) for it in items) * heads
    f32 = np.float32

    def length(x):
        return max(int(min(f32(total) * f32(LENGTHS[x]) / f32(min(sms, SHARES - 1)), f32(1e9))) + 1, LEAST)

    longest = length(0)
    if any(parts_at(rounds(it), longest) > 1 for it in items):
        best = None
        for c in range(4):
            cut = [it for it in items if parts_at(rounds(it), length(c)) > 1]
            parts = sum(parts_at(rounds(it), length(c)) for it in cut) * heads
            whole = total - sum(rounds(it) for it in cut) * heads
            turns = 1 if parts == 0 or whole * 4 > total else -(-parts // sms)
            if best is None or f32(turns) * f32(length(c)) < best:
                best, longest = f32(turns) * f32(length(c)), length(c)
    out, joins, slots = [], [], 0
    for bundle in bundles:
        entries = []
        for it in bundle:
            parts = parts_at(rounds(it), longest)
            steps = max(it["n0"], it["n1"])
            per = -(-steps // (2 * parts)) * 2 if it["rows"] <= TILE else -(-steps // parts)
            if parts > 1:
                joins.append((it["q_row"], it["rows"], parts))
                slots += parts * heads
            for y in range(parts):
                skip = y * per if parts > 1 else 0
                e = dict(it, kv_start=it["kv_start"] + skip * TILE, kv_len=it["kv_len"] - skip * TILE,
                         vis0=it["vis0"] - skip * TILE, part=y, parts=parts)
                for n in ("n0", "n1"):
                    e[n] = max(0, min(it[n] - skip, per if parts > 1 else it[n]))
                e["dealt"] = int(e["rows"] <= TILE and e["n0"] > 1)
                entries.append(e)
        out.append(entries)
    threads = SMALL if max_items <= SMALL and batch <= SMALL else THREADS
    shift = 0
    while (n_kv // TILE + 1) >> shift >= threads:
        shift += 1
    return dict(bundles=out, joins=joins, slots=slots, size=size, longest=longest, total=total, shift=shift,
                threads=threads, max_items=max_items, keys=[max(rounds(it) for it in b) for b in bundles])
