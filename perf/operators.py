"""Workloads of the operators around the latent-attention decode: what a serving
program runs between the projections of a layer and the cache, and the attention
of prompts.

  rope_append   normalises new latents, rotates their RoPE keys and writes them
                into a paged cache (any format) in one pass
  cache_read    reads cached tokens back as bf16 rows (latent, RoPE key), as the
                expanded form of the attention needs them before its up-projection
  rope_query    rotates the RoPE part of queries
  mla_prefill   attention of ragged prompts over expanded keys and values: 128
                content channels a head and one RoPE key a token for all heads

A case is a dict of plain values:

  kind      "step":   what precedes a decode step: each sequence's newest token
                      normalised, rotated and written, the queries rotated, and
                      the new tokens read back
            "chunk":  a prompt chunk written, then the whole sequences read back
            "query":  the queries of a prompt rotated
            "attend": the attention of prompts
  cache     "int4", "int2", "c4r4" or "bf16" (step and chunk)
  protect   sink4/local128 rows written and read (packed caches)
  norm      the latents are normalised on the way
  interleaved
            rotation of neighbouring channels, else of channels i and i + 32
  batch, heads
  new_lo, new_hi, ctx_lo, ctx_hi
            new tokens of each sequence and tokens before them, spread over these
            ranges (the same for every seed)
  causal    attend: new token i sees the context and the new tokens up to i; else
            every new token sees the context alone (the part of a chunked prompt
            that is merged by its log-sum-exp)
  pad       attend: query rows behind the last sequence, which stay as they are

Latents have per-channel gains with outlier channels (Student-t for INT2) as in
the repository's synthetic workloads; queries are N(0, 1), expanded keys and values
N(0, 1) times a gain, so that a softmax of scale 1/sqrt(192) is neither flat nor
a single peak.
"""
from __future__ import annotations

import math

import torch

own = False

TAU = 1.0 / math.sqrt(192.0)
EPS = 1e-6
BLOCK = 64
DC, DR, DN, DV = 512, 64, 128, 128
TOKEN_BYTES = {"int4": 324, "int2": 196, "c4r4": 320, "bf16": 1152}
BLOCK_BYTES = {"int4": 20736, "int2": 12544, "c4r4": 20480, "bf16": 73728}


def _case(name, kind, cache="int4", protect=False, norm=True, interleaved=False, batch=1, heads=16, new=(1, 1),
          ctx=(0, 0), causal=True, pad=0):
    c = {"kind": kind, "cache": cache, "protect": protect, "norm": norm, "interleaved": interleaved, "batch": batch,
         "heads": heads, "new_lo": new[0], "new_hi": new[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1], "causal": causal,
         "pad": pad}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One chat turn's next token, 16 heads on this GPU: all latency.
        _case("step_b1_h16_int4", "step", "int4", heads=16, ctx=(256, 256)),
        # The DeepSeek-V3-shaped serving step on the paper's page with protection.
        _case("step_b64_h128_c4r4_protected", "step", "c4r4", protect=True, interleaved=True, batch=64, heads=128,
              ctx=(4096, 4096)),
        # Prompts of several requests written in one call and read back for their up-projection.
        _case("chunk_8x_int4_32k", "chunk", "int4", batch=8, new=(2500, 5700)),
        # A later chunk of chunked prompts at odd offsets, INT2 with protection.
        _case("chunk_ctx_int2_protected", "chunk", "int2", protect=True, interleaved=True, batch=3, new=(700, 1301),
              ctx=(1900, 9001)),
        # A short question behind one long document on the unquantised cache: reading dominates.
        _case("chunk_long_bf16", "chunk", "bf16", norm=False, batch=1, new=(517, 517), ctx=(98304, 98304)),
        # The queries of a few speculative tokens, and those of a chunk of prompts.
        _case("query_b5_h16", "query", batch=5, heads=16, ctx=(300, 2500)),
        _case("query_8k_h128", "query", interleaved=True, batch=4, heads=128, new=(1900, 2196), ctx=(0, 4096)),
        # One short prompt, 16 heads on this GPU: all latency.
        _case("attend_b1_h16_37", "attend", heads=16, new=(37, 37)),
        # A batch of ragged chat prompts with rows of padding behind them.
        _case("attend_b8_h128_chat", "attend", batch=8, heads=128, new=(100, 1500), pad=45),
        # One prompt of the DeepSeek-V3-shaped workload's length.
        _case("attend_4k_h128", "attend", heads=128, new=(4096, 4096)),
        # Context part of a later chunk: ragged long contexts, one sequence without any.
        _case("attend_ctx_h64", "attend", batch=3, heads=64, new=(300, 811), ctx=(0, 14001), causal=False),
        # A long prompt, heads sharded to 64: the largest.
        _case("attend_8k_h64", "attend", heads=64, new=(8192, 8192)),
    ]


_MAX_PAIRS = 64 * 8192 * 8192  # heads x queries x keys of the largest listed attention
_MAX_READ = 98821


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["step", "chunk", "chunk", "query", "attend", "attend", "attend"])
    cache = rng.choice(["int4", "int4", "int2", "c4r4", "bf16"])
    protect = cache != "bf16" and rng.random() < 0.4
    norm, inter = rng.random() < 0.75, rng.random() < 0.5
    heads = rng.choice([16, 20, 32, 64, 100, 128, 128])
    if kind == "step":
        hi = _log_int(rng, 1, 9000)
        return _case(None, kind, cache, protect, norm, inter, _log_int(rng, 1, 128), heads, (1, 1),
                     (rng.randint(0, hi), hi))
    if kind == "chunk":
        total = _log_int(rng, 64, 65536)
        batch = rng.randint(1, max(1, min(16, total // 40)))
        new = max(1, int(total / batch * rng.choice([1.0, 1.0, 0.5, 0.1])))
        ctx = max(0, total // batch - new)
        return _case(None, kind, cache, protect, norm, inter, batch, 16, (max(1, new // 2), new), (ctx // 3, ctx))
    if kind == "query":
        total = _log_int(rng, 1, 8192)
        batch = rng.randint(1, max(1, min(16, total // 8)))
        new = max(1, total // batch)
        return _case(None, kind, "int4", False, True, inter, batch, heads, (max(1, new // 2), new),
                     (0, rng.randint(0, 9000)))
    causal = rng.random() < 0.75
    batch = _log_int(rng, 1, 16)
    hi = _log_int(rng, 1, 8192)
    ctx = rng.choice([0, 0, _log_int(rng, 1, 16384)]) if causal else _log_int(rng, 1, 16384)
    while batch * heads * hi * (hi * causal + ctx) > _MAX_PAIRS:
        hi, ctx, batch = max(1, hi * 3 // 4), ctx * 3 // 4, max(1, batch * 3 // 4)
    if not causal:
        ctx = max(1, ctx)
    return _case(None, kind, batch=batch, heads=heads, new=(max(1, int(hi * rng.uniform(0.1, 1.0))), hi),
                 ctx=(int(ctx * rng.uniform(0.0, 1.0)), ctx), causal=causal, pad=rng.choice([0, 0, rng.randint(1, 200)]))


# ---------------------------------------------------------------- inputs
def _spread(lo, hi, batch, step):
    """batch lengths from lo to hi, both ends taken, in a scattered order."""
    if batch == 1:
        return [hi]
    return [lo + ((i * (hi - lo)) // (batch - 1)) for i in sorted(range(batch), key=lambda i: (i * step) % 1.0)]


def _lengths(case):
    """(new tokens, context tokens) of each sequence."""
    return (_spread(case["new_lo"], case["new_hi"], case["batch"], 0.6180339887),
            _spread(case["ctx_lo"], case["ctx_hi"], case["batch"], 0.4142135624))


def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1_000_003 + stream)
    return g


def _table(rope_len):
    """cos | sin of the angles of the positions 0 .. rope_len - 1, as a model keeps them."""
    freq = 10000.0 ** (-torch.arange(DR // 2, device="cuda", dtype=torch.float64) / (DR // 2))
    ang = torch.arange(rope_len, device="cuda", dtype=torch.float64)[:, None] * freq[None, :]
    return torch.cat([torch.cos(ang), torch.sin(ang)], 1).float()


def _rows(counts, first):
    """(sequence, position) of counts[b] tokens from position first[b] on, sequence by sequence."""
    n = torch.tensor(counts, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), n, output_size=sum(counts))
    at = torch.arange(sum(counts), device="cuda") - (torch.cumsum(n, 0) - n)[seq]
    return seq.int(), (at + torch.tensor(first, device="cuda")[seq]).int()


def _draw_rows(case, seed, stream, n):
    """n rows of the down-projection: 512 latent channels and 64 of the RoPE key."""
    g = _gen(seed, stream)
    gain = torch.exp(0.5 * torch.randn(DC, generator=_gen(seed, 1), device="cuda"))
    if case["cache"] != "int2":
        gain[torch.randperm(DC, generator=_gen(seed, 2), device="cuda")[:4]] *= 8.0
    x = torch.randn(n, DC, generator=g, device="cuda")
    if case["cache"] == "int2":  # Student-t with 4 degrees of freedom
        u = 1.0 - torch.rand(2, n, DC, generator=g, device="cuda")
        x = x / torch.sqrt(-0.5 * (torch.log(u[0]) + torch.log(u[1]))).clamp_min(1e-3)
    return torch.cat([x * gain, torch.randn(n, DR, generator=g, device="cuda")], 1).bfloat16()


def _draw_weight(seed):
    return (1.0 + 0.2 * torch.randn(DC, generator=_gen(seed, 3), device="cuda")).bfloat16()


def _draw_queries(case, seed, n):
    return torch.randn(n, case["heads"], DN + DR, generator=_gen(seed, 4), device="cuda").bfloat16()


def _prepare_cache(case, seed):
    B, (new, ctx) = case["batch"], _lengths(case)
    ends = [a + b for a, b in zip(new, ctx)]
    nblk = [max(1, -(-n // BLOCK)) for n in ends]
    perm = torch.randperm(sum(nblk), generator=_gen(seed, 5), device="cuda").int()
    table = torch.full((B, max(nblk)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(nblk):
        table[b, :n] = perm[at:at + n]
        at += n
    st = {"case": case, "table": table, "cos_sin": _table(max(ends)),
          "pool": torch.zeros((sum(nblk), BLOCK_BYTES[case["cache"]]), dtype=torch.uint8, device="cuda"),
          "prot": torch.zeros((B, 132, DC + DR), dtype=torch.bfloat16, device="cuda") if case["protect"] else None,
          "lens": torch.tensor(ends, dtype=torch.int32, device="cuda"), "weight": _draw_weight(seed),
          "err": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if sum(ctx):  # what earlier calls wrote
        seq, pos = _rows(ctx, [0] * B)
        _plain_append(case, st, _draw_rows(case, seed, 6, sum(ctx)), seq, pos,
                      torch.tensor(ctx, dtype=torch.int32, device="cuda"))
    st["rows"] = _draw_rows(case, seed, 7, sum(new))
    st["seq"], st["pos"] = _rows(new, ctx)
    whole = case["kind"] == "chunk"
    st["read_seq"], st["read_pos"] = _rows(ends, [0] * B) if whole else (st["seq"], st["pos"])
    st["values"] = torch.zeros((st["read_seq"].numel(), DC + DR), dtype=torch.bfloat16, device="cuda")
    return st


def _prepare_attend(case, seed):
    H, (new, ctx) = case["heads"], _lengths(case)
    kv = [(a if case["causal"] else 0) + b for a, b in zip(new, ctx)]
    nq, nkv, g = sum(new) + case["pad"], sum(kv), _gen(seed, 8)
    cu = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")  # noqa: E731
    st = {"case": case, "q": _draw_queries(case, seed, nq), "cu_q": cu(new), "cu_kv": cu(kv), "max_q": max(new),
          "max_kv": max(kv), "total": sum(new),
          # the up-projection's output, keys beside values, and rows as cache_read leaves them
          "kv": (1.2 * torch.randn(nkv, H, DN + DV, generator=g, device="cuda")).bfloat16(),
          "rows": torch.randn(nkv, DC + DR, generator=g, device="cuda").bfloat16(),
          "out": torch.zeros((nq, H, DV), dtype=torch.bfloat16, device="cuda"),
          "lse": torch.zeros((nq, H), dtype=torch.float32, device="cuda"),
          "err": torch.zeros(1, dtype=torch.int32, device="cuda")}
    # one workspace for every call of the program: more than any of these cases asks for
    st["ws"] = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    return st


def prepare(case, seed):
    """The rows, cache, tables and buffers that a serving program holds."""
    if case["kind"] == "attend":
        return _prepare_attend(case, seed)
    new, ctx = _lengths(case)
    if case["kind"] == "query":
        st = {"case": case, "cos_sin": _table(max(a + b for a, b in zip(new, ctx))), "pos": _rows(new, ctx)[1],
              "err": torch.zeros(1, dtype=torch.int32, device="cuda")}
    else:
        st = _prepare_cache(case, seed)
    if case["kind"] != "chunk":
        st["q"] = _draw_queries(case, seed, sum(new))
        st["q_pe"] = torch.zeros((sum(new), case["heads"], DR), dtype=torch.bfloat16, device="cuda")
    return st


# ---------------------------------------------------------------- plain forms
def _plain_rotate(x, cos_sin, pos, interleaved):
    """x [n, ..., 64] at positions pos [n], in 64 bits: rounded once, to 32, before bf16."""
    t = cos_sin[pos.long()].double().view(-1, *([1] * (x.dim() - 2)), DR)
    c, s = t[..., :DR // 2], t[..., DR // 2:]
    x = x.double()
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :DR // 2], x[..., DR // 2:])
    u, v = a * c - b * s, a * s + b * c
    return (torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)).float().bfloat16()


def _plain_rows(case, st, rows, pos):
    """Rows as the cache takes them: the latent normalised, the RoPE key rotated, in bf16."""
    x = rows[:, :DC]
    if case["norm"]:
        d = x.double()
        x = (d * st["weight"].double() / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS)).float().bfloat16()
    return torch.cat([x, _plain_rotate(rows[:, DC:], st["cos_sin"], pos, case["interleaved"])], 1)


def _plain_groups(cache, x, bits, content):
    """Codes, scales and zero points of bf16 groups x [n, groups, 64]."""
    m = float(2 ** bits - 1)
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = ((hi - lo).clamp_min(1e-8).double() / m).float()
    if cache == "c4r4":
        s = s.bfloat16().float() if content else s
        z = torch.round((-lo.double() / s.double()).float()).clamp(0, m)
        q = torch.round((x.double() / s.double()).float() + z).clamp(0, m)
    else:
        s = s.half().float()
        s = torch.where(s == 0, torch.full_like(s, 2.0 ** -24), s).clamp_max(65504.0)
        z = torch.round(-lo.double() / s.double()).clamp(0, m).float()
        q = torch.round(x.double() / s.double() + z.double()).clamp(0, m)
    return q.to(torch.uint8), s, z


def _plain_pack(q, bits):
    if bits == 4:
        return q[..., 0::2] | (q[..., 1::2] << 4)
    return q[..., 0::4] | (q[..., 1::4] << 2) | (q[..., 2::4] << 4) | (q[..., 3::4] << 6)


def _bytes(x, dtype):
    return x.to(dtype).contiguous().view(torch.uint8)


def _regions(case):
    """Byte offsets of a token slot's parts in a block: (offset, bytes per slot, bytes per group, groups)."""
    if case["cache"] == "bf16":
        return [(0, 1152, 0, 1)]
    cb = 16 if case["cache"] == "int2" else 32
    if case["cache"] == "c4r4":
        return [(0, 32, 2048, 8), (16384, 32, 0, 1), (18432, 2, 128, 8), (19456, 4, 0, 1), (19712, 1, 64, 9)]
    return [(0, cb, 64 * cb, 8), (512 * cb, 32, 0, 1), (512 * cb + 2048, 4, 256, 9)]


def _place(st, seq, pos):
    blk = st["table"][seq.long(), (pos // BLOCK).long()].long()
    return blk, (pos % BLOCK).long()


def _where(region, blk, slot):
    """Indices [n, groups, bytes] into a pool of one region's bytes of each token."""
    off, per_slot, per_group, groups = region
    d = torch.device("cuda")
    col = (off + slot[:, None, None] * per_slot + torch.arange(groups, device=d)[None, :, None] * per_group
           + torch.arange(per_slot, device=d)[None, None, :])
    return blk[:, None, None].expand_as(col), col


def _plain_append(case, st, rows, seq, pos, lens):
    x = _plain_rows(case, st, rows, pos)
    blk, slot = _place(st, seq, pos)
    if case["cache"] == "bf16":
        parts = [x.contiguous().view(torch.uint8).view(-1, 1, 1152)]
    else:
        bits = 2 if case["cache"] == "int2" else 4
        cq, cs, cz = _plain_groups(case["cache"], x[:, :DC].view(-1, 8, 64), bits, True)
        rq, rs, rz = _plain_groups(case["cache"], x[:, DC:].view(-1, 1, 64), 4, False)
        parts = [_plain_pack(cq, bits), _plain_pack(rq, 4)]
        if case["cache"] == "c4r4":
            parts += [_bytes(cs, torch.bfloat16), _bytes(rs, torch.float32), torch.cat([cz, rz], 1).to(torch.uint8)]
        else:
            parts += [_bytes(torch.cat([torch.cat([cs, cz], -1), torch.cat([rs, rz], -1)], 1), torch.float16)]
    for region, p in zip(_regions(case), parts):
        st["pool"][_where(region, blk, slot)] = p
    if case["protect"]:
        s, at = seq.long(), pos.long()
        sink = torch.where(at < 4, at, torch.full_like(at, 132))
        late = torch.where(at >= lens[s] - 128, 4 + at % 128, torch.full_like(at, 132))
        wide = torch.cat([st["prot"], torch.zeros_like(st["prot"][:, :1])], 1)  # row 132: written by nobody else
        wide[s, sink] = x
        wide[s, late] = x
        st["prot"].copy_(wide[:, :132])


def _plain_read(case, st):
    seq, pos = st["read_seq"], st["read_pos"]
    blk, slot = _place(st, seq, pos)
    got = [st["pool"][_where(r, blk, slot)] for r in _regions(case)]
    n = seq.numel()
    if case["cache"] == "bf16":
        return got[0].view(n, 1152).view(torch.bfloat16)
    nib = lambda p: torch.stack([p & 15, p >> 4], -1).flatten(-2)  # noqa: E731
    crumb = lambda p: torch.stack([p & 3, (p >> 2) & 3, (p >> 4) & 3, p >> 6], -1).flatten(-2)  # noqa: E731
    c, r = (crumb if case["cache"] == "int2" else nib)(got[0]).float(), nib(got[1]).float()
    if case["cache"] == "c4r4":
        cs, rs = got[2].view(torch.bfloat16).float(), got[3].view(torch.float32)
        cz, rz = got[4][:, :8].float(), got[4][:, 8:].float()
    else:
        sz = got[2].view(torch.float16).float()
        cs, cz, rs, rz = sz[:, :8, :1], sz[:, :8, 1:], sz[:, 8:, :1], sz[:, 8:, 1:]
    x = torch.cat([(cs * (c - cz)).reshape(n, DC), (rs * (r - rz)).reshape(n, DR)], 1).bfloat16()
    if case["protect"]:
        s, at = seq.long(), pos.long()
        row = torch.where(at < 4, at, 4 + at % 128)
        kept = (at < 4) | (at >= st["lens"][s] - 128)
        x = torch.where(kept[:, None], st["prot"][s, row], x)
    return x


def _plain_attend(st):
    """Sequences side by side in [batch, longest] rectangles, in 32 bits."""
    case = st["case"]
    H, B, lq, lk = case["heads"], case["batch"], st["max_q"], st["max_kv"]
    d = torch.device("cuda")
    nq, nk = st["cu_q"][1:] - st["cu_q"][:-1], st["cu_kv"][1:] - st["cu_kv"][:-1]
    qi, ki = torch.arange(lq, device=d), torch.arange(lk, device=d)
    at_q = (st["cu_q"][:-1, None] + qi).clamp_max(st["total"] - 1).long()
    at_k = (st["cu_kv"][:-1, None] + ki).clamp_max(max(0, st["kv"].size(0) - 1)).long()
    q = st["q"][at_q].float().transpose(1, 2)  # [B, H, lq, 192]
    k, pe = st["kv"][at_k, :, :DN].float().transpose(1, 2), st["rows"][at_k, DC:].float()
    s = torch.matmul(q[..., :DN], k.transpose(-1, -2))
    s += torch.matmul(q[..., DN:].reshape(B, H * lq, DR), pe.transpose(-1, -2)).view(B, H, lq, lk)
    s *= TAU
    hide = (ki[None, None, :] >= nk[:, None, None]) | (qi[None, :, None] >= nq[:, None, None])
    if case["causal"]:
        hide = hide | (ki[None, None, :] > (qi[None, :, None] + (nk - nq)[:, None, None]))
    s.masked_fill_(hide[:, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s -= torch.where(torch.isinf(top), torch.zeros_like(top), top)
    s.exp_()
    den = s.sum(-1, keepdim=True)
    v = st["kv"][at_k, :, DN:].float().transpose(1, 2)
    o = torch.where(den > 0, torch.matmul(s, v) / den, torch.zeros_like(den))
    lse = (top + torch.log(den)).squeeze(-1)
    seq = torch.repeat_interleave(torch.arange(B, device=d), nq, output_size=st["total"])
    row = torch.arange(st["total"], device=d) - st["cu_q"][:-1].long()[seq]
    out, out_lse = torch.zeros_like(st["out"]), torch.zeros_like(st["lse"])
    out[:st["total"]] = o.transpose(1, 2)[seq, row].bfloat16()
    out_lse[:st["total"]] = lse.transpose(1, 2)[seq, row]
    return {"out": out, "lse": out_lse}


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        return _own(case, st)
    if kind == "attend":
        return _plain_attend(st)
    got = {}
    if kind != "query":
        _plain_append(case, st, st["rows"], st["seq"], st["pos"], st["lens"])
        got["values"] = _plain_read(case, st)
        if case["protect"]:
            got["prot"] = st["prot"]
    if kind != "chunk":
        got["q_pe"] = _plain_rotate(st["q"][..., DN:], st["cos_sin"], st["pos"], case["interleaved"])
    return got


def _own(case, st):
    import paper_2609_36760_gb300 as Q
    kind = case["kind"]
    if kind == "attend":
        Q.mla_prefill(st["q"], st["kv"][..., :DN], st["kv"][..., DN:], st["rows"][:, DC:], st["cu_q"], st["cu_kv"], TAU,
                      st["out"], st["lse"], st["ws"], st["err"], causal=case["causal"])
        return {"out": st["out"], "lse": st["lse"]}
    got = {}
    if kind != "query":
        cache = {"int4": 4, "int2": 2}.get(case["cache"], case["cache"])
        Q.rope_append(st["pool"], cache, st["rows"][:, :DC], st["rows"][:, DC:], st["seq"], st["pos"], st["table"],
                      st["cos_sin"], st["err"], norm_weight=st["weight"] if case["norm"] else None, eps=EPS,
                      interleaved=case["interleaved"], seq_lens=st["lens"] if case["protect"] else None,
                      prot=st["prot"])
        Q.cache_read(st["pool"], cache, st["read_seq"], st["read_pos"], st["table"], st["values"], st["err"],
                     seq_lens=st["lens"] if case["protect"] else None, prot=st["prot"])
        got["values"] = st["values"]
        if case["protect"]:
            got["prot"] = st["prot"]
    if kind != "chunk":
        Q.rope_query(st["q"][..., DN:], st["pos"], st["cos_sin"], st["q_pe"], st["err"],
                     interleaved=case["interleaved"])
        got["q_pe"] = st["q_pe"]
    return got


def work(case):
    H, (new, ctx) = case["heads"], _lengths(case)
    n = sum(new)
    if case["kind"] == "attend":
        flops = 0
        for a, b in zip(new, ctx):
            pairs = a * b + (a * (a + 1) // 2 if case["causal"] else 0)
            flops += 2 * (DN + DR + DV) * H * pairs
        kv = sum(ctx) + (n if case["causal"] else 0)
        return {"bytes": n * H * (2 * (DN + DR) + 2 * DV + 4) + kv * (H * 2 * (DN + DV) + 2 * DR), "flops": flops}
    turn = n * H * 2 * 2 * DR + n * 4 * DR  # queries in and out, the angles of their tokens
    if case["kind"] == "query":
        return {"bytes": turn, "flops": n * H * 3 * DR}
    per = TOKEN_BYTES[case["cache"]]
    read = n if case["kind"] == "step" else n + sum(ctx)
    write = n * (2 * (DC + DR) + 4 * DR + per)
    if case["protect"]:
        write += sum(min(a, 132) for a in new) * 2 * (DC + DR)
    return {"bytes": write + (read - n) * per + read * 2 * (DC + DR) + (turn if case["kind"] == "step" else 0),
            "flops": n * 8 * DC + read * 2 * (DC + DR)}


# ---------------------------------------------------------------- 64-bit values
def _exact_row(case, cos_sin, weight, rows, pos):
    """What a row holds once it is normalised and rotated, before and after its rounding to bf16."""
    x = rows.double()
    lat, k = x[:, :DC], x[:, DC:]
    if case["norm"]:
        lat = weight.double() * lat * torch.rsqrt(lat.pow(2).sum(1, keepdim=True) / DC + EPS)
    e = torch.complex(cos_sin[:, :DR // 2].double(), cos_sin[:, DR // 2:].double())[pos.long()]
    if case["interleaved"]:
        k = torch.view_as_real(torch.view_as_complex(k.reshape(-1, DR // 2, 2).contiguous()) * e).flatten(1)
    else:
        w = torch.complex(k[:, :DR // 2].contiguous(), k[:, DR // 2:].contiguous()) * e
        k = torch.cat([w.real, w.imag], 1)
    return torch.cat([lat, k], 1)


def _exact_cached(case, x, first):
    """s (q - z) of rows x (bf16 values) for the groups from channel `first` on."""
    if case["cache"] == "bf16":
        return x.double()
    paper, content = case["cache"] == "c4r4", first < DC
    m = 3.0 if case["cache"] == "int2" and content else 15.0
    g = x.float().reshape(x.size(0), -1, 64)
    lo, span = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values - g.min(-1, keepdim=True).values
    s = span.clamp_min(1e-8).double().div(m).float()
    if paper:
        s = s.bfloat16().float() if content else s
        z = (-lo.double() / s.double()).float().round().clamp(0, m)
        q = ((g.double() / s.double()).float() + z).round().clamp(0, m)
    else:
        s = s.half().float().clamp(2.0 ** -24, 65504.0)
        z = (-lo.double() / s.double()).round().clamp(0, m)
        q = (g.double() / s.double() + z).round().clamp(0, m)
    return (s.double() * (q.double() - z.double())).reshape(x.size(0), -1)


def _exact_attend(case, seed):
    st = _prepare_attend(case, seed)
    new, ctx = _lengths(case)
    H = case["heads"]
    out = torch.zeros(st["q"].size(0), H, DV, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["q"].size(0), H, dtype=torch.float64, device="cuda")
    aq = ak = 0
    for a, b in zip(new, ctx):
        n = b + (a if case["causal"] else 0)
        pe = st["rows"][ak:ak + n, DC:].double()
        for h in range(H):
            key = torch.cat([st["kv"][ak:ak + n, h, :DN].double(), pe], 1)
            for i in range(0, a, 4096):  # some queries at a time
                sc = TAU * st["q"][aq + i:aq + min(a, i + 4096), h].double() @ key.T
                if case["causal"]:
                    sc = sc + torch.full_like(sc, -math.inf).triu(n - a + i + 1)
                z = torch.logsumexp(sc, 1)
                rows = slice(aq + i, aq + i + sc.size(0))
                lse[rows, h] = z
                if n:
                    w = torch.exp(sc - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
                    out[rows, h] = w @ st["kv"][ak:ak + n, h, DN:].double()
        aq, ak = aq + a, ak + n
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["kind"] == "attend":
        return _exact_attend(case, seed)
    B, (new, ctx) = case["batch"], _lengths(case)
    got = {}
    table = _table(max(a + b for a, b in zip(new, ctx)))
    pos = _rows(new, ctx)[1]
    if case["kind"] != "query":
        parts = [(_draw_rows(case, seed, 7, sum(new)), *_rows(new, ctx))]
        if case["kind"] == "chunk" and sum(ctx):
            parts.insert(0, (_draw_rows(case, seed, 6, sum(ctx)), *_rows(ctx, [0] * B)))
        ends = torch.tensor([a + b for a, b in zip(new, ctx)], device="cuda")
        vals, keys = [], []
        for rows, seq, at in parts:
            x = _exact_row(case, table, _draw_weight(seed), rows, at)
            r = x.float().bfloat16()
            if not case["norm"]:
                r[:, :DC] = rows[:, :DC]
            c = torch.cat([_exact_cached(case, r[:, :DC], 0), _exact_cached(case, r[:, DC:], DC)], 1)
            if case["cache"] == "bf16":
                c = x
            if case["protect"]:
                kept = (at < 4) | (at >= ends[seq.long()] - 128)
                c = torch.where(kept[:, None], x, c)
            vals.append(c)
            keys.append(seq.long() * (1 << 32) + at.long())
        order = torch.argsort(torch.cat(keys))
        got["values"] = torch.cat(vals)[order]
        if case["protect"]:
            got["prot"] = None
    if case["kind"] != "chunk":
        q = _draw_queries(case, seed, sum(new))[..., DN:]
        flat = torch.cat([torch.zeros(q.size(0) * case["heads"], DC, device="cuda", dtype=q.dtype),
                          q.reshape(-1, DR)], 1)
        rep = torch.repeat_interleave(pos, case["heads"])
        got["q_pe"] = _exact_row({**case, "norm": False}, table, None, flat, rep)[:, DC:].reshape(q.shape)
    return got
