"""Workloads of one step of speculative decoding over the paged latent caches: a
draft model proposes a tree of tokens for every sequence, the target scores all of
its nodes in one pass, the drafts are verified, and the cache keeps what was accepted.

  mla_decode_tree   attention of the nodes over the cached context and their own
                    ancestors, from any of the four caches
  tree_verify       walks each tree from its root: accepts drafted children against
                    the target's probabilities with given random numbers, and draws
                    the token after the last accepted node
  cache_keep        moves the accepted nodes' cache rows together behind the context,
                    in place, and gives the new lengths

A case is a dict of plain values:

  kind      "tree":   mla_decode_tree, the nodes' rows already in the cache
            "settle": tree_verify, then cache_keep of the path that it found
  cache     "int4", "int2", "c4r4" or "bf16"
  protect   sink4/local128 rows (packed caches); the nodes' own bf16 rows beside them
  batch, heads
  nodes     nodes of the largest tree, the committed token (its root) among them
  few       nodes of the smallest tree: the batch's counts are spread over few .. nodes
  branch    drafted children a node, about (1: a chain)
  ctx_lo, ctx_hi
            cached tokens before the tree, spread over this range
  vocab     settle: tokens of the vocabulary
  probs     settle: "f32" or "bf16" probabilities
  drafts    settle: "sampled": the draft model's probabilities are given, "certain":
            the drafts were chosen without randomness

Latents have per-channel gains with outlier channels as in the repository's synthetic
workloads, queries a spread that gives scores of standard deviation about 1.4. Draft
probabilities are a softmax of N(0, 2.5^2) logits, the target's of the same logits with
N(0, 0.7^2) added; the drafted tokens are drawn from the draft's.
"""
from __future__ import annotations

import math

import torch

own = False

TAU = 1.0 / math.sqrt(192.0)
BLOCK = 64
DC, DR = 512, 64
ROW = DC + DR
MAX_NODES = 64
TOKEN_BYTES = {"int4": 324, "int2": 196, "c4r4": 320, "bf16": 1152}
BLOCK_BYTES = {"int4": 20736, "int2": 12544, "c4r4": 20480, "bf16": 73728}
WORKSPACE = 1 << 29  # one workspace for every call of the program: more than any of these cases asks for


def _case(name, kind, cache="int4", protect=False, batch=1, heads=16, nodes=8, few=None, branch=2, ctx=(256, 256),
          vocab=0, probs="f32", drafts="sampled"):
    c = {"kind": kind, "cache": cache, "protect": protect, "batch": batch, "heads": heads, "nodes": nodes,
         "few": nodes if few is None else few, "branch": branch, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "vocab": vocab,
         "probs": probs, "drafts": drafts}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One chat turn with a small tree of drafts, 16 heads on this GPU: all latency.
        _case("tree_b1_h16_n8", "tree", heads=16, nodes=8, ctx=(300, 300)),
        # A lightly loaded server on the paper's page with protection, trees of different sizes.
        _case("tree_b4_h128_n26_c4r4_protected", "tree", "c4r4", True, 4, 128, 26, 11, 3, (1500, 6000)),
        # Wide trees over long documents, heads sharded to 64, INT2.
        _case("tree_b2_h64_n64_int2_30k", "tree", "int2", False, 2, 64, 64, 64, 4, (21001, 30000)),
        # Sixteen conversations, 16 heads on this GPU, the unquantised cache.
        _case("tree_b16_h16_n25_bf16", "tree", "bf16", False, 16, 16, 25, 9, 3, (700, 9001)),
        # The DeepSeek-V3-shaped serving batch with three drafts a sequence.
        _case("tree_b64_h128_n4_4k", "tree", "int4", False, 64, 128, 4, 4, 2, (4096, 4096)),
        # All 128 heads, thirty-one drafts for each of sixteen sequences: the largest.
        _case("tree_b16_h128_n32_4k", "tree", "int4", False, 16, 128, 32, 32, 3, (4096, 4096)),
        # One sequence with a chain of seven drafts: all latency.
        _case("settle_b1_n8_chain", "settle", nodes=8, branch=1, ctx=(300, 300), vocab=32000),
        # The serving batch with protection on the paper's page, trees of fifteen drafts, a large vocabulary.
        _case("settle_b64_n16_128k", "settle", "c4r4", True, 64, 16, 16, 7, 3, (100, 1500), vocab=131072),
        # Large trees, an odd vocabulary, probabilities kept in bf16.
        _case("settle_b16_n64_bf16_50001", "settle", "int2", False, 16, 16, 64, 40, 4, (90, 1203), vocab=50001,
              probs="bf16"),
        # Many sequences with drafts looked up in their own text (no draft probabilities), unquantised cache.
        _case("settle_b128_n6_certain", "settle", "bf16", False, 128, 16, 6, 1, 2, (37, 900), vocab=100003,
              drafts="certain"),
    ]


_MAX_PAIRS = 16 * 32 * 128 * 4128  # rows x keys of the largest listed attention
_MAX_ROWS = 16 * 32 * 128
_MAX_PROBS = 64 * 16 * 131072


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    cache = rng.choice(["int4", "int4", "int2", "c4r4", "bf16"])
    protect = cache != "bf16" and rng.random() < 0.4
    nodes, branch = _log_int(rng, 1, MAX_NODES), rng.choice([1, 2, 3, 4, 7])
    few = nodes if rng.random() < 0.5 else rng.randint(1, nodes)
    if rng.random() < 0.55:
        heads, batch = rng.choice([16, 20, 32, 64, 100, 128, 128]), _log_int(rng, 1, 64)
        while batch * heads * nodes > _MAX_ROWS:
            batch = max(1, batch * 3 // 4)
        hi = _log_int(rng, 200, 40000)
        while batch * heads * nodes * (hi + nodes) > _MAX_PAIRS:
            hi = max(200, hi * 3 // 4)
            batch = max(1, batch * 7 // 8)
        return _case(None, "tree", cache, protect, batch, heads, nodes, few, branch, (rng.randint(200, hi), hi))
    vocab, batch = _log_int(rng, 1000, 200000), _log_int(rng, 1, 128)
    while batch * nodes * vocab > _MAX_PROBS:
        batch, vocab = max(1, batch * 3 // 4), max(1000, vocab * 7 // 8)
    hi = _log_int(rng, 1, 2000)
    return _case(None, "settle", cache, protect, batch, 16, nodes, few, branch, (rng.randint(0, hi), hi), vocab,
                 rng.choice(["f32", "f32", "bf16"]), rng.choice(["sampled", "sampled", "certain"]))


# ---------------------------------------------------------------- inputs
def _spread(lo, hi, batch, step):
    """batch values from lo to hi, both ends taken, in a scattered order."""
    if batch == 1:
        return [hi]
    return [lo + ((i * (hi - lo)) // (batch - 1)) for i in sorted(range(batch), key=lambda i: (i * step) % 1.0)]


def _sizes(case):
    """(nodes, context tokens) of each sequence."""
    return (_spread(case["few"], case["nodes"], case["batch"], 0.6180339887),
            _spread(case["ctx_lo"], case["ctx_hi"], case["batch"], 0.4142135624))


def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1_000_003 + stream)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rows(counts, first):
    """(sequence, position) of counts[b] tokens from position first[b] on, sequence by sequence."""
    n = torch.tensor(counts, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), n, output_size=sum(counts))
    at = torch.arange(sum(counts), device="cuda") - (torch.cumsum(n, 0) - n)[seq]
    return seq, at + torch.tensor(first, device="cuda")[seq]


def _draw_rows(case, seed, stream, n):
    """n rows as the cache takes them: 512 latent channels and 64 of the RoPE key."""
    g = _gen(seed, stream)
    gain = torch.exp(0.5 * torch.randn(DC, generator=_gen(seed, 1), device="cuda"))
    gain[torch.randperm(DC, generator=_gen(seed, 2), device="cuda")[:4]] *= 8.0
    x = torch.randn(n, ROW, generator=g, device="cuda")
    x[:, :DC] *= gain
    return x.bfloat16()


def _draw_parents(case, seed):
    """Each node's parent: about `branch` children a node, the earliest nodes first, jittered."""
    t = torch.arange(case["nodes"], device="cuda").expand(case["batch"], -1)
    if case["branch"] == 1:
        return (t - 1).int().contiguous()
    back = torch.randint(0, 2, t.shape, generator=_gen(seed, 3), device="cuda")
    return torch.where(t == 0, t - 1, ((t - 1) // case["branch"] - back).clamp_min(0)).int()


def _parts(case, nblocks):
    """(offset, groups, bytes a slot) of the regions [groups][64 slots][bytes] of a block."""
    if case["cache"] == "bf16":
        return [(0, 1, 1152)]
    cb = 16 if case["cache"] == "int2" else 32
    if case["cache"] == "c4r4":
        return [(0, 8, 32), (16384, 1, 32), (18432, 8, 2), (19456, 1, 4), (19712, 9, 1)]
    return [(0, 8, cb), (512 * cb, 1, 32), (512 * cb + 2048, 9, 4)]


def _views(case, pool):
    n = pool.size(0)
    return [pool[:, o:o + g * BLOCK * w].view(n, g, BLOCK, w) for o, g, w in _parts(case, n)]


def _quantise(case, x, bits, content):
    """Codes, scales and zero points of groups x [n, groups, 64]."""
    m = float(2 ** bits - 1)
    x = x.double()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = ((hi - lo).float().clamp_min(1e-8).double() / m).float()
    s = s if case["cache"] == "c4r4" and not content else s.bfloat16() if case["cache"] == "c4r4" else s.half()
    s = s.double().clamp(2.0 ** -24, 65504.0)
    z = torch.round(-lo / s).clamp(0, m)
    return torch.round(x / s + z).clamp(0, m).to(torch.uint8), s, z


def _pack(q, bits):
    if bits == 4:
        return q[..., 0::2] | (q[..., 1::2] << 4)
    return q[..., 0::4] | (q[..., 1::4] << 2) | (q[..., 2::4] << 4) | (q[..., 3::4] << 6)


def _as_bytes(x, dtype):
    return x.to(dtype).contiguous().view(torch.uint8)


def _write(case, st, x, seq, pos):
    """What the writers leave in the cache for rows x of these sequences and positions."""
    blk, slot = st["table"][seq, pos // BLOCK].long(), pos % BLOCK
    if case["cache"] == "bf16":
        parts = [x.contiguous().view(torch.uint8).view(-1, 1, 1152)]
    else:
        bits = 2 if case["cache"] == "int2" else 4
        cq, cs, cz = _quantise(case, x[:, :DC].reshape(-1, 8, 64), bits, True)
        rq, rs, rz = _quantise(case, x[:, DC:].reshape(-1, 1, 64), 4, False)
        parts = [_pack(cq, bits), _pack(rq, 4)]
        if case["cache"] == "c4r4":
            parts += [_as_bytes(cs, torch.bfloat16), _as_bytes(rs, torch.float32),
                      torch.cat([cz, rz], 1).to(torch.uint8)]
        else:
            parts += [_as_bytes(torch.cat([torch.cat([cs, cz], -1), torch.cat([rs, rz], -1)], 1), torch.float16)]
    for view, p in zip(_views(case, st["pool"]), parts):
        view[blk, :, slot] = p


def prepare(case, seed):
    """The cache, trees, queries or probabilities, and buffers that a serving program holds."""
    B, T = case["batch"], case["nodes"]
    nodes, ctx = _sizes(case)
    ends = [a + b for a, b in zip(nodes, ctx)]
    nblk = [max(1, -(-n // BLOCK)) for n in ends]
    perm = torch.randperm(sum(nblk), generator=_gen(seed, 4), device="cuda").int()
    table = torch.full((B, max(nblk)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(nblk):
        table[b, :n] = perm[at:at + n]
        at += n
    st = {"case": case, "table": table, "lens": _ints(ends), "counts": _ints(nodes),
          "parents": _draw_parents(case, seed), "err": _ints([0]),
          "pool": torch.zeros((sum(nblk), BLOCK_BYTES[case["cache"]]), dtype=torch.uint8, device="cuda"),
          "prot": None, "drafts": None}
    seq, pos = _rows(nodes, ctx)
    x = _draw_rows(case, seed, 5, sum(nodes))
    _write(case, st, x, seq, pos)
    if case["protect"]:
        st["prot"] = torch.zeros((B, 132, ROW), dtype=torch.bfloat16, device="cuda")
        st["drafts"] = torch.zeros((B, MAX_NODES, ROW), dtype=torch.bfloat16, device="cuda")
        st["drafts"][seq, pos - torch.tensor(ctx, device="cuda")[seq]] = x
    if case["kind"] == "tree":
        seq, pos = _rows(ctx, [0] * B)
        for i in range(0, seq.numel(), 1 << 16):  # what earlier calls wrote
            s, p = seq[i:i + (1 << 16)], pos[i:i + (1 << 16)]
            x = _draw_rows(case, seed, 100 + (i >> 16), s.numel())
            _write(case, st, x, s, p)
            if case["protect"]:
                late, sink = p >= torch.tensor(ctx, device="cuda")[s] - 128, p < 4
                st["prot"][s[late], 4 + p[late] % 128] = x[late]
                st["prot"][s[sink], p[sink]] = x[sink]
        g, H = _gen(seed, 6), case["heads"]
        st["q"] = (0.5 * torch.randn(B, T, H, DC, generator=g, device="cuda")).bfloat16()
        st["q_pe"] = torch.randn(B, T, H, DR, generator=g, device="cuda").bfloat16()
        st["out"] = torch.zeros((B, T, H, DC), dtype=torch.bfloat16, device="cuda")
        st["lse"] = torch.zeros((B, T, H), dtype=torch.float32, device="cuda")
        st["ws"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
        return st
    V, kind = case["vocab"], torch.float32 if case["probs"] == "f32" else torch.bfloat16
    target = torch.empty((B, T, V), dtype=kind, device="cuda")
    draft = torch.empty((B, T, V), dtype=kind, device="cuda") if case["drafts"] == "sampled" else None
    tokens = torch.zeros((B, T), dtype=torch.int32, device="cuda")
    parents = st["parents"].long().clamp_min(0)
    for b in range(B):
        g = _gen(seed, 1000 + b)
        d = 2.5 * torch.randn(T, V, generator=g, device="cuda")
        target[b] = torch.softmax(d + 0.7 * torch.randn(T, V, generator=g, device="cuda"), -1).to(kind)
        if draft is not None:
            draft[b] = torch.softmax(d, -1).to(kind)
        cut = torch.rand(T, 1, generator=g, device="cuda")  # each node's token, from its parent's distribution
        tokens[b] = torch.searchsorted(torch.cumsum(torch.softmax(d, -1), -1)[parents[b]], cut)[:, 0].clamp_max(V - 1).int()
    st.update(target=target, draft=draft, tokens=tokens,
              uniforms=torch.rand(B, T, generator=_gen(seed, 7), device="cuda"),
              path=torch.zeros((B, T), dtype=torch.int32, device="cuda"), kept=_ints([0] * B), next=_ints([0] * B),
              new_lens=_ints([0] * B))
    return st


# ---------------------------------------------------------------- plain forms
def _plain_read(case, st, longest):
    """The cached rows [batch, longest, 576] in 32 bits (rows behind a sequence's end hold anything finite)."""
    B = case["batch"]
    pos = torch.arange(longest, device="cuda").expand(B, -1)
    seq = torch.arange(B, device="cuda")[:, None].expand_as(pos)
    blk, slot = st["table"][seq, pos // BLOCK].long().clamp_min(0), pos % BLOCK
    got = [v[blk, :, slot] for v in _views(case, st["pool"])]
    if case["cache"] == "bf16":
        return got[0].reshape(B, longest, 1152).view(torch.bfloat16).float()
    nib = lambda p: torch.stack([p & 15, p >> 4], -1).flatten(-2)  # noqa: E731
    crumb = lambda p: torch.stack([p & 3, (p >> 2) & 3, (p >> 4) & 3, p >> 6], -1).flatten(-2)  # noqa: E731
    c, r = (crumb if case["cache"] == "int2" else nib)(got[0]).float(), nib(got[1]).float()
    if case["cache"] == "c4r4":
        cs, rs = got[2].contiguous().view(torch.bfloat16).float(), got[3].contiguous().view(torch.float32)
        cz, rz = got[4][..., :8, :].float(), got[4][..., 8:, :].float()
    else:
        sz = got[2].contiguous().view(torch.float16).float()
        cs, cz, rs, rz = sz[..., :8, :1], sz[..., :8, 1:], sz[..., 8:, :1], sz[..., 8:, 1:]
    x = torch.cat([(cs * (c - cz)).flatten(-2), (rs * (r - rz)).flatten(-2)], -1)
    if case["protect"]:
        ctx = (st["lens"] - st["counts"]).long()[:, None]
        kept = (pos < ctx) & ((pos < 4) | (pos >= ctx - 128))
        x = torch.where(kept[..., None], st["prot"][seq, torch.where(pos < 4, pos, 4 + pos % 128)].float(), x)
        node = pos - ctx
        x = torch.where((node >= 0)[..., None], st["drafts"][seq, node.clamp(0, MAX_NODES - 1)].float(), x)
    return x


def _plain_sees(st, longest):
    """Which positions each node sees [batch, nodes, longest]: the context, its ancestors and itself."""
    B, T = st["parents"].shape
    d = st["parents"].device
    t = torch.arange(T, device=d)
    step = ((st["parents"][..., None] == t) | (t[:, None] == t)).float()
    for _ in range(6):  # paths of up to 64 steps
        step = (step @ step > 0).float()
    node = torch.arange(longest, device=d) - (st["lens"] - st["counts"])[:, None]
    tree = step.gather(-1, node.clamp(0, T - 1)[:, None].expand(B, T, longest)) > 0
    sees = (node < 0)[:, None] | (tree & (node < st["counts"][:, None])[:, None])
    return sees & (t < st["counts"][:, None])[..., None]


def _plain_tree(st):
    case = st["case"]
    B, T, H, longest = case["batch"], case["nodes"], case["heads"], max(a + b for a, b in zip(*_sizes(case)))
    x = _plain_read(case, st, longest)
    s = torch.matmul(torch.cat([st["q"], st["q_pe"]], -1).float().view(B, T * H, ROW), x.transpose(-1, -2))
    s = s.view(B, T, H, longest).mul_(TAU)
    s.masked_fill_(~_plain_sees(st, longest)[:, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s -= torch.where(torch.isinf(top), torch.zeros_like(top), top)
    s.exp_()
    den = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, T * H, longest), x[..., :DC]).view(B, T, H, DC)
    o = torch.where(den > 0, o / den, torch.zeros_like(den))
    return {"out": o.bfloat16(), "lse": (top + torch.log(den)).squeeze(-1)}


def _plain_verify(st):
    """The walk of all trees side by side, in 64 bits: nodes are looked at in their order, which meets a node's
    children after it and each before its later siblings."""
    target, draft = st["target"], st["draft"]
    B, T, V = target.shape
    d = target.device
    b, tokens, parents = torch.arange(B, device=d), st["tokens"].long(), st["parents"].long()
    u = st["uniforms"].double()
    live = st["counts"] > 0
    cur = torch.zeros(B, dtype=torch.long, device=d)
    a, mass = torch.zeros(B, dtype=torch.float64, device=d), torch.ones(B, dtype=torch.float64, device=d)
    gone = torch.zeros((B, V), dtype=torch.bool, device=d)
    path, kept = torch.full((B, T), -1, device=d), live.long()
    path[:, 0] = torch.where(live, 0, -1)

    def left(a):
        p = target[b, cur].double()
        return torch.where(gone, 0.0, p) if draft is None else (p - a[:, None] * draft[b, cur].double()).clamp_min(0)

    for t in range(1, T):
        x, asked = tokens[:, t], live & (t < st["counts"]) & (parents[:, t] == cur)
        p = target[b, cur, x].double()
        if draft is None:
            p = torch.where(gone[b, x], 0.0, p)
            ok = u[:, t] * mass < p
        else:
            q = draft[b, cur, x].double()
            p = (p - a * q).clamp_min(0)
            ok = u[:, t] * q * mass < p
        took, lost = asked & ok, asked & ~ok
        if draft is None:
            gone[b, x] |= lost
            mass = torch.where(lost, mass - p, mass)
            gone &= ~took[:, None]
        else:
            a = torch.where(lost, a + mass, a)
            mass = torch.where(lost, left(a).sum(-1), mass)
            a = torch.where(took, 0.0, a)
        mass = torch.where(took, 1.0, mass)
        path.scatter_(1, torch.where(took, kept, T - 1)[:, None],
                      torch.where(took, t, path[:, T - 1])[:, None])
        kept, cur = kept + took, torch.where(took, t, cur)
    r = left(a)
    c = torch.cumsum(r, -1)
    over = c > u[:, :1] * c[:, -1:]
    last = V - 1 - torch.argmax((r > 0).flip(-1).int(), -1)
    pick = torch.where(over.any(-1), torch.argmax(over.int(), -1), last)
    return path.int(), kept.int(), torch.where(live, pick, -1).int()


def _plain_keep(case, st, path, kept):
    """Accepted nodes' bytes moved together, all read before any is written."""
    B, T = path.shape
    ctx = (st["lens"] - st["counts"]).long()[:, None]
    i = torch.arange(T, device="cuda").expand(B, -1)
    mine = i < kept[:, None]
    still = (ctx + 0 * i).clamp(0, st["table"].size(1) * BLOCK - 1)  # an entry that moves nothing copies a row on itself
    still = torch.where(st["counts"][:, None] > 0, still, (still - 1).clamp_min(0))
    src, dst = torch.where(mine, ctx + path, still), torch.where(mine, ctx + i, still)
    seq = torch.arange(B, device="cuda")[:, None]
    sb, db = st["table"][seq, src // BLOCK].long(), st["table"][seq, dst // BLOCK].long()
    for view in _views(case, st["pool"]):
        view[db, :, dst % BLOCK] = view[sb, :, src % BLOCK]
    if case["protect"]:
        rows = st["drafts"][seq, path.long().clamp_min(0)]
        wide = torch.cat([st["prot"], torch.zeros_like(st["prot"][:, :1])], 1)  # row 132: written by nobody else
        wide[seq, torch.where(mine & (dst < 4), dst, 132)] = rows
        wide[seq, torch.where(mine, 4 + dst % 128, 132)] = rows
        st["prot"].copy_(wide[:, :132])
    return (ctx[:, 0] + kept).int()


def run(st):
    case = st["case"]
    if own:
        return _own(case, st)
    if case["kind"] == "tree":
        return _plain_tree(st)
    path, kept, token = _plain_verify(st)
    got = {"path": path, "kept": kept, "next": token, "lens": _plain_keep(case, st, path, kept), "pool": st["pool"]}
    if case["protect"]:
        got["prot"] = st["prot"]
    return got


def _own(case, st):
    import paper_2609_36760_gb300 as Q
    cache = {"int4": 4, "int2": 2}.get(case["cache"], case["cache"])
    if case["kind"] == "tree":
        Q.mla_decode_tree(st["pool"], cache, st["q"], st["q_pe"], st["table"], st["lens"], st["parents"], TAU,
                          st["out"], st["lse"], st["ws"], st["err"], tree_lens=st["counts"], prot=st["prot"],
                          draft_rows=st["drafts"])
        return {"out": st["out"], "lse": st["lse"]}
    Q.tree_verify(st["target"], st["draft"], st["tokens"], st["parents"], st["uniforms"], st["path"], st["kept"],
                  st["next"], st["err"], tree_lens=st["counts"])
    Q.cache_keep(st["pool"], cache, st["table"], st["lens"], st["path"], st["kept"], st["new_lens"], st["err"],
                 tree_lens=st["counts"], prot=st["prot"], draft_rows=st["drafts"])
    got = {"path": st["path"], "kept": st["kept"], "next": st["next"], "lens": st["new_lens"], "pool": st["pool"]}
    if case["protect"]:
        got["prot"] = st["prot"]
    return got


def work(case):
    B, T, H = case["batch"], case["nodes"], case["heads"]
    nodes, ctx = _sizes(case)
    if case["kind"] == "tree":
        # every node over the context and, of a tree of n nodes, its path: log n of them at least
        pairs = sum(H * n * (c + 1 + int(math.log2(n))) for n, c in zip(nodes, ctx))
        return {"bytes": sum(ctx) * TOKEN_BYTES[case["cache"]] + sum(nodes) * (2 * ROW if case["protect"] else TOKEN_BYTES[case["cache"]])
                + sum(nodes) * H * 2 * ROW + B * T * H * (2 * DC + 4), "flops": 2 * (ROW + DC) * pairs}
    # the target's and, where a draft is refused, the draft's probabilities of the node where a walk ends; two
    # values a node, tokens, parents and random numbers; the accepted tokens' rows are a few
    size = 4 if case["probs"] == "f32" else 2
    rows = 2 if case["drafts"] == "sampled" else 1
    return {"bytes": B * rows * case["vocab"] * size + sum(nodes) * (2 * size + 12) + B * T * 4 + B * 16,
            "flops": B * 3 * case["vocab"]}


# ---------------------------------------------------------------- 64-bit values
def _exact_rows(case, st, b, n):
    """Rows 0 .. n - 1 of sequence b as attention sees them."""
    blk = st["table"][b, :-(-n // BLOCK)].long()
    v = [x[blk].permute(0, 2, 1, 3).reshape(-1, g, w)[:n] for x, (_, g, w) in zip(_views(case, st["pool"]), _parts(case, 0))]
    if case["cache"] == "bf16":
        return v[0].reshape(n, -1).contiguous().view(torch.bfloat16).double()
    per = 4 if case["cache"] == "int2" else 2
    bits = torch.arange(per, device="cuda") * (8 // per)
    code = ((v[0].long()[..., None] >> bits) & (2 ** (8 // per) - 1)).reshape(n, 8, 64).double()
    key = ((v[1].long()[..., None] >> torch.tensor([0, 4], device="cuda")) & 15).reshape(n, 1, 64).double()
    if case["cache"] == "c4r4":
        s, z = v[2].contiguous().view(torch.bfloat16).double(), v[4].double()
        parts = [(code - z[:, :8]) * s, (key - z[:, 8:]) * v[3].contiguous().view(torch.float32).double()]
    else:
        m = v[2].contiguous().view(torch.float16).double()
        parts = [(code - m[:, :8, 1:]) * m[:, :8, :1], (key - m[:, 8:, 1:]) * m[:, 8:, :1]]
    return torch.cat([p.reshape(n, -1) for p in parts], 1)


def exact(case, seed):
    if case["kind"] != "tree":
        return None  # whole numbers and moved bytes
    st = prepare(case, seed)
    B, T, H = case["batch"], case["nodes"], case["heads"]
    out = torch.zeros(B, T, H, DC, dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, H), -math.inf, dtype=torch.float64, device="cuda")
    parents = st["parents"].tolist()
    for b, (n, c) in enumerate(zip(*_sizes(case))):
        x = _exact_rows(case, st, b, c + n)
        if case["protect"]:
            for p in [*range(min(4, c)), *range(max(0, c - 128), c)]:
                x[p] = st["prot"][b, p if p < 4 else 4 + p % 128].double()
            x[c:] = st["drafts"][b, :n].double()
        for t in range(n):
            line, at = [], t
            while at >= 0:
                line.append(c + at)
                at = parents[b][at]
            keys = torch.cat([x[:c], x[line]])
            z = TAU * (st["q"][b, t].double() @ keys[:, :DC].T + st["q_pe"][b, t].double() @ keys[:, DC:].T)
            lse[b, t] = torch.logsumexp(z, -1)
            out[b, t] = torch.softmax(z, -1) @ keys[:, :DC]
    return {"out": out, "lse": lse}
