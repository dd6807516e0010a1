"""A step of speculative decoding as a program runs it: the nodes' rows written (their keys turned by
their own depth), attended to, verified, and the accepted ones kept. The cache then has to be, byte
for byte, the one of a program that wrote the accepted tokens one after the other, and so its next
decode. Also the writer with angle positions of their own, and the calls' refusals on the device."""
import numpy as np
import pytest
import torch

import paper_2609_36760_gb300 as Q
from oracle import speculation as OS
from speculation_cases import KINDS, TAU, WIDTH, distributions, drafted, queries, trees
from test_gpu_rows import normed, rotated, table_of

pytestmark = pytest.mark.gpu


def depths(parents):
    B, T = parents.shape
    d = torch.zeros(B, T, dtype=torch.int32)
    for t in range(1, T):
        d[:, t] = torch.gather(d, 1, parents[:, t:t + 1].long().clamp_min(0))[:, 0] + 1
    return d


@pytest.mark.parametrize("kind,protect", [(4, False), (4, True), (2, True), ("c4r4", True), ("c4r4", False), ("bf16", False)])
@pytest.mark.parametrize("heads", [16, 128])
def test_steps_leave_the_cache_of_the_accepted_tokens(kind, protect, heads):
    B, T, V, steps = 3, 11, 211, 3
    g = torch.Generator().manual_seed(heads)
    lens = [0, 125, 190]
    cols = 6
    table = torch.randperm(B * cols, generator=g).int().view(B, cols).cuda()
    cs = table_of(400).cuda()
    weight = (1 + 0.2 * torch.randn(512, generator=g)).bfloat16().cuda()
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731

    class Side:
        def __init__(self):
            self.pool = torch.zeros((B * cols, WIDTH[kind]), dtype=torch.uint8, device="cuda")
            self.prot = torch.zeros((B, 132, 576), dtype=torch.bfloat16, device="cuda") if protect else None

    tree, plain = Side(), Side()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    scratch = torch.zeros((B, 73728), dtype=torch.uint8, device="cuda")  # the nodes' rows: a bf16 block a sequence
    draft_rows = scratch.view(torch.bfloat16).view(B, 64, 576) if protect else None

    def write(side, rows, seq, pos, after=None, **kw):
        Q.rope_append(side.pool, kind, rows[:, :512], rows[:, 512:], i32(seq), i32(pos), table, cs, err, norm_weight=weight,
                      seq_lens=None if after is None else i32(after), prot=None if after is None else side.prot, **kw)

    prompt = [torch.randn(n, 576, generator=g).bfloat16() for n in lens]
    x = torch.cat(prompt).cuda()
    seq = [b for b, n in enumerate(lens) for _ in range(n)]
    pos = [p for n in lens for p in range(n)]
    for side in (tree, plain):
        write(side, x, seq, pos, lens if protect else None)
    seq_lens, new_lens = i32(lens), i32([0] * B)
    path, kept, nxt = i32(np.zeros((B, T))), i32([0] * B), i32([0] * B)
    ws = torch.empty(Q.tree_workspace_bytes(B, T, heads, 64 * cols), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        parents = trees("any", B, T, step)
        dep = depths(parents)
        rows = torch.randn(B * T, 576, generator=g).bfloat16().cuda()
        ctx = torch.tensor(lens)
        at = (ctx[:, None] + torch.arange(T)).reshape(-1)
        turn = (ctx[:, None] + dep).reshape(-1)
        node_seq = torch.arange(B).repeat_interleave(T)
        write(tree, rows, node_seq, at, rope_positions=i32(turn))
        if protect:
            Q.rope_append(scratch, "bf16", rows[:, :512], rows[:, 512:], i32(node_seq), i32(torch.arange(T).repeat(B)),
                          i32(torch.arange(B)[:, None]), cs, err, norm_weight=weight, rope_positions=i32(turn))
        seq_lens.copy_(i32(ctx + T))
        q, q_pe = (y.cuda() for y in queries(B, T, heads, step))
        Q.rope_query(q_pe.view(B * T, heads, 64), i32(turn), cs, q_pe.view(B * T, heads, 64), err)
        out = torch.empty((B, T, heads, 512), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((B, T, heads), device="cuda")
        Q.mla_decode_tree(tree.pool, kind, q, q_pe, table, seq_lens, i32(parents), TAU, out, lse, ws, err, prot=tree.prot,
                          draft_rows=draft_rows)
        target, draft = distributions(B, T, V, step)
        tokens, u = drafted(draft, parents, step), torch.rand(B, T, generator=g)
        Q.tree_verify(target.cuda(), draft.cuda(), tokens.cuda(), i32(parents), u.cuda(), path, kept, nxt, err)
        Q.cache_keep(tree.pool, kind, table, seq_lens, path, kept, new_lens, err, prot=tree.prot, draft_rows=draft_rows)
        torch.cuda.synchronize()
        assert Q.read_dev_err(err) == 0
        # the other program: the accepted tokens one after the other
        took = kept.cpu().tolist()
        for b in range(B):
            want, want_next = OS.verify_tree(target[b], draft[b], tokens[b].tolist(), parents[b].tolist(), T, u[b])
            assert path[b, :took[b]].tolist() == want and int(nxt[b]) == want_next
            for i, node in enumerate(want):
                after = [lens[c] + (i + 1 if c == b else 0) for c in range(B)]
                write(plain, rows[b * T + node:b * T + node + 1], [b], [lens[b] + i], after if protect else None)
            lens[b] += took[b]
        assert new_lens.tolist() == lens
        one, two = (torch.empty((sum(lens), 576), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        seq = i32([b for b, n in enumerate(lens) for _ in range(n)])
        pos = i32([p for n in lens for p in range(n)])
        for side, rows_out in ((tree, one), (plain, two)):
            Q.cache_read(side.pool, kind, seq, pos, table, rows_out, err, seq_lens=new_lens if protect else None,
                         prot=side.prot)
        outs = []
        for side in (tree, plain):
            o = torch.empty((B, heads, 512), device="cuda")
            Q.mla_decode_ex(side.pool, kind, q[:, 0].contiguous(), q_pe[:, 0].contiguous(), table, new_lens, TAU, o, None,
                            Q.workspace_for(B, heads), err, prot=side.prot)
            outs.append(o)
        torch.cuda.synchronize()
        assert Q.read_dev_err(err) == 0
        assert torch.equal(one, two) and torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 7, 300, 4300])
@pytest.mark.parametrize("interleaved", [False, True])
def test_angle_positions_of_their_own(kind, n, interleaved):
    g = torch.Generator().manual_seed(n)
    rows = torch.randn(n, 576, generator=g).bfloat16()
    cs = table_of(700)
    turn = torch.randint(0, 700, (n,), generator=g).int()
    pos = torch.arange(n, dtype=torch.int32)
    cols = -(-n // 64)
    table = torch.randperm(cols, generator=g).int().view(1, cols)
    x = torch.cat([normed(rows[:, :512], None, 1e-6), rotated(rows[:, 512:], cs, turn, interleaved)], 1).cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, want = (torch.zeros((cols, WIDTH[kind]), dtype=torch.uint8, device="cuda") for _ in range(2))
    seq = torch.zeros(n, dtype=torch.int32).cuda()
    lat, kpe = x[:, :512].contiguous(), x[:, 512:].contiguous()
    if kind == "bf16":
        Q.bf16_append(want, lat, kpe, seq, pos.cuda(), table.cuda(), err)
    elif kind == "c4r4":
        Q.quant_append_c4r4(want, lat, kpe, seq, pos.cuda(), table.cuda(), err)
    else:
        Q.quant_append(want, kind, lat, kpe, seq, pos.cuda(), table.cuda(), err)
    r = rows.cuda()
    Q.rope_append(got, kind, r[:, :512], r[:, 512:], seq, pos.cuda(), table.cuda(), cs.cuda(), err, norm=True,
                  interleaved=interleaved, rope_positions=turn.cuda())
    assert Q.read_dev_err(err) == 0 and torch.equal(got, want)


@pytest.mark.parametrize("n", [5, 4300])
def test_bad_angle_positions_are_not_written(n):
    rows = torch.randn(n, 576).bfloat16().cuda()
    cols = -(-n // 64)
    table = torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
    turn = torch.zeros(n, dtype=torch.int32)
    turn[1], turn[3] = -1, 64
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    pool = torch.full((cols, 73728), 7, dtype=torch.uint8, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    Q.rope_append(pool, "bf16", rows[:, :512], rows[:, 512:], torch.zeros_like(pos), pos, table, table_of(64).cuda(), err,
                  rope_positions=turn.cuda())
    assert Q.read_dev_err(err) == Q.DEVERR_BAD_POSITION
    slots = pool.view(-1, 1152)[:n].cpu()
    assert (slots[[1, 3]] == 7).all() and not (slots[[0, 2, 4]] == 7).all(1).any()


def test_the_binding_refuses_other_devices_types_and_shapes():
    B, T = 2, 4
    dev = dict(device="cuda")
    i = lambda *s: torch.zeros(s, dtype=torch.int32, **dev)  # noqa: E731
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16, **dev)  # noqa: E731
    pool = torch.zeros((3, 20736), dtype=torch.uint8, **dev)

    def tree(**kw):
        a = dict(pool=pool, cache_kind=4, q_latent=b(B, T, 8, 512), q_pe=b(B, T, 8, 64), block_table=i(B, 3), seq_lens=i(B),
                 parents=i(B, T), softmax_scale=0.1, out=b(B, T, 8, 512), lse=None, dev_err=None,
                 workspace=torch.zeros(Q.tree_workspace_bytes(B, T, 8), dtype=torch.uint8, **dev))
        Q.mla_decode_tree(**{**a, **kw})

    def verify(**kw):
        a = dict(target=torch.ones(B, T, 30, **dev), draft=None, tokens=i(B, T), parents=i(B, T),
                 uniforms=torch.zeros(B, T, **dev), path=i(B, T), kept=i(B), next_token=i(B), dev_err=None)
        Q.tree_verify(**{**a, **kw})

    def keep(**kw):
        a = dict(pool=pool, cache_kind=4, block_table=i(B, 3), seq_lens=i(B), path=i(B, T), kept=i(B), new_lens=i(B),
                 dev_err=None)
        Q.cache_keep(**{**a, **kw})

    tree(), verify(), keep()
    torch.cuda.synchronize()
    for call, kw, word in (
            (tree, {"q_pe": b(B, T, 8, 32)}, "q_pe"), (tree, {"block_table": i(3, 3), "seq_lens": i(3)}, "block_table"),
            (tree, {"parents": i(B, T + 1)}, "parents"), (tree, {"parents": i(B, T).long()}, "parents"),
            (tree, {"parents": i(B, T).cpu()}, "device"), (tree, {"tree_lens": i(B + 1)}, "tree_lens"),
            (tree, {"out": torch.zeros(B, T, 8, 512, **dev)}, "out"), (tree, {"out": b(B, 8, T, 512).transpose(1, 2)}, "out"),
            (tree, {"lse": b(B, T, 8)}, "lse"), (tree, {"draft_rows": b(B, T, 576)}, "draft_rows"),
            (tree, {"prot": b(B, 132, 512)}, "prot"),
            (verify, {"draft": torch.ones(B, T, 31, **dev)}, "draft"), (verify, {"draft": b(B, T, 30)}, "draft"),
            (verify, {"target": torch.ones(B, 30, T, **dev).transpose(1, 2)}, "target"),
            (verify, {"tokens": i(B, T).long()}, "tokens"), (verify, {"uniforms": torch.zeros(B, T + 1, **dev)}, "uniforms"),
            (verify, {"path": i(B, T, 1)}, "path"), (verify, {"kept": i(1)}, "kept"), (verify, {"next_token": i(B).cpu()}, "device"),
            (keep, {"kept": i(B + 1)}, "kept"), (keep, {"path": i(B + 1, T)}, "path"), (keep, {"new_lens": i(1)}, "new_lens")):
        with pytest.raises(ValueError, match=word):
            call(**kw)
    for kw in ({"prot": b(B, 132, 576)}, {"draft_rows": b(B, 64, 576)}):
        for call in (tree, keep):
            with pytest.raises(Q.QmlaError, match="invalid"):
                call(**kw)


@pytest.mark.parametrize("kind,protect", [(4, False), ("c4r4", True)])
def test_a_step_captured_as_one_graph(kind, protect):
    """Writer, attention, verification and move in one graph (their launches overlap), replayed with new
    rows, trees, lengths and probabilities in place; against the same calls one by one."""
    B, T, H, V, cols = 4, 9, 32, 1001, 8
    g = torch.Generator().manual_seed(5)
    cs = table_of(600).cuda()
    table = torch.randperm(B * cols, generator=g).int().view(B, cols).cuda()
    ctx = [0, 100, 190, 300]
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    err = i32([0])

    def fresh():
        d = {"pool": torch.zeros((B * cols, WIDTH[kind]), dtype=torch.uint8, device="cuda"),
             "prot": torch.zeros((B, 132, 576), dtype=torch.bfloat16, device="cuda") if protect else None,
             "drafts": torch.zeros((B, 64, 576), dtype=torch.bfloat16, device="cuda"),
             "out": torch.zeros((B, T, H, 512), dtype=torch.bfloat16, device="cuda"), "path": i32(np.zeros((B, T))),
             "kept": i32([0] * B), "next": i32([0] * B), "new": i32([0] * B)}
        gen = torch.Generator().manual_seed(9)
        n = max(ctx)
        for b, c in enumerate(ctx):
            x = torch.randn(n, 576, generator=gen).bfloat16()[:c].cuda()
            if c:
                lens = i32(ctx)
                Q.rope_append(d["pool"], kind, x[:, :512], x[:, 512:], i32([b] * c), i32(range(c)), table, cs, err,
                              seq_lens=lens if protect else None, prot=d["prot"])
        return d

    def inputs(seed):
        gen = torch.Generator().manual_seed(seed)
        parents = trees("any", B, T, seed)
        target, draft = distributions(B, T, V, seed)
        c = torch.tensor(ctx)
        q, q_pe = queries(B, T, H, seed)
        return [torch.randn(B * T, 576, generator=gen).bfloat16().cuda(), i32(parents), target.cuda(), draft.cuda(),
                drafted(draft, parents, seed).cuda(), torch.rand(B, T, generator=gen).cuda(), q.cuda(), q_pe.cuda(),
                i32((c[:, None] + torch.arange(T)).reshape(-1)), i32((c[:, None] + depths(parents)).reshape(-1)), i32(c + T)]

    seq, node = i32(torch.arange(B).repeat_interleave(T)), i32(torch.arange(T).repeat(B))
    own = i32(torch.arange(B)[:, None])
    ws = torch.empty(Q.tree_workspace_bytes(B, T, H, 64 * cols), dtype=torch.uint8, device="cuda")

    def step(d, x):
        rows, parents, target, draft, tokens, u, q, q_pe, at, turn, lens = x
        Q.rope_append(d["pool"], kind, rows[:, :512], rows[:, 512:], seq, at, table, cs, err, rope_positions=turn)
        drafts = d["drafts"] if protect else None
        if protect:
            Q.rope_append(d["drafts"].view(B, -1).view(torch.uint8), "bf16", rows[:, :512], rows[:, 512:], seq, node, own, cs,
                          err, rope_positions=turn)
        Q.mla_decode_tree(d["pool"], kind, q, q_pe, table, lens, parents, TAU, d["out"], None, ws, err, prot=d["prot"],
                          draft_rows=drafts)
        Q.tree_verify(target, draft, tokens, parents, u, d["path"], d["kept"], d["next"], err)
        Q.cache_keep(d["pool"], kind, table, lens, d["path"], d["kept"], d["new"], err, prot=d["prot"], draft_rows=drafts)

    first, second = inputs(1), inputs(2)
    wants = []
    for x in (first, second):
        d = fresh()
        step(d, x)
        torch.cuda.synchronize()
        wants.append(d)
    d, x = fresh(), [t.clone() for t in first]
    start = {k: None if v is None else v.clone() for k, v in d.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(d, x)
    for values, want in ((second, wants[1]), (first, wants[0]), (second, wants[1])):
        for to, v in zip(x, values):
            to.copy_(v)
        for k, v in start.items():
            if v is not None:
                d[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for k in d:
            assert d[k] is None or torch.equal(d[k], want[k]), k
    assert Q.read_dev_err(err) == 0


def test_two_streams_at_once():
    """Calls that overlap, each with a workspace of its own."""
    B, T, H, n = 2, 8, 32, 700
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    pool = torch.randn(B * 12, 64 * 576, generator=g, device="cuda").bfloat16().view(torch.uint8)
    table = torch.arange(B * 12, dtype=torch.int32, device="cuda").view(B, 12)
    lens = torch.tensor([n, n + 60], dtype=torch.int32, device="cuda")
    parents = trees("any", B, T).cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    qs = [tuple(x.cuda() for x in queries(B, T, H, s)) for s in range(2)]
    spaces = [torch.empty(Q.tree_workspace_bytes(B, T, H, 768), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.zeros((B, T, H, 512), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def call(i, stream=None):
        Q.mla_decode_tree(pool, "bf16", *qs[i], table, lens, parents, TAU, outs[i], None, spaces[i], err, stream=stream)

    call(0), call(1)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for i, s in enumerate(streams):
                call(i, s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert Q.read_dev_err(err) == 0
