"""mla_prefill against the formula in 64 bits, and the prompt operators together.

Tolerances, per element, from the roundings alone. A weight w_j reaches the tensor
core as bf16 (relative 2^-8), the result is rounded to bf16 (2^-8), and a score is
off by at most e = 192 * 2^-24 * max_j tau sum_c |q_c k_c| (fp32 sums of 192 products),
which moves a weight and the sum of weights by a factor exp(e) each:
    |out - exact| <= (2^-8 + 2 e + 2^-18) sum_j w_j |v_j| + 2^-8 |exact|
    |lse - exact| <= e + 2^-18 + 2^-21 |exact|
2^-18 stands for the exponential (ex2.approx, 2^-22) and the fp32 sums (at most a few
hundred additions in a chain, 2^-24 each)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_36760_gb300 as Q

pytestmark = pytest.mark.gpu
TAU = 1.0 / math.sqrt(192.0)


def cu(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


class Prompt:
    def __init__(self, lq, lk, heads, seed=0, pad_q=0, pad_kv=0, scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lq, self.lk, self.H = lq, lk, heads
        nq, nkv = sum(lq) + pad_q, sum(lk) + pad_kv
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.q = (scale * rnd(nq, heads, 192)).bfloat16()
        self.kv = rnd(nkv, heads, 256).bfloat16()
        self.rows = rnd(nkv, 576).bfloat16()
        self.out = torch.full((nq, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((nq, heads), 7.0, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(Q.prefill_workspace_bytes(len(lq), nq), dtype=torch.uint8, device="cuda")

    def run(self, causal=True, cu_q=None, cu_kv=None, **kw):
        a = dict(q=self.q, k=self.kv[..., :128], v=self.kv[..., 128:], k_pe=self.rows[:, 512:])
        a.update(kw)
        Q.mla_prefill(a["q"], a["k"], a["v"], a["k_pe"], cu(self.lq) if cu_q is None else cu_q,
                      cu(self.lk) if cu_kv is None else cu_kv, TAU, self.out, self.lse, self.ws, self.err, causal=causal)
        return Q.read_dev_err(self.err)

    def check(self, causal=True, sequences=None):
        aq = ak = 0
        for b, (n, m) in enumerate(zip(self.lq, self.lk)):
            if n and (sequences is None or b in sequences):
                q = self.q[aq:aq + n].double().transpose(0, 1)
                k = torch.cat([self.kv[ak:ak + m, :, :128].double(),
                               self.rows[ak:ak + m, None, 512:].double().expand(m, self.H, 64)], -1).transpose(0, 1)
                v = self.kv[ak:ak + m, :, 128:].double().transpose(0, 1)
                got, lse = self.out[aq:aq + n].double().transpose(0, 1), self.lse[aq:aq + n].double().T
                if m == 0:
                    assert bool((got == 0).all()) and bool((lse == -math.inf).all())
                    aq += n
                    continue
                s = TAU * q @ k.transpose(1, 2)
                hide = torch.zeros(n, m, dtype=torch.bool, device="cuda")
                if causal:
                    hide = torch.arange(m, device="cuda")[None] > torch.arange(n, device="cuda")[:, None] + m - n
                s = s.masked_fill(hide, -math.inf)
                empty = hide.all(1)
                e = 192 * 2.0 ** -24 * float(TAU * (q.abs().amax(1) @ k.abs().amax(1).T).max()) if n * m > 1 << 22 else \
                    192 * 2.0 ** -24 * float((TAU * q.abs() @ k.abs().transpose(1, 2)).max())
                z = torch.logsumexp(s, 2)
                w = torch.exp(s - torch.where(z.isinf(), 0.0, z)[..., None])
                want, size = w @ v, w @ v.abs()
                off = (got - want).abs() - ((2.0 ** -8 + 2 * e + 2.0 ** -18) * size + 2.0 ** -8 * want.abs())
                assert bool((off[:, ~empty] <= 0).all()), (b, float(off.max()))
                assert bool((got[:, empty] == 0).all()) and bool((lse[:, empty] == -math.inf).all())
                gap = (lse - z).abs()[:, ~empty] - (e + 2.0 ** -18 + 2.0 ** -21 * z.abs()[:, ~empty])
                assert bool((gap <= 0).all()), (b, float(gap.max()))
            aq, ak = aq + n, ak + m
        assert bool((self.out[sum(self.lq):] == 7).all()) and bool((self.lse[sum(self.lq):] == 7).all())


@pytest.mark.parametrize("n", [1, 2, 31, 64, 127, 128, 129, 255, 256, 257, 385, 512, 1000])
def test_one_prompt(n):
    p = Prompt([n], [n], 3, seed=n)
    assert p.run() == 0
    p.check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m", [(1, 1), (1, 128), (1, 129), (1, 5000), (7, 700), (130, 131), (256, 1024), (300, 2049),
                                 (128, 127), (300, 40), (513, 256), (700, 1), (5, 0), (260, 0)])
def test_queries_behind_a_context(n, m, causal):
    """Fewer keys than queries leave the first rows without any (causal)."""
    p = Prompt([n], [m], 2, seed=n + m)
    assert p.run(causal) == 0
    p.check(causal)


@pytest.mark.parametrize("heads", [1, 16, 100, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_batches(heads, causal):
    lq, lk = [5, 0, 300, 128, 1, 77, 257], [5, 9, 300, 500, 0, 78, 1000]
    p = Prompt(lq, lk, heads, seed=heads, pad_q=40, pad_kv=3)
    assert p.run(causal) == 0
    p.check(causal)


def test_many_items_per_cta_and_head_groups():
    """More (item, head) pairs than CTAs, and keys of more than one head group (48 MB)."""
    p = Prompt([1300, 900, 2500], [1300, 2000, 2500], 24, seed=1)
    assert p.run() == 0
    p.check()
    p = Prompt([600], [30000], 7, seed=2)
    assert p.run() == 0
    p.check()


@pytest.mark.parametrize("n,m,heads", [(1, 40000, 1), (40, 5000, 1), (200, 20000, 1), (300, 9000, 3), (700, 3000, 2)])
@pytest.mark.parametrize("causal", [True, False])
def test_few_rows_over_long_contexts(n, m, heads, causal):
    """Keys in parts: up to 59 of them, of one and two tiles, joined from the workspace."""
    p = Prompt([n], [m], heads, seed=n + m)
    assert p.run(causal) == 0
    p.check(causal)


def test_one_long_sequence_among_short_ones():
    """Only the long one's keys go in parts; rows without keys in some of them (causal)."""
    p = Prompt([3, 600, 1, 0, 90], [3, 12000, 0, 7, 40], 4, seed=12)
    assert p.run() == 0
    p.check()


def test_large_scores_raise_the_reference():
    """Scores whose maximum grows along the keys by far more than 2^8 a step: the running
    maximum is raised and the sums rescaled many times."""
    p = Prompt([200], [2000], 2, seed=3, scale=4.0)
    ramp = torch.linspace(0.05, 6.0, 2000, device="cuda")[:, None, None]
    p.kv[..., :128] = (p.kv[..., :128].float() * ramp).bfloat16()
    assert p.run(False) == 0
    p.check(False)


def test_equal_scores_give_the_mean():
    p = Prompt([4], [1000], 2, seed=4)
    p.q.zero_()
    assert p.run(False) == 0
    p.check(False)
    assert bool((p.lse == torch.tensor(math.log(1000.0), device="cuda")).all() | ((p.lse - math.log(1000.0)).abs() < 1e-5).all())


@pytest.mark.parametrize("causal", [True, False])
def test_other_sequences_values_never_reach_a_result(causal):
    """Infinities and NaN in the rows of other sequences and in padding rows."""
    lq, lk = [130, 70, 60], [130, 200, 60]
    p = Prompt(lq, lk, 3, seed=5, pad_q=9, pad_kv=70)
    clean = Prompt(lq, lk, 3, seed=5, pad_q=9, pad_kv=70)
    assert clean.run(causal) == 0
    for t, a, n in ((p.kv, 130, 200), (p.rows, 130, 200), (p.q, 130, 70)):
        t[a:a + n:2] = math.nan
        t[a + 1:a + n:2] = math.inf
    p.kv[390:], p.rows[390:], p.q[260:] = math.nan, math.inf, math.nan
    assert p.run(causal) == 0
    p.check(causal, sequences={0, 2})
    assert torch.equal(p.out[:130], clean.out[:130]) and torch.equal(p.out[200:260], clean.out[200:260])
    assert torch.equal(p.lse[:130], clean.lse[:130]) and bool(p.out[130:200].isnan().any())


def test_strides_and_orders():
    p = Prompt([150, 20], [150, 90], 4, seed=6)
    assert p.run() == 0
    want, lse = p.out.clone(), p.lse.clone()
    # heads outermost; keys and values apart; a wide RoPE row
    q = p.q.transpose(0, 1).contiguous().transpose(0, 1)
    k = p.kv[..., :128].transpose(0, 1).contiguous().transpose(0, 1)
    v = p.kv[..., 128:].contiguous()
    pe = torch.zeros(p.rows.size(0), 72, dtype=torch.bfloat16, device="cuda")
    pe[:, :64] = p.rows[:, 512:]
    p.out.zero_()
    assert p.run(q=q, k=k, v=v, k_pe=pe[:, :64]) == 0
    assert torch.equal(p.out, want) and torch.equal(p.lse, lse)
    one = Prompt([9], [9], 1, seed=7)  # one head: its stride is never used
    assert one.run() == 0
    one.check()


def test_without_lse_and_repeatable():
    p = Prompt([500, 33], [500, 33], 16, seed=8)
    assert p.run() == 0
    first = p.out.clone()
    for _ in range(3):
        p.out.fill_(7)
        Q.mla_prefill(p.q, p.kv[..., :128], p.kv[..., 128:], p.rows[:, 512:], cu(p.lq), cu(p.lk), TAU, p.out, None, p.ws,
                      p.err)
        assert torch.equal(p.out, first)


def test_more_sequences_than_fit_on_chip():
    """2,600 tiny sequences, some empty: the plan's prefix goes through the workspace."""
    g = torch.Generator().manual_seed(5)
    lq = torch.randint(0, 4, (2600,), generator=g).tolist()
    lk = [n + m for n, m in zip(lq, torch.randint(0, 5, (2600,), generator=g).tolist())]
    p = Prompt(lq, lk, 2, seed=13)
    assert p.run() == 0
    p.check(sequences=set(range(0, 2600, 37)) | {2599})


def test_offsets_past_32_bits():
    """Keys and values of over 4 GB, and queries and results that lie behind 4 GB."""
    n, m, heads = 5, 140_000, 64
    g = torch.Generator(device="cuda").manual_seed(6)
    kv = torch.randn(m, heads, 256, generator=g, device="cuda", dtype=torch.bfloat16)
    pe = torch.randn(m, 64, generator=g, device="cuda", dtype=torch.bfloat16)
    rows = 180_000  # x 64 heads x 192 channels: 4.4 GB
    q = torch.empty(rows, heads, 192, dtype=torch.bfloat16, device="cuda")
    q[-n:] = torch.randn(n, heads, 192, generator=g, device="cuda")
    out = torch.zeros(rows * 2, heads, 128, dtype=torch.bfloat16, device="cuda")[-rows:]
    lse, err = torch.zeros(rows, heads, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(Q.prefill_workspace_bytes(1, rows), dtype=torch.uint8, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    Q.mla_prefill(q, kv[..., :128], kv[..., 128:], pe, i32(rows - n, rows), i32(0, m), TAU, out, lse, ws, err)
    assert Q.read_dev_err(err) == 0
    for h in (0, 31, 63):
        k = torch.cat([kv[:, h, :128], pe], 1).double()
        s = TAU * q[-n:, h].double() @ k.T
        e = 192 * 2.0 ** -24 * float((TAU * q[-n:, h].double().abs() @ k.abs().T).max())
        s = s.masked_fill(torch.arange(m, device="cuda")[None] > torch.arange(n, device="cuda")[:, None] + m - n, -math.inf)
        w, v = torch.softmax(s, 1), kv[:, h, 128:].double()
        want = w @ v
        gap = (out[-n:, h].double() - want).abs()
        assert bool((gap <= (2.0 ** -8 + 2 * e + 2.0 ** -18) * (w @ v.abs()) + 2.0 ** -8 * want.abs()).all())
    assert not bool(out[:-n].any())


def test_bad_offsets_are_left_out():
    """Decreasing, negative and too large offsets: reported, their rows left as they were."""
    p = Prompt([50, 60, 70, 80], [50, 60, 70, 80], 2, seed=9)
    good = cu(p.lq)
    for cq, ck in [([0, 50, 40, 180, 260], [0, 50, 110, 180, 260]), ([0, 50, 110, 180, 261], [0, 50, 110, 180, 260]),
                   ([-1, 50, 110, 180, 260], [0, 50, 110, 180, 260]), ([0, 50, 110, 180, 260], [0, 50, 300, 180, 260])]:
        p.err.zero_()
        p.out.fill_(7)
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        assert p.run(cu_q=dev(cq), cu_kv=dev(ck)) == Q.DEVERR_BAD_OFFSETS
    p.err.zero_()
    over = torch.tensor([0, 260, 0, 260, 0, 260, 0, 260, 0], dtype=torch.int32, device="cuda")  # overlapping prompts
    p.ws = torch.empty(Q.prefill_workspace_bytes(8, 260), dtype=torch.uint8, device="cuda")
    assert p.run(cu_q=over, cu_kv=over) == Q.DEVERR_BAD_OFFSETS
    p.err.zero_()
    p.out.fill_(7), p.lse.fill_(7)
    assert p.run(cu_q=good, cu_kv=good) == 0
    p.check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([37], [37]), ([200, 1, 0, 129, 90], [200, 300, 40, 129, 0]), ([300, 256], [500, 256])])
def test_calls_with_and_without_a_plan_agree(lq, lk, causal):
    """The rows behind the last sequence make the second call a long one: the same items, from the plan's list."""
    a, b = Prompt(lq, lk, 5, seed=12, pad_q=3), Prompt(lq, lk, 5, seed=12, pad_q=3, pad_kv=9000)
    b.q.copy_(a.q), b.kv[:sum(lk)].copy_(a.kv), b.rows[:sum(lk)].copy_(a.rows)
    b.kv[sum(lk):], b.rows[sum(lk):] = math.nan, math.inf
    assert a.run(causal) == 0 and b.run(causal) == 0
    a.check(causal)
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


@pytest.mark.parametrize("pad_kv", [0, 9000])
def test_the_sequences_beside_a_bad_one(pad_kv):
    """A sequence whose offsets are bad is left out, in short calls and planned ones; the others are computed."""
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    p = Prompt([50, 60, 70, 80], [50, 60, 70, 80], 2, seed=9, pad_kv=pad_kv)
    for cq, ck, left in [(dev(0, 50, 110, 180, 261), cu(p.lk), {0, 1, 2}), (dev(-1, 50, 110, 180, 260), cu(p.lk), {1, 2, 3}),
                         (cu(p.lq), dev(0, 50, 110, 180, 261 + pad_kv), {0, 1, 2}),
                         (cu(p.lq), dev(0, 50, 110, -5, 0), {0, 1})]:
        p.err.zero_()
        p.out.fill_(7), p.lse.fill_(7)
        assert p.run(cu_q=cq, cu_kv=ck) == Q.DEVERR_BAD_OFFSETS
        p.check(sequences=left)
        for b in {0, 1, 2, 3} - left:
            assert bool((p.out[sum(p.lq[:b]):sum(p.lq[:b + 1])] == 7).all())


def test_a_planned_call_in_a_graph_on_two_workspaces():
    a, b = (Prompt([40, 200, 700], [9000, 200, 700], 8, seed=s) for s in (13, 14))
    cq, ck = cu(a.lq), cu(a.lk)
    graph, streams = torch.cuda.CUDAGraph(), [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        for s, p in zip(streams, (a, b)):
            s.wait_stream(main)
            Q.mla_prefill(p.q, p.kv[..., :128], p.kv[..., 128:], p.rows[:, 512:], cq, ck, TAU, p.out, p.lse, p.ws, p.err, stream=s)
            main.wait_stream(s)
    for _ in range(3):
        a.out.fill_(7), b.out.fill_(7)
        graph.replay()
    torch.cuda.synchronize()
    a.check()
    b.check()
    assert Q.read_dev_err(a.err) == 0 and Q.read_dev_err(b.err) == 0


def test_two_streams_and_a_replayed_graph():
    a, b = Prompt([300], [300], 8, seed=10), Prompt([40, 200], [900, 200], 8, seed=11)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    cqa, cqb, cka, ckb = cu(a.lq), cu(b.lq), cu(a.lk), cu(b.lk)
    torch.cuda.synchronize()
    for _ in range(4):
        for s, p, cq, ck in ((sa, a, cqa, cka), (sb, b, cqb, ckb)):
            Q.mla_prefill(p.q, p.kv[..., :128], p.kv[..., 128:], p.rows[:, 512:], cq, ck, TAU, p.out, p.lse, p.ws, p.err, stream=s)
    torch.cuda.synchronize()
    a.check()
    b.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Q.mla_prefill(b.q, b.kv[..., :128], b.kv[..., 128:], b.rows[:, 512:], cqb, ckb, TAU, b.out, b.lse, b.ws, b.err)
    b.q.mul_(0.5)
    b.out.fill_(7)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    b.check()
    assert Q.read_dev_err(a.err) == 0 and Q.read_dev_err(b.err) == 0
