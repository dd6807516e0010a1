"""Calls of mla_prefill that its documentation allows and that a tensor of torch does not
make by itself, through the descriptor."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

import paper_2609_36760_gb300 as Q

pytestmark = pytest.mark.gpu
TAU = 1.0 / math.sqrt(192.0)


@pytest.mark.parametrize("heads", [1, 5])
@pytest.mark.parametrize("batch", [1, 70])
@pytest.mark.parametrize("k_head,v_head,others", [(0, 0, 0), (3, 129, 5), (-8, 1 << 40, -1)])
def test_without_keys_their_addresses_and_strides_are_not_used(heads, batch, k_head, v_head, others):
    """n_kv = 0: null k, v and k_pe, whatever stands in their strides (70 sequences: with a plan)."""
    n = 3 * batch
    q = torch.randn(n, heads, 192, device="cuda").bfloat16()
    out = torch.full((n, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, heads), 7.0, device="cuda")
    cu_q = torch.arange(0, n + 1, 3, dtype=torch.int32, device="cuda")
    cu_kv = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    ws = torch.empty(Q.prefill_workspace_bytes(batch, n), dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = Q.PrefillDesc(q=q.data_ptr(), q_token_stride=heads * 192, q_head_stride=192, k_token_stride=others,
                      k_head_stride=k_head, v_token_stride=others, v_head_stride=v_head, k_pe_stride=others, n_q=n,
                      n_kv=0, heads=heads, batch=batch, cu_q=cu_q.data_ptr(), cu_kv=cu_kv.data_ptr(), causal=1,
                      softmax_scale=TAU, out=out.data_ptr(), lse=lse.data_ptr(), workspace=ws.data_ptr(),
                      workspace_bytes=ws.numel(), dev_err=err.data_ptr())
    assert Q.lib().qmla_mla_prefill(ctypes.byref(d), torch.cuda.current_stream().cuda_stream) == 0
    assert Q.read_dev_err(err) == 0
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_the_prompt_operators_without_an_error_word():
    """dev_err may be None, as for the calls around them; a workspace is bytes of any type and shape."""
    n, heads = 70, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    proj, q, kv = rnd(n, 576), rnd(n, heads, 192), rnd(n, heads, 256)
    seq, pos, table = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, device="cuda").int(), i32(1, 0)[None]
    cs = torch.rand(n, 64, device="cuda")
    need = Q.prefill_workspace_bytes(1, n)
    got = []
    for err in (torch.zeros(1, dtype=torch.int32, device="cuda"), None):
        pool = torch.zeros(2, Q.block_bytes(4), dtype=torch.uint8, device="cuda")
        rows, turned = torch.zeros(n, 576, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(q[..., 128:].contiguous())
        out, lse = torch.zeros(n, heads, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, heads, device="cuda")
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if err is not None else \
            torch.empty(8, need // 32 + 1, dtype=torch.float32, device="cuda")
        Q.rope_append(pool, 4, proj[:, :512], proj[:, 512:], seq, pos, table, cs, err, norm=True)
        Q.cache_read(pool, 4, seq, pos, table, rows, err)
        Q.rope_query(q[..., 128:], pos, cs, turned, err)
        Q.mla_prefill(q, kv[..., :128], kv[..., 128:], rows[:, 512:], i32(0, n), i32(0, n), TAU, out, lse, ws, err)
        got.append((pool, rows, turned, out, lse))
        assert err is None or Q.read_dev_err(err) == 0
    # and what an error word would report is left out all the same
    rows = torch.full((2, 576), 7.0, dtype=torch.bfloat16, device="cuda")
    Q.cache_read(got[0][0], 4, i32(0, 9), i32(5, 5), table, rows, None)
    Q.mla_prefill(q, kv[..., :128], kv[..., 128:], got[0][1][:, 512:], i32(0, n + 1), i32(0, n), TAU, got[0][3].clone(), None,
                  torch.empty(need, dtype=torch.uint8, device="cuda"), None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert bool((rows[1] == 7).all()) and torch.equal(rows[0], got[0][1][5])
