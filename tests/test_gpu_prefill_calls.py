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
