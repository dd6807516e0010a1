"""A call that the CUDA runtime refuses is reported by its own status and by no later one."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

# A stream that is being captured cannot be waited for: read_dev_err fails there, and the capture is
# void. (A process of its own: torch's graph is of no more use after that.)
SCRIPT = """
import torch
import paper_2609_36760_gb300 as Q

i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
n, H = 9, 2
q, kv, pe = (torch.randn(*s, device="cuda").bfloat16() for s in ((n, H, 192), (n, H, 256), (n, 64)))
out, ws = torch.zeros(n, H, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(Q.prefill_workspace_bytes(1, n), dtype=torch.uint8, device="cuda")
cu, err, cs, table = i32(0, n), i32(0), torch.rand(n, 64, device="cuda"), i32(0)[None]
pool, rows = torch.zeros(1, Q.block_bytes(4), dtype=torch.uint8, device="cuda"), torch.randn(n, 576, device="cuda").bfloat16()
seq, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, device="cuda").int()
side, other = torch.cuda.Stream(), torch.cuda.Stream()
attend = lambda **kw: Q.mla_prefill(q, kv[..., :128], kv[..., 128:], pe, cu, cu, 0.07, out, None, ws, err, **kw)
append = lambda **kw: Q.rope_append(pool, 4, rows[:, :512], rows[:, 512:], seq, pos, table, cs, err, **kw)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
refused = False
with torch.cuda.stream(side):
    graph.capture_begin()
    try:
        Q.read_dev_err(err, stream=side)
    except Q.QmlaError as e:
        refused = e.status == 4
    append(stream=other)
    try:
        graph.capture_end()
    except RuntimeError:
        pass
assert refused
attend()
torch.cuda.synchronize()
assert Q.read_dev_err(err) == 0 and bool(pool.any()) and bool(out.any())
print("fine")
"""


def test_a_refused_call_does_not_fail_the_next_one():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", SCRIPT], cwd=root, capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.strip().endswith("fine"), run.stderr[-2000:]
