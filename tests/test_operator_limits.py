"""The documented limits of the prompt operators: refused just beyond, accepted at the limit (as far
as a machine without a GPU goes: past every check of the arguments)."""
import ctypes

import pytest
import torch

import paper_2609_36760_gb300 as Q
from test_operator_checks import FAKE, INVALID, L, append_desc, prefill_desc  # noqa: F401 (L: a fixture)


def up(x):
    return float(torch.nextafter(torch.tensor(x, dtype=torch.float32), torch.tensor(torch.inf)))


ONE = float(torch.tensor(1e30, dtype=torch.float32))


@pytest.fixture
def no_gpu():
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")


@pytest.mark.parametrize("at,beyond", [(0.0, -1e-45), (ONE, up(ONE))])
def test_eps(L, no_gpu, at, beyond):  # noqa: F811
    assert L.qmla_rope_append(ctypes.byref(append_desc(norm=1, norm_eps=beyond)), None) == INVALID
    assert L.qmla_rope_append(ctypes.byref(append_desc(norm=1, norm_eps=at)), None) not in (0, INVALID)
    assert L.qmla_rope_append(ctypes.byref(append_desc(norm=0, norm_eps=beyond)), None) not in (0, INVALID)


@pytest.mark.parametrize("n,heads,good", [(1, 1 << 24, True), (1, (1 << 24) + 1, False), (4096, 1 << 24, True),
                                          (4097, 1 << 24, False), (2 ** 31 - 1, 32, True), (2 ** 31 - 1, 33, False)])
def test_rope_query_rows(L, no_gpu, n, heads, good):  # noqa: F811
    args = [FAKE, 0, 0, FAKE, n, heads, FAKE, 64, 0, FAKE, 64 * heads, 64, None, None]
    assert (L.qmla_rope_query(*args) == INVALID) == (not good)


@pytest.mark.parametrize("at,beyond", [(1e-45, 0.0), (ONE, up(ONE))])
def test_softmax_scale(L, no_gpu, at, beyond):  # noqa: F811
    assert L.qmla_mla_prefill(ctypes.byref(prefill_desc(softmax_scale=beyond, workspace_bytes=1 << 30)), None) == INVALID
    assert L.qmla_mla_prefill(ctypes.byref(prefill_desc(softmax_scale=at, workspace_bytes=1 << 30)), None) not in (0, INVALID)


@pytest.mark.parametrize("kw,bad", [({"n_q": 1 << 26}, False), ({"n_kv": 1 << 26}, False), ({"heads": 1024}, False),
                                    ({"batch": 65536}, False), ({"q_token_stride": (1 << 38) - 8}, False),
                                    ({"q_token_stride": 1 << 38}, True),
                                    ({"n_kv": 0, "k": None, "v": None, "k_pe": None, "k_head_stride": 3, "v_head_stride": -1,
                                      "k_token_stride": 5, "k_pe_stride": 0}, False)])
def test_sizes_of_mla_prefill(L, no_gpu, kw, bad):  # noqa: F811
    d = prefill_desc(workspace_bytes=1 << 33, **kw)
    assert (L.qmla_mla_prefill(ctypes.byref(d), None) == INVALID) == bad


def test_workspace_is_what_the_header_says():
    for batch, n_q in [(1, 37), (8, 6400), (65536, 1 << 26)]:
        rest = Q.prefill_workspace_bytes(batch, n_q) - 320 * 133120
        assert 0 < rest < 64 * (n_q // 256 + batch) + 4 * batch + 64 * 320 + 16 * 160 + 2048
