"""Host checks of the prompt operators (rope_append, cache_read, rope_query, mla_prefill):
bad arguments are refused before anything is launched. No GPU needed."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_36760_gb300 as Q

FAKE = 0x10000  # never dereferenced: validation fails first
INVALID, TOO_SMALL = 1, 3


@pytest.fixture(scope="module")
def L():
    from paper_2609_36760_gb300 import build
    if not os.path.exists(Q.library_path()):
        build.build()
    return Q.lib()


def append_desc(**kw):
    d = Q.AppendDesc()
    base = dict(pool=FAKE, cache_kind=4, num_blocks=4, latent=FAKE, latent_stride=512, k_pe=FAKE, k_pe_stride=64, norm=0,
                norm_eps=0.0, norm_weight=None, cos_sin=FAKE, rope_len=64, interleaved=0, seq_ids=None, positions=FAKE,
                n=2, num_seqs=1, block_table=FAKE, max_blocks=1, seq_lens=None, prot=None, dev_err=None)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw", [
    {"cache_kind": 8}, {"pool": None}, {"pool": FAKE + 16}, {"latent": None}, {"k_pe": None}, {"positions": None},
    {"block_table": None}, {"latent": FAKE + 2}, {"latent_stride": 513}, {"latent_stride": 256}, {"k_pe_stride": 63},
    {"k_pe_stride": 32}, {"cos_sin": None}, {"cos_sin": FAKE + 4}, {"rope_len": 0}, {"interleaved": 2},
    {"norm": 1, "norm_eps": -1.0}, {"norm": 1, "norm_eps": float("nan")}, {"norm": 1, "norm_weight": FAKE + 2},
    {"n": -1}, {"num_blocks": 0}, {"num_seqs": 0}, {"max_blocks": 0}, {"prot": FAKE}, {"prot": FAKE + 8, "seq_lens": FAKE},
    {"prot": FAKE, "seq_lens": FAKE, "cache_kind": 16}, {"max_blocks": 1 << 26},
])
def test_rope_append_refuses(L, kw):
    assert L.qmla_rope_append(ctypes.byref(append_desc(**kw)), None) == INVALID


def read_desc(**kw):
    d = Q.ReadDesc()
    base = dict(pool=FAKE, cache_kind=4, num_blocks=4, seq_ids=None, positions=FAKE, n=2, num_seqs=2, block_table=FAKE,
                max_blocks=1, seq_lens=None, prot=None, rows=FAKE, row_stride=576, dev_err=None)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw", [
    {"cache_kind": 3}, {"pool": None}, {"pool": FAKE + 16}, {"positions": None}, {"rows": None}, {"rows": FAKE + 8},
    {"row_stride": 580}, {"row_stride": 568}, {"row_stride": -576}, {"block_table": None}, {"n": -1}, {"num_seqs": 0},
    {"max_blocks": 0}, {"num_blocks": 0}, {"prot": FAKE}, {"prot": FAKE, "seq_lens": FAKE, "cache_kind": 16},
    {"prot": FAKE + 8, "seq_lens": FAKE}, {"seq_ids": FAKE + 1},
])
def test_cache_read_refuses(L, kw):
    assert L.qmla_cache_read(ctypes.byref(read_desc(**kw)), None) == INVALID


@pytest.mark.parametrize("at,value", [
    (0, None), (0, FAKE + 8), (1, 12), (1, -8), (2, 4), (3, None), (4, -1), (5, 0), (6, None), (6, FAKE + 4), (7, 0),
    (8, 2), (9, None), (9, FAKE + 2), (10, 32), (11, 0), (11, 60),
])
def test_rope_query_refuses(L, at, value):
    args = [FAKE, 192 * 16, 192, FAKE, 2, 16, FAKE, 64, 0, FAKE, 64 * 16, 64, None, None]
    args[at] = value
    assert L.qmla_rope_query(*args) == INVALID


def test_rope_query_refuses_rows_that_overlap(L):
    """Of out: token and head strides of which neither steps over the other axis."""
    call = lambda ot, oh, n=3, h=4: L.qmla_rope_query(FAKE, 768, 192, None, n, h, FAKE, 64, 0, FAKE, ot, oh, None, None)  # noqa: E731
    good = lambda ot, oh, n=3, h=4: L.qmla_rope_query(FAKE, 768, 192, FAKE, n, h, FAKE, 64, 0, FAKE, ot, oh, None, None)  # noqa: E731
    assert call(256, 64) == INVALID  # (no positions: the arguments before are fine)
    for ot, oh in [(64, 64), (192, 64), (64, 128), (72, 64), (0, 64), (256, 0)]:
        assert good(ot, oh) == INVALID, (ot, oh)


def test_rope_query_refuses_strides_past_all_addresses(L):
    """Token strides whose product with the tokens leaves 64 bits (and looks small there)."""
    big = (1 << 38) - 8
    assert L.qmla_rope_query(FAKE, 768, 192, FAKE, 1 << 30, 32, FAKE, 64, 0, FAKE, 1 << 37, big, None, None) == INVALID


@pytest.mark.parametrize("fn,desc", [("qmla_rope_append", append_desc(n=1, latent_stride=3, k_pe_stride=-5)),
                                     ("qmla_cache_read", read_desc(n=1, row_stride=-3))])
def test_a_single_row_has_no_stride(L, fn, desc):
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    assert getattr(L, fn)(ctypes.byref(desc), None) not in (0, INVALID)  # (no device: the checks before are through)
    assert L.qmla_rope_query(FAKE, 3, -5, FAKE, 1, 1, FAKE, 64, 0, FAKE, 1, 7, None, None) not in (0, INVALID)


def prefill_desc(**kw):
    d = Q.PrefillDesc()
    base = dict(q=FAKE, q_token_stride=192 * 16, q_head_stride=192, k=FAKE, k_token_stride=256 * 16, k_head_stride=256,
                v=FAKE, v_token_stride=256 * 16, v_head_stride=256, k_pe=FAKE, k_pe_stride=576, n_q=5, n_kv=7, heads=16,
                batch=2, cu_q=FAKE, cu_kv=FAKE, causal=1, softmax_scale=0.1, out=FAKE, lse=None, workspace=FAKE,
                workspace_bytes=1 << 20, dev_err=None)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw", [
    {"q": None}, {"q": FAKE + 8}, {"q_token_stride": 4}, {"q_head_stride": 0}, {"k": None}, {"k": FAKE + 2},
    {"k_token_stride": -8}, {"k_head_stride": 0}, {"v": None}, {"v": FAKE + 4}, {"v_token_stride": 1 << 38},
    {"v_head_stride": 129}, {"k_pe": None}, {"k_pe": FAKE + 8}, {"k_pe_stride": 0}, {"n_q": -1}, {"n_kv": -1},
    {"n_q": (1 << 26) + 1}, {"n_kv": (1 << 26) + 1}, {"heads": 0}, {"heads": 1025}, {"batch": 0}, {"batch": 65537},
    {"cu_q": None}, {"cu_kv": None}, {"cu_q": FAKE + 2}, {"causal": 2}, {"softmax_scale": 0.0},
    {"softmax_scale": float("nan")}, {"softmax_scale": float("inf")}, {"out": None}, {"out": FAKE + 8}, {"out": FAKE + 16},
    {"lse": FAKE + 2}, {"workspace": None}, {"workspace": FAKE + 128},
])
def test_mla_prefill_refuses(L, kw):
    assert L.qmla_mla_prefill(ctypes.byref(prefill_desc(**kw)), None) == INVALID


def test_workspace_and_empty_calls(L):
    need = Q.prefill_workspace_bytes(2, 5)
    assert need > 0 and Q.prefill_workspace_bytes(2, 1 << 26) > Q.prefill_workspace_bytes(2, 1 << 20)
    for bad in [(0, 5), (65537, 5), (1, -1), (1, (1 << 26) + 1)]:
        assert Q.prefill_workspace_bytes(*bad) == 0
    assert L.qmla_mla_prefill(ctypes.byref(prefill_desc(workspace_bytes=need - 1)), None) == TOO_SMALL
    # null descriptors, and calls without rows, which touch nothing
    for f in (L.qmla_rope_append, L.qmla_cache_read, L.qmla_mla_prefill):
        assert f(None, None) == INVALID
    assert L.qmla_rope_append(ctypes.byref(append_desc(n=0, pool=None, latent=None, k_pe=None, cos_sin=None)), None) == 0
    assert L.qmla_cache_read(ctypes.byref(read_desc(n=0, pool=None, rows=None)), None) == 0
    assert L.qmla_rope_query(None, 0, 0, None, 0, 16, None, 64, 0, None, 0, 0, None, None) == 0
    assert L.qmla_mla_prefill(ctypes.byref(prefill_desc(n_q=0, q=None, out=None, workspace=None)), None) == 0


def test_binding_refuses_wrong_tensors():
    """The binding looks at types, shapes and devices before it passes addresses on."""
    bf, i32 = torch.bfloat16, torch.int32
    pool, table, err = torch.zeros(2, 20736, dtype=torch.uint8), torch.zeros(1, 2, dtype=i32), torch.zeros(1, dtype=i32)
    lat, kpe, pos, cs = torch.zeros(3, 512, dtype=bf), torch.zeros(3, 64, dtype=bf), torch.zeros(3, dtype=i32), torch.zeros(9, 64)
    with pytest.raises(ValueError, match="CUDA"):
        Q.rope_append(pool, 4, lat, kpe, None, pos, table, cs, err)
    with pytest.raises(ValueError, match="bfloat16"):
        Q.rope_append(pool, 4, lat.float(), kpe, None, pos, table, cs, err)
    with pytest.raises(ValueError, match="shape"):
        Q.rope_append(pool, 4, lat[:, :500], kpe, None, pos, table, cs, err)
    with pytest.raises(ValueError, match="last axis"):
        Q.rope_append(pool, 4, torch.zeros(512, 3, dtype=bf).T, kpe, None, pos, table, cs, err)
    with pytest.raises(ValueError):
        Q.cache_read(pool, 4, None, pos, table, torch.zeros(3, 512, dtype=bf), err)
    with pytest.raises(ValueError):
        Q.rope_query(torch.zeros(3, 2, 64), pos, cs, torch.zeros(3, 2, 64, dtype=bf), err)
    q, kv = torch.zeros(3, 2, 192, dtype=bf), torch.zeros(3, 2, 256, dtype=bf)
    with pytest.raises(ValueError):
        Q.mla_prefill(q, kv[..., :128], kv[..., 128:], kpe, pos[:2], pos[:2], 0.1, torch.zeros(3, 2, 128, dtype=bf), None,
                      torch.zeros(1 << 16, dtype=torch.uint8), err)


@pytest.mark.parametrize("name,cls", [("qmla_append_desc", Q.AppendDesc), ("qmla_read_desc", Q.ReadDesc),
                                      ("qmla_prefill_desc", Q.PrefillDesc)])
def test_descriptors_match_the_header(tmp_path, name, cls):
    """Sizes and offsets of the binding's structures are those of include/qmla.h in C."""
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    fields = [f for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "qmla.h"\nint main(void) {\n'
                   f'printf("%zu\\n", sizeof({name}));\n'
                   + "".join(f'printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields) + "return 0; }\n")
    exe = tmp_path / "layout"
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([cc, "-I", inc, str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]
