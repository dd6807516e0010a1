"""Host checks of mla_decode_tree, tree_verify, cache_keep and rope_append_at: bad arguments are
refused before anything is launched. No GPU needed."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_36760_gb300 as Q

FAKE = 0x10000  # never dereferenced: validation fails first
INVALID = 1


@pytest.fixture(scope="module")
def L():
    from paper_2609_36760_gb300 import build
    if not os.path.exists(Q.library_path()):
        build.build()
    return Q.lib()


def filled(d, base, kw):
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


def tree_desc(**kw):
    return filled(Q.TreeDesc(), dict(pool=FAKE, cache_kind=4, num_blocks=4, q_latent=FAKE, q_pe=FAKE, batch=2, nodes=8,
                                     heads=16, max_len=0, parents=FAKE, tree_lens=None, block_table=FAKE, max_blocks=3,
                                     softmax_scale=0.1, seq_lens=FAKE, prot=None, draft_rows=None, out=FAKE, lse=None,
                                     workspace=FAKE, workspace_bytes=1 << 40, dev_err=None), kw)


@pytest.mark.parametrize("kw", [
    {"cache_kind": 8}, {"cache_kind": 0}, {"pool": None}, {"pool": FAKE + 16}, {"q_latent": None}, {"q_latent": FAKE + 8},
    {"q_pe": None}, {"q_pe": FAKE + 2}, {"batch": 0}, {"nodes": 0}, {"nodes": 65}, {"heads": 0}, {"heads": 129},
    {"max_len": -1}, {"parents": None}, {"parents": FAKE + 2}, {"tree_lens": FAKE + 1}, {"block_table": None},
    {"max_blocks": 0}, {"max_blocks": 1 << 26}, {"num_blocks": 0}, {"softmax_scale": 0.0},
    {"softmax_scale": float("nan")}, {"softmax_scale": 2e30}, {"seq_lens": None}, {"seq_lens": FAKE + 3}, {"prot": FAKE},
    {"draft_rows": FAKE}, {"prot": FAKE + 8, "draft_rows": FAKE}, {"prot": FAKE, "draft_rows": FAKE + 8},
    {"prot": FAKE, "draft_rows": FAKE, "cache_kind": 16}, {"out": None}, {"out": FAKE + 16}, {"lse": FAKE + 2},
    {"workspace": None}, {"workspace": FAKE + 16}, {"batch": 1 << 30, "max_blocks": 1 << 20},
])
def test_mla_decode_tree_refuses(L, kw):
    assert L.qmla_mla_decode_tree(ctypes.byref(tree_desc(**kw)), None) == INVALID


def verify_desc(**kw):
    return filled(Q.VerifyDesc(), dict(target=FAKE, target_seq_stride=800, target_row_stride=100, draft=FAKE,
                                       draft_seq_stride=800, draft_row_stride=100, probs=0, batch=2, nodes=8, vocab=100,
                                       tokens=FAKE, parents=FAKE, tree_lens=None, uniforms=FAKE, path=FAKE, kept=FAKE,
                                       next_token=FAKE, dev_err=None), kw)


@pytest.mark.parametrize("kw", [
    {"target": None}, {"target": FAKE + 2}, {"target": FAKE + 1, "probs": 1}, {"draft": FAKE + 2}, {"probs": 2},
    {"probs": -1}, {"batch": 0}, {"batch": 65536}, {"nodes": 0}, {"nodes": 65}, {"vocab": 0}, {"vocab": (1 << 24) + 1},
    {"tokens": None}, {"parents": None}, {"uniforms": None}, {"path": None}, {"kept": None}, {"next_token": None},
    {"tokens": FAKE + 2}, {"parents": FAKE + 2}, {"tree_lens": FAKE + 2}, {"uniforms": FAKE + 2}, {"path": FAKE + 2},
    {"kept": FAKE + 2}, {"next_token": FAKE + 2}, {"target_seq_stride": -1}, {"target_row_stride": 1 << 40},
    {"draft_seq_stride": -5}, {"draft_row_stride": -1},
])
def test_tree_verify_refuses(L, kw):
    assert L.qmla_tree_verify(ctypes.byref(verify_desc(**kw)), None) == INVALID


def keep_desc(**kw):
    return filled(Q.KeepDesc(), dict(pool=FAKE, cache_kind=4, num_blocks=4, batch=2, nodes=8, block_table=FAKE,
                                     max_blocks=3, seq_lens=FAKE, tree_lens=None, path=FAKE, kept=FAKE, prot=None,
                                     draft_rows=None, new_lens=FAKE, dev_err=None), kw)


@pytest.mark.parametrize("kw", [
    {"cache_kind": 3}, {"pool": None}, {"pool": FAKE + 16}, {"num_blocks": 0}, {"batch": 0}, {"nodes": 0}, {"nodes": 65},
    {"block_table": None}, {"max_blocks": 0}, {"max_blocks": 1 << 26}, {"seq_lens": None}, {"path": None},
    {"kept": None}, {"new_lens": None}, {"seq_lens": FAKE + 2}, {"tree_lens": FAKE + 2}, {"path": FAKE + 2},
    {"kept": FAKE + 2}, {"new_lens": FAKE + 2}, {"prot": FAKE}, {"draft_rows": FAKE},
    {"prot": FAKE, "draft_rows": FAKE + 8}, {"prot": FAKE, "draft_rows": FAKE, "cache_kind": 16},
])
def test_cache_keep_refuses(L, kw):
    assert L.qmla_cache_keep(ctypes.byref(keep_desc(**kw)), None) == INVALID


def test_no_descriptor(L):
    assert all(f(None, None) == INVALID for f in (L.qmla_mla_decode_tree, L.qmla_tree_verify, L.qmla_cache_keep))
    assert L.qmla_rope_append_at(None, None, None) == INVALID


def test_rope_positions_off_their_boundary(L):
    from test_operator_checks import append_desc
    assert L.qmla_rope_append_at(ctypes.byref(append_desc()), FAKE + 2, None) == INVALID


def test_workspace_bytes_of_bad_arguments(L):
    for args in ((0, 8, 16, 0), (-1, 8, 16, 0), (2, 0, 16, 0), (2, 65, 16, 0), (2, 8, 0, 0), (2, 8, 129, 0), (2, 8, 16, -1)):
        assert L.qmla_tree_workspace_bytes(*args) == 0


@pytest.mark.parametrize("name,cls", [("qmla_tree_desc", Q.TreeDesc), ("qmla_verify_desc", Q.VerifyDesc),
                                      ("qmla_keep_desc", Q.KeepDesc)])
def test_descriptors_match_the_header(name, cls, tmp_path):
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = [f'printf("%zu %zu\\n", offsetof({name}, {f}), sizeof((({name}*)0)->{f}));' for f, _ in cls._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qmla.h"\nint main(void) {\n'
                   + "\n".join(lines) + f'\nprintf("%zu 0\\n", sizeof({name}));return 0; }}\n')
    exe = tmp_path / "s"
    subprocess.run([cc, "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [tuple(map(int, r.split())) for r in subprocess.run([str(exe)], capture_output=True, text=True).stdout.splitlines()]
    want = [(getattr(cls, f).offset, getattr(cls, f).size) for f, _ in cls._fields_] + [(ctypes.sizeof(cls), 0)]
    assert got == want


def test_the_binding_refuses_tensors_that_are_not_the_calls():
    """Types, shapes and devices (there is no CUDA tensor here: every one is refused for its device, but
    only after its type and shape)."""
    B, T, H, V = 2, 4, 8, 30
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    pool = torch.zeros((3, 20736), dtype=torch.uint8)
    ws = torch.zeros(64, dtype=torch.uint8)

    def tree(**kw):
        a = dict(pool=pool, cache_kind=4, q_latent=b(B, T, H, 512), q_pe=b(B, T, H, 64), block_table=i(B, 3), seq_lens=i(B),
                 parents=i(B, T), softmax_scale=0.1, out=b(B, T, H, 512), lse=None, workspace=ws, dev_err=None)
        Q.mla_decode_tree(**{**a, **kw})

    def verify(**kw):
        a = dict(target=torch.zeros(B, T, V), draft=None, tokens=i(B, T), parents=i(B, T), uniforms=torch.zeros(B, T),
                 path=i(B, T), kept=i(B), next_token=i(B), dev_err=None)
        Q.tree_verify(**{**a, **kw})

    def keep(**kw):
        a = dict(pool=pool, cache_kind=4, block_table=i(B, 3), seq_lens=i(B), path=i(B, T), kept=i(B), new_lens=i(B),
                 dev_err=None)
        Q.cache_keep(**{**a, **kw})

    for call in (tree, verify, keep):
        with pytest.raises(ValueError, match="device"):
            call()
    for call, kw, word in ((tree, {"cache_kind": 5}, "cache kind"), (tree, {"pool": pool[:, :-1]}, "pool"),
                           (verify, {"target": torch.zeros(B, T, V).half()}, "float32 or bfloat16"),
                           (verify, {"target": torch.zeros(B, T, V).double()}, "float32 or bfloat16"),
                           (keep, {"cache_kind": "int4"}, "cache kind"), (keep, {"pool": pool.int()}, "pool")):
        with pytest.raises(ValueError, match=word):
            call(**kw)
