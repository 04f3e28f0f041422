"""Refusals of the speculative decode step's calls (made before any device call), the binding's checks, and the
oracle's own pins."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import decode_oracle as R
from paper_2609_05228_gb300 import ace, build

OK, INVALID, UNSUPPORTED = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ace.LIBPATH):
        build.build()
    ace._lib = None
    return ace.lib()


def _create(L, k=16, v=16, ks=16, vs=16, desc=(1, 4, 16, 2, 64, 0, 1)):
    out = ctypes.c_void_p(7)
    d = ace.ace_kv_desc(*desc)
    st = L.ace_kv_create(ctypes.byref(d), k, v, ks, vs, None, ctypes.byref(out))
    assert out.value is None
    return st


@pytest.mark.parametrize("desc,want,text", [
    ((0, 4, 16, 2, 64, 0, 1), INVALID, b"positive"), ((1, 0, 16, 2, 64, 0, 1), INVALID, b"positive"),
    ((1, 4, -16, 2, 64, 0, 1), INVALID, b"positive"), ((1, 4, 16, 0, 64, 0, 1), INVALID, b"positive"),
    ((1, 4, 16, 2, 0, 0, 1), INVALID, b"positive"), ((1, 4, 16, 2, 64, 2, 1), INVALID, b"dtype"),
    ((1, 4, 16, 2, 64, 0, 2), INVALID, b"format"), ((1, 4, 8, 2, 64, 0, 1), UNSUPPORTED, b"page_size"),
    ((1, 4, 48, 2, 64, 0, 1), UNSUPPORTED, b"page_size"), ((1, 4, 512, 2, 64, 0, 1), UNSUPPORTED, b"page_size"),
    ((1, 4, 16, 2, 68, 0, 1), UNSUPPORTED, b"head_dim"), ((1, 4, 16, 2, 264, 0, 1), UNSUPPORTED, b"head_dim"),
    ((1, 1 << 30, 16, 2, 64, 0, 1), UNSUPPORTED, b"2^31"), ((1 << 20, 1 << 20, 16, 1 << 20, 64, 0, 1), UNSUPPORTED, b"2^31")])
def test_create_refuses(L, desc, want, text):
    assert _create(L, desc=desc) == want and text in L.ace_last_error_message()


def test_create_refuses_pointers(L):
    for bad in ({"k": None}, {"v": None}, {"k": 24}, {"v": 17}, {"ks": None}, {"vs": None}):
        assert _create(L, **bad) == INVALID
    assert L.ace_kv_create(None, 16, 16, 16, 16, None, None) == INVALID
    L.ace_kv_destroy(None)


def test_calls_refuse_a_missing_cache(L):
    assert L.ace_kv_sync(None) == INVALID
    assert L.ace_kv_write(None, 0, 16, 1, 1, 16, 1, 1, 16, 1, None) == INVALID
    assert L.ace_kv_read(None, 0, 16, 1, 16, 16, None) == INVALID
    assert L.ace_kv_keep(None, 16, 1, 16, 16, 1, 16, 1, None, None) == INVALID
    assert L.ace_tree_attention(None, 0, 16, 1, 1, 1, 16, 1, 16, 16, None, 1, 1, 1, 1.0, 16, None, None) == INVALID


def test_tree_mask_refuses(L):
    assert L.ace_tree_mask(16, 16, -1, 4, 16, None, None) == INVALID
    for n in (0, -1, 257):
        assert L.ace_tree_mask(16, 16, 1, n, 16, None, None) == INVALID and b"max_nodes" in L.ace_last_error_message()
    for args in ((None, 16, 16), (16, None, 16), (16, 16, None)):
        assert L.ace_tree_mask(args[0], args[1], 1, 4, args[2], None, None) == INVALID
    assert L.ace_tree_mask(None, None, 0, 4, None, None, None) == OK


def _verify(L, **kw):
    a = dict(logits=16, dtype=0, ls=8, V=8, tokens=16, parents=16, off=16, B=1, T=4, n=4, draft=16, ds=8, temp=None, u=16,
             noise=16, ns=8, path=16, keep=16, nxt=16)
    a.update(kw)
    return L.ace_verify_tree(*a.values(), None)


def test_verify_refuses(L):
    for kw in ({"dtype": 2}, {"V": 0}, {"B": -1}, {"T": -1}, {"n": 0}, {"n": 257}, {"ls": 7}, {"ds": 7}, {"ns": 7}, {"logits": None},
               {"logits": 17}, {"tokens": None}, {"parents": None}, {"off": None}, {"u": None}, {"noise": None}, {"path": None},
               {"keep": None}, {"nxt": None}):
        assert _verify(L, **kw) == INVALID, kw
    assert _verify(L, B=0) == OK


def test_desc_layout_matches_header(tmp_path):
    import subprocess
    src = tmp_path / "l.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ace.h"\nint main(void) { printf("%zu %zu %zu", sizeof(ace_kv_desc),'
                   " offsetof(ace_kv_desc, head_dim), offsetof(ace_kv_desc, format)); return 0; }\n")
    subprocess.run(["gcc", "-I", build.INCLUDE, str(src), "-o", str(tmp_path / "l")], check=True)
    got = subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in got] == [ctypes.sizeof(ace.ace_kv_desc), ace.ace_kv_desc.head_dim.offset, ace.ace_kv_desc.format.offset]


def test_binding_checks_tensors():
    f, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="logits must be"):
        ace.ace_verify_tree(f.double(), i, i, i[:2], 4, f[:, 0], f[:1], i.view(1, 4), i[:1], i[:1])
    with pytest.raises(ValueError, match="on a GPU"):
        ace._want("x", f, "float32")
    with pytest.raises(ValueError, match="shape"):
        ace._want("x", f, "float32", (4, 9))
    with pytest.raises(ValueError, match="contiguous"):
        ace._want("x", f.T, "float32")
    with pytest.raises(ValueError, match="must be int32"):
        ace._want("x", f, "int32")
    with pytest.raises(ValueError, match="dtype must be"):
        ace.AceKvCache(1, 64, 16, 1, dtype="f16")


# ----------------------------------------------------------------------- the oracle's pins


def test_oracle_e4m3_agrees_with_torch():
    v = R.e4m3_values()
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, want, equal_nan=True)
    x = np.random.default_rng(0).standard_normal((200, 64)) * np.exp(np.random.default_rng(1).uniform(-20, 20, (200, 1)))
    x = x.astype(np.float32)
    code, byte, value = R.quantise_rows(x)
    amax = np.abs(x).max(1).astype(float)
    e = byte.astype(int) - 127
    assert (amax <= 448 * np.ldexp(1.0, e)).all() and (amax > 448 * np.ldexp(1.0, e - 1)).all()
    want = torch.from_numpy(np.ldexp(x, -e[:, None]).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (code == want).all()
    assert (np.abs(value - x) <= np.maximum(np.abs(x) / 16, np.ldexp(1.0, e - 10)[:, None])).all()


def test_oracle_attention_worked():
    """Two keys of equal score, then one masked: means of the values that are seen."""
    q, k = np.zeros((2, 1, 2)), np.ones((3, 1, 2))
    v = np.array([[1.0, 0.0], [3.0, 4.0], [np.nan, np.nan]])[:, None]
    out, lse = R.tree_attention(q, k, v, 1, np.array([[True, False], [False, False]]), 1.0)
    assert out[0, 0].tolist() == [2.0, 2.0] and out[1, 0].tolist() == [1.0, 0.0]
    assert np.allclose(lse[:, 0], [np.log(2.0), 0.0], rtol=0, atol=1e-15)
    out, lse = R.tree_attention(q, k[1:], v[1:], 0, np.array([[False, False], [True, False]]), 1.0)
    assert (out[0] == 0).all() and np.isneginf(lse[0, 0]) and out[1, 0].tolist() == [3.0, 4.0]


def test_oracle_verify_worked():
    """r = (1/2, 1/4, 1/4), q = (1/4, 1/2, 1/4), child 1: accepted with u <= 1/2; after its rejection r = (1, 0, 0)."""
    z, q = np.log(np.array([[0.5, 0.25, 0.25]] * 2)), np.array([[0.25, 0.5, 0.25]] * 2)
    noise = np.array([10.0, 0.1, 0.1])
    assert R.verify(z, [0, 1], [-1, 0], q, 1.0, [0, 0.49], noise) == ([0, 1], 1)
    assert R.verify(z, [0, 1], [-1, 0], q, 1.0, [0, 0.51], noise) == ([0], 0)
    # without draft probabilities the rejected token loses its share: (2/3, 0, 1/3)
    assert R.verify(z, [0, 1], [-1, 0], None, 1.0, [0, 0.26], noise) == ([0], 2)
    assert R.verify(z, [0, 1], [-1, 0], None, 1.0, [0, 0.24], noise) == ([0, 1], 1)
    assert R.verify(z, [0, 0], [-1, 0], q, 0.0, [0, 1.0], noise) == ([0, 1], 0)
