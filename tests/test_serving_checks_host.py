"""What the calls around a decoder's attention refuse before any device call, and pins of their oracle."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2609_05228_gb300 import ace, build

INVALID, UNSUPPORTED = 1, 2
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ace.LIBPATH):
        build.build()
    ace._lib = None
    return ace.lib()


# ----------------------------------------------------------------------- the oracle


@pytest.mark.parametrize("m", range(8, 16))
@pytest.mark.parametrize("e", [-20, 0, 7])
def test_oracle_scale_is_the_least_that_holds(m, e):
    s = m * 2.0 ** e
    assert S.scale4(7 * s) == s
    assert S.scale4(math.nextafter(7 * s, math.inf)) == (m + 1) * 2.0 ** e
    assert S.scale4(math.nextafter(7 * s, 0)) == s


def test_oracle_rows_in_4_bits():
    """A worked group: the largest 6.9 wants 6.9 / 7 = 0.9857, so s = 1; 2.5 and -2.5 go to the even neighbours."""
    x = np.zeros(40)
    x[:6] = [6.9, 2.5, -2.5, 3.5, 0.49, -6.51]
    x[32:34] = [0.875, -0.0625]
    codes, s, v = S.quantise4(x)
    assert s.tolist() == [1.0, 0.125]
    assert v[:6].tolist() == [7, 2, -2, 4, 0, -7] and v[32:34].tolist() == [0.875, 0.0]
    assert codes[:3].tolist() == [15 | 10 << 4, 6 | 12 << 4, 8 | 1 << 4] and codes[16] == 15 | 8 << 4
    assert np.isnan(S.quantise4(np.array([1.0, np.inf] + [0.0] * 38))[2][:32]).all()
    assert (np.abs(S.quantise4(np.random.default_rng(0).standard_normal((50, 64)))[2]) <= 4 * 8 / 7).all()


def test_oracle_rotation():
    """A quarter of a turn, lengths and angles between rows, and the inverse."""
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    assert np.allclose(S.rotate(x, [1], [math.pi / 2, math.pi])[0, 0], [-3, -2, 1, -4, 5])
    assert np.allclose(S.rotate(x, [1], [math.pi / 2, math.pi], "interleaved")[0, 0], [-2, 1, -3, -4, 5])
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 16))
    f = S.frequencies(16)
    dots = [(S.rotate(q, [p + 3], f) * S.rotate(k, [p], f)).sum() for p in (0, 5, 10 ** 6)]
    assert np.allclose(dots, dots[0])
    assert np.allclose(S.rotate(S.rotate(q, [9], f, magnitude=2.0), [9], f, inverse=True, magnitude=2.0), 4 * q)


def test_oracle_frequencies():
    t = S.frequencies(64)
    assert t[0] == 1 and np.allclose(t[16], 0.01)
    assert np.allclose(S.frequencies(64, scaling="linear", factor=4), t / 4)
    for kind in ("by_turns", "by_index"):
        f = S.frequencies(64, scaling=kind, factor=8, original_len=4096, low=1, high=32)
        turns = 4096 * t / (2 * math.pi)
        assert np.allclose(f[turns > 60], t[turns > 60]) and np.allclose(f[turns < 0.6], t[turns < 0.6] / 8)
        assert (np.diff(f) < 0).all()


def test_oracle_pages():
    """Two requests share a partly filled page: the first to grow copies it, the second keeps it."""
    table = np.array([[4, 2, -1], [4, 2, -1], [1, -1, -1]], np.int32)
    refs = np.array([0, 1, 2, 0, 2, 0], np.int32)
    t, r, missing, moves = S.reserve(table, np.array([20, 20, 16]), np.array([1, 1, 1]), refs, 16)
    assert t.tolist() == [[4, 0, -1], [4, 2, -1], [1, 3, -1]] and r.tolist() == [1, 1, 1, 1, 2, 0] and moves == [(2, 0, 4)] and missing == 0
    wide = np.concatenate([table, np.full((3, 5), -1, np.int32)], 1)
    t, r, missing, moves = S.reserve(wide, np.array([20, 20, 16]), np.array([1, 0, 100]), refs, 16)
    assert missing == 8 - 3 and (t == wide).all() and (r == refs).all() and moves == []
    new, lens, r = S.fork(table, np.array([20, 17, 16]), [1, -1, 2, 2], refs, 16)
    assert new.tolist() == [[4, 2, -1], [-1] * 3, [1, -1, -1], [1, -1, -1]] and lens.tolist() == [17, 0, 16, 16] and r.tolist() == [0, 2, 1, 0, 1, 0]
    t, r, n, at, moves = S.compact(table, refs)
    assert n == 3 and moves == [(4, 0)] and t.tolist() == [[0, 2, -1], [0, 2, -1], [1, -1, -1]] and at.tolist() == [-1, 1, 2, -1, 0, -1]


# ----------------------------------------------------------------------- the C calls


def test_struct_layout(tmp_path):
    src = tmp_path / "layout.c"
    fields = ["head_dim", "scaling", "base", "original_len", "low", "magnitude"]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ace.h"\nint main(void) { printf("%zu %d", sizeof(ace_rope_desc), ACE_KV_INT4);'
                   + "".join(f' printf(" %zu", offsetof(ace_rope_desc, {f}));' for f in fields) + " return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in got] == [ctypes.sizeof(ace.ace_rope_desc), ace.ACE_KV_INT4] + [getattr(ace.ace_rope_desc, f).offset for f in fields]


def _rope(L, divisors=None, **kw):
    d = dict(head_dim=64, rot_dim=64, layout=0, dtype=0, scaling=0, base=1e4, factor=1.0, original_len=0.0, low=1.0, high=32.0, magnitude=1.0)
    d.update(kw)
    out = ctypes.c_void_p(7)
    st = L.ace_rope_create(ctypes.byref(ace.ace_rope_desc(*d.values())), divisors, None, ctypes.byref(out))
    assert out.value is None
    return st


@pytest.mark.parametrize("kw,want,text", [
    (dict(head_dim=60), UNSUPPORTED, b"head_dim"), (dict(head_dim=264), UNSUPPORTED, b"head_dim"), (dict(head_dim=0), UNSUPPORTED, b"head_dim"),
    (dict(rot_dim=0), INVALID, b"rot_dim"), (dict(rot_dim=7), INVALID, b"rot_dim"), (dict(rot_dim=66), INVALID, b"rot_dim"),
    (dict(layout=2), INVALID, b"layout"), (dict(dtype=2), INVALID, b"dtype"), (dict(scaling=4), INVALID, b"scaling"), (dict(scaling=-1), INVALID, b"scaling"),
    (dict(base=1.0), INVALID, b"base"), (dict(base=math.nan), INVALID, b"base"), (dict(base=math.inf), INVALID, b"base"),
    (dict(magnitude=0.0), INVALID, b"magnitude"), (dict(magnitude=1e39), INVALID, b"magnitude"), (dict(magnitude=math.nan), INVALID, b"magnitude"),
    (dict(scaling=1, factor=0.0), INVALID, b"factor"), (dict(scaling=1, factor=math.inf), INVALID, b"factor"),
    (dict(scaling=2), INVALID, b"original_len"), (dict(scaling=3, original_len=10.0, low=0.0), INVALID, b"low"),
    (dict(scaling=3, original_len=10.0, low=32.0), INVALID, b"low"), (dict(scaling=2, original_len=10.0, high=math.inf), INVALID, b"high"),
    (dict(scaling=2, original_len=math.nan), INVALID, b"original_len"), (dict(scaling=1, factor=5e-324), INVALID, b"finite")])
def test_rope_create_refuses(L, kw, want, text):
    assert _rope(L, **kw) == want and text in L.ace_last_error_message()


def test_rope_create_refuses_divisors_and_null(L):
    for bad in (0.0, -1.0, math.nan, math.inf):
        d = (ctypes.c_double * 32)(*([1.0] * 31 + [bad]))
        assert _rope(L, d) == INVALID and b"divisors" in L.ace_last_error_message()
    out = ctypes.c_void_p(7)
    assert L.ace_rope_create(None, None, None, ctypes.byref(out)) == INVALID
    assert L.ace_rope_create(ctypes.byref(ace.ace_rope_desc()), None, None, None) == INVALID
    L.ace_rope_destroy(None)
    with pytest.raises(ValueError, match="divisors"):
        ace.ace_rope_create(ace.ace_rope_desc(64, 32), [1.0] * 15)
    for kw in (dict(layout="left"), dict(scaling="twice"), dict(dtype="f16")):
        with pytest.raises(ValueError):
            ace.AceRope(64, **kw)


def test_int4_create_refuses(L):
    out = ctypes.c_void_p(7)
    d = ace.ace_kv_desc(1, 4, 16, 2, 64, 0, ace.ACE_KV_INT4)
    for args, text in (((16, 16, None, 16), b"k_scale"), ((16, 16, 16, None), b"k_scale"), ((16, 16, 24, 16), b"scales"), ((24, 16, 16, 16), b"pools")):
        assert L.ace_kv_create(ctypes.byref(d), *args, None, ctypes.byref(out)) == INVALID and text in L.ace_last_error_message()
    with pytest.raises(ValueError, match="int4"):
        ace.AceKvCache(2, 64, 16, 4, fmt="int8")


class Handle:
    """Memory that reads as a handle: what a call checks of it before it asks for the device. kv: desc; rope: desc."""

    def __init__(self, desc):
        self.buf = ctypes.create_string_buffer(bytes(desc) + b"\0" * 1024)
        self.at = ctypes.addressof(self.buf)


@pytest.fixture
def kv():
    # (layers, n_pages, page_size, n_kv_heads, head_dim, dtype, format), device, num_sms, elem
    return Handle(bytes(ace.ace_kv_desc(2, 100, 16, 2, 64, 0, 4)) + bytes((ctypes.c_int * 3)(0, 1, 2)))


@pytest.fixture
def rope():
    return Handle(ace.ace_rope_desc(64, 64, 0, 0, 0, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0))


def _apply(L, handle, **kw):
    a = dict(rope=handle.at, inverse=0, positions=64, T=4, q=1 << 20, qt=128, qh=64, heads=2, qo=2 << 20, qot=128, qoh=64, k=3 << 20, kt=128, kh=64,
             kv_heads=2, ko=4 << 20, kot=128, koh=64, stream=None)
    a.update(kw)
    return L.ace_rope_apply(*a.values())


@pytest.mark.parametrize("kw,text", [
    (dict(rope=None), b"rope"), (dict(T=-1), b"T"), (dict(heads=-1), b"n_heads"), (dict(kv_heads=-1), b"n_kv_heads"), (dict(qt=-1), b"strides"), (dict(koh=-1), b"strides"),
    (dict(positions=None), b"non-NULL"), (dict(q=None), b"non-NULL"), (dict(qo=None), b"non-NULL"), (dict(k=None), b"non-NULL"), (dict(ko=None), b"non-NULL"),
    (dict(q=(1 << 20) + 1), b"aligned"), (dict(ko=(1 << 20) + 1), b"aligned"),
    (dict(qot=0), b"apart"), (dict(qoh=0), b"apart"), (dict(qoh=32), b"apart"), (dict(qot=64), b"apart"), (dict(qot=127), b"apart"), (dict(kot=64, koh=64), b"apart"),
    (dict(qot=64, qoh=255), b"apart"),
    (dict(qo=1 << 20, qot=256), b"strides"), (dict(ko=3 << 20, kot=64, koh=256), b"strides"), (dict(q=2 << 20, qt=0), b"strides")])
def test_rope_apply_refuses(L, rope, kw, text):
    assert _apply(L, rope, **kw) == INVALID and text in L.ace_last_error_message()


def _rotated(L, cache, handle, **kw):
    a = dict(kv=cache.at, layer=0, rope=handle.at, positions=64, q=1 << 20, qt=128, qh=64, heads=2, qo=2 << 20, qot=128, qoh=64, k=3 << 20, kt=128, kh=64,
             v=4 << 20, vt=128, vh=64, slots=64, T=4, stream=None)
    a.update(kw)
    return L.ace_kv_write_rotated(*a.values())


@pytest.mark.parametrize("kw,text", [
    (dict(kv=None), b"non-NULL"), (dict(rope=None), b"non-NULL"), (dict(layer=2), b"layer"), (dict(layer=-1), b"layer"), (dict(T=-1), b"T"), (dict(heads=-1), b"n_heads"),
    (dict(vt=-1), b"strides"), (dict(positions=None), b"non-NULL"), (dict(k=None), b"non-NULL"), (dict(v=None), b"non-NULL"), (dict(slots=None), b"non-NULL"),
    (dict(q=None), b"non-NULL"), (dict(qo=None), b"non-NULL"), (dict(v=(1 << 20) + 1), b"aligned"), (dict(qot=64), b"apart"), (dict(qo=1 << 20, qot=192), b"strides")])
def test_write_rotated_refuses(L, kv, rope, kw, text):
    assert _rotated(L, kv, rope, **kw) == INVALID and text in L.ace_last_error_message()


def test_write_rotated_refuses_another_kind(L, kv):
    for d in (ace.ace_rope_desc(128, 64, 0, 0, 0, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0), ace.ace_rope_desc(64, 64, 0, 1, 0, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0)):
        assert _rotated(L, kv, Handle(d)) == INVALID and b"same head_dim" in L.ace_last_error_message()


A = [(i + 1) << 20 for i in range(8)]


@pytest.mark.parametrize("call,args,text", [
    ("ace_kv_fork", (A[0], A[1], -1, A[2], 4, 3, A[3], A[4], A[5]), b"B"), ("ace_kv_fork", (A[0], A[1], 4, A[2], -4, 3, A[3], A[4], A[5]), b"B"),
    ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 0, A[3], A[4], A[5]), b"max_pages"), ("ace_kv_fork", (None, A[1], 4, A[2], 4, 3, A[3], A[4], A[5]), b"non-NULL"),
    ("ace_kv_fork", (A[0], None, 4, A[2], 4, 3, A[3], A[4], A[5]), b"non-NULL"), ("ace_kv_fork", (A[0], A[1], 4, None, 4, 3, A[3], A[4], A[5]), b"non-NULL"),
    ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, None, A[4], A[5]), b"non-NULL"), ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[3], None, A[5]), b"non-NULL"),
    ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[3], A[4], None), b"non-NULL"), ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[3], A[0], A[5]), b"overlap"),
    ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[3], A[0] + 44, A[5]), b"overlap"), ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[3], A[4], A[1]), b"overlap"),
    ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[3], A[4], A[4] + 44), b"overlap"), ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[3], A[3] + 396, A[5]), b"overlap"),
    ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[0] + 44, A[4], A[5]), b"overlap"), ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[1] + 12, A[4], A[5]), b"overlap"),
    ("ace_kv_fork", (A[0], A[1], 4, A[2], 4, 3, A[2] - 396, A[4], A[5]), b"overlap"),
    ("ace_kv_reserve", (A[0], 3, A[1], A[2], -1, A[3], A[4]), b"B"), ("ace_kv_reserve", (A[0], 0, A[1], A[2], 4, A[3], A[4]), b"max_pages"),
    ("ace_kv_reserve", (None, 3, A[1], A[2], 4, A[3], A[4]), b"non-NULL"), ("ace_kv_reserve", (A[0], 3, None, A[2], 4, A[3], A[4]), b"non-NULL"),
    ("ace_kv_reserve", (A[0], 3, A[1], None, 4, A[3], A[4]), b"non-NULL"), ("ace_kv_reserve", (A[0], 3, A[1], A[2], 4, None, A[4]), b"non-NULL"),
    ("ace_kv_reserve", (A[0], 3, A[1], A[2], 4, A[3], None), b"non-NULL"), ("ace_kv_reserve", (A[0], 3, A[0] + 44, A[2], 4, A[3], A[4]), b"overlap"),
    ("ace_kv_reserve", (A[0], 3, A[1], A[2], 4, A[3], A[1] + 12), b"overlap"), ("ace_kv_reserve", (A[0], 3, A[1], A[2], 4, A[2] - 396, A[4]), b"overlap"),
    ("ace_kv_release", (A[0], 3, A[1], A[2], -1, A[3]), b"B"), ("ace_kv_release", (A[0], 0, A[1], A[2], 4, A[3]), b"max_pages"),
    ("ace_kv_release", (None, 3, A[1], A[2], 4, A[3]), b"non-NULL"), ("ace_kv_release", (A[0], 3, None, A[2], 4, A[3]), b"non-NULL"),
    ("ace_kv_release", (A[0], 3, A[1], None, 4, A[3]), b"non-NULL"), ("ace_kv_release", (A[0], 3, A[1], A[2], 4, None), b"non-NULL"),
    ("ace_kv_release", (A[0], 3, A[1], A[1] + 4, 4, A[3]), b"overlap"),
    ("ace_kv_compact", (A[0], 3, -1, A[1], A[2], None), b"B"), ("ace_kv_compact", (A[0], 0, 4, A[1], A[2], None), b"max_pages"),
    ("ace_kv_compact", (None, 3, 4, A[1], A[2], None), b"non-NULL"), ("ace_kv_compact", (A[0], 3, 4, None, A[2], None), b"non-NULL"),
    ("ace_kv_compact", (A[0], 3, 4, A[1], None, None), b"non-NULL"), ("ace_kv_compact", (A[0], 3, 4, A[0] + 4, A[2], None), b"overlap"),
    ("ace_kv_compact", (A[0], 3, 4, A[1], A[2], A[1]), b"overlap"), ("ace_kv_compact", (A[0], 3, 4, A[1], A[2], A[2] - 4), b"overlap"),
    ("ace_kv_copy_pages", (A[0], A[1], -1), b"n"), ("ace_kv_copy_pages", (None, A[1], 4), b"non-NULL"), ("ace_kv_copy_pages", (A[0], None, 4), b"non-NULL")])
def test_page_calls_refuse(L, kv, call, args, text):
    assert getattr(L, call)(kv.at, *args, None) == INVALID and text in L.ace_last_error_message()
    assert getattr(L, call)(None, *args, None) == INVALID and b"NULL" in L.ace_last_error_message()


def test_reserve_refuses_sizes(L, kv):
    assert L.ace_kv_reserve(kv.at, 1 << 30, 3, 2 << 30, 3 << 30, 8193, 4 << 30, 5 << 30, None) == UNSUPPORTED
    assert L.ace_kv_reserve(kv.at, 1 << 30, (1 << 26) + 1, 2 << 30, 3 << 30, 8, 4 << 30, 5 << 30, None) == UNSUPPORTED


# ----------------------------------------------------------------------- the binding


class Calls:
    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            return 0
        return call


@pytest.fixture
def cache(monkeypatch):
    """A cache and a rope over a library that does nothing; CPU tensors count as the GPU's."""
    fake = Calls()
    monkeypatch.setattr(ace, "lib", lambda: fake)
    want = ace._want

    def on_cpu(name, t, *args):
        try:
            want(name, t, *args)
        except ValueError as e:
            if "on a GPU" not in str(e):
                raise
    monkeypatch.setattr(ace, "_want", on_cpu)
    monkeypatch.setattr(ace, "_raw_stream", lambda device: 0, raising=False)
    c = ace.AceKvCache.__new__(ace.AceKvCache)
    c.handle, c._dt, c.n_kv_heads, c.head_dim, c.n_pages = 5, "bfloat16", 2, 64, 100
    r = ace.AceRope.__new__(ace.AceRope)
    r.handle, r._dt, r.head_dim = 6, "bfloat16", 64
    yield c, r, fake.made
    c.handle = r.handle = None          # there is nothing to free


def _i(*s):
    return torch.zeros(*s, dtype=torch.int32)


@pytest.mark.parametrize("name,t", [
    ("page_table", torch.zeros(4, 3)), ("page_table", _i(12)), ("page_table", _i(4, 6)[:, ::2]), ("refs", _i(99)), ("lens", _i(5)), ("parents", torch.zeros(5, dtype=torch.int64)),
    ("new_table", _i(5, 4)), ("new_table", _i(4, 3)), ("new_lens", _i(4))])
def test_fork_refuses_tensors(cache, name, t):
    a = dict(page_table=_i(4, 3), lens=_i(4), parents=_i(5), refs=_i(100), new_table=_i(5, 3), new_lens=_i(5))
    cache[0].fork(**a)
    assert cache[2].pop()[0] == "ace_kv_fork"
    with pytest.raises(ValueError, match=name):
        cache[0].fork(**dict(a, **{name: t}))
    assert cache[2] == []


@pytest.mark.parametrize("call,name,t", [
    ("reserve", "page_table", torch.zeros(4, 3)), ("reserve", "lens", _i(3)), ("reserve", "grow", _i(4, 1)), ("reserve", "refs", _i(101)), ("reserve", "missing", _i(2)),
    ("release", "ended", torch.zeros(4, dtype=torch.bool)), ("release", "lens", _i(3)), ("release", "refs", torch.zeros(100)),
    ("compact", "used", _i(0)), ("compact", "new_page", _i(99)), ("compact", "refs", _i(1)), ("copy_pages", "src", torch.zeros(3)), ("copy_pages", "dst", _i(4))])
def test_page_calls_refuse_tensors(cache, call, name, t):
    a = {"reserve": dict(page_table=_i(4, 3), lens=_i(4), grow=_i(4), refs=_i(100), missing=_i(1)),
         "release": dict(page_table=_i(4, 3), lens=_i(4), ended=_i(4), refs=_i(100)),
         "compact": dict(page_table=_i(4, 3), refs=_i(100), used=_i(1), new_page=_i(100)), "copy_pages": dict(src=_i(3), dst=_i(3))}[call]
    getattr(cache[0], call)(**a)
    assert cache[2].pop()[0] == "ace_kv_" + call
    with pytest.raises(ValueError, match=name):
        getattr(cache[0], call)(**dict(a, **{name: t}))
    assert cache[2] == []


@pytest.mark.parametrize("name,t", [
    ("q", torch.zeros(4, 3, 64)), ("q", torch.zeros(4, 3, 32, dtype=torch.bfloat16)), ("q_out", torch.zeros(4, 2, 64, dtype=torch.bfloat16)), ("positions", _i(3)),
    ("positions", torch.zeros(4, dtype=torch.int64)), ("k", torch.zeros(3, 2, 64, dtype=torch.bfloat16)), ("k", torch.zeros(4, 2, 128, dtype=torch.bfloat16)[..., ::2]),
    ("v", torch.zeros(5, 2, 64, dtype=torch.bfloat16)), ("slots", _i(4))])
def test_rotations_refuse_tensors(cache, name, t):
    c, r, made = cache
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)       # noqa: E731
    a = dict(layer=0, rope=r, positions=_i(4), q=b(4, 3, 64), q_out=b(4, 3, 64), k=b(4, 2, 64), v=b(4, 2, 64), slots=torch.zeros(4, dtype=torch.int64))
    c.write_rotated(**a)
    assert made.pop()[0] == "ace_kv_write_rotated"
    with pytest.raises(ValueError):
        c.write_rotated(**dict(a, **{name: t}))
    if name not in ("v", "slots"):
        a = dict(positions=_i(4), q=b(4, 3, 64), q_out=b(4, 3, 64), k=b(4, 2, 64), k_out=b(4, 2, 64))
        r.apply(**a)
        assert made.pop()[0] == "ace_rope_apply"
        with pytest.raises(ValueError):
            r.apply(**dict(a, **{name: t}))
        with pytest.raises(ValueError, match="together"):
            r.apply(**dict(a, k_out=None))
    assert made == []
