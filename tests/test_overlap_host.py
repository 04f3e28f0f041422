"""Whether rows of tensors share memory: the host's answer against a count of the bytes, and what the rotary calls refuse by it."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2609_05228_gb300 import ace, build

from test_serving_checks_host import INVALID, Handle, L, _apply, _rotated, kv, rope       # noqa: F401

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_05228_gb300", "csrc")


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "overlap.cpp").write_text('#include "ace_overlap.h"\nextern "C" int meet(const long long* a, const long long* b) {\n'
                                   "    auto of = [](const long long* x) { return ace::RowSet{(uintptr_t)x[0], x[1], x[2], x[3], x[4], x[5]}; };\n"
                                   "    return ace::rows_meet(of(a), of(b));\n}\n")
    lib = d / "overlap.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", CSRC, str(d / "overlap.cpp"), "-o", str(lib)], check=True)
    f = ctypes.CDLL(str(lib)).meet
    return lambda a, b: bool(f((ctypes.c_longlong * 6)(*a), (ctypes.c_longlong * 6)(*b)))


def _bytes(s):
    at, token, head, tokens, heads, row = s
    return {at + t * token + h * head + i for t in range(tokens) for h in range(heads) for i in range(row)}


def test_rows_meet_is_exact(meet):
    """Against the sets of bytes: strides alike and not, of zero, rows of different length, single rows, none."""
    rng = np.random.default_rng(0)
    seen = [0, 0]
    for _ in range(6000):
        def some():
            row = int(rng.integers(1, 9))
            return [1000 + int(rng.integers(-60, 60)), int(rng.integers(0, 40)), int(rng.integers(0, 40)), int(rng.integers(0, 6)), int(rng.integers(0, 5)), row]
        a, b = some(), some()
        if rng.random() < 0.5:
            b[1] = a[1]
        if rng.random() < 0.5:
            b[2] = a[2]
        want = bool(_bytes(a) & _bytes(b))
        assert meet(a, b) == want == meet(b, a), (a, b)
        seen[want] += 1
    assert min(seen) > 500


def test_rows_meet_at_large_sizes(meet):
    """Projections of 2^20 tokens whose q, k and v alternate; strides near the largest; other strides row by row."""
    D, T = 256, 1 << 20
    q, k = [1 << 40, 80 * D, D, T, 64, D], [(1 << 40) + 64 * D, 80 * D, D, T, 8, D]
    assert not meet(q, k) and meet(q, k[:0] + [k[0] - 1] + k[1:]) and not meet(q, [k[0] + 8 * D] + k[1:])
    assert meet(q, [k[0] + 8 * D + 1] + k[1:])      # the last v head reaches the next token's q
    by_heads = [[(1 << 40) + i * T * D, D, 3 * T * D, T, 8, D] for i in range(3)]
    assert not meet(*by_heads[:2]) and not meet(*by_heads[1:]) and meet(by_heads[0], [by_heads[1][0] - 1] + by_heads[1][1:])
    assert not meet([1 << 40, (1 << 62), D, 3, 2, D], [(1 << 40) + 2 * D, (1 << 62) + 1, D, 3, 1, D])
    assert not meet([1 << 40, 3 * D, 0, 4000, 1, D], [(1 << 40) + D, 6 * D, 0, 2000, 1, D])
    assert meet([1 << 40, 3 * D, 0, 4000, 1, D], [(1 << 40) + D, 6 * D, 0, 2001, 1, 2 * D + 1])


M = 1 << 20
PACKED = dict(qt=384, qh=64, kt=384, kh=64)         # q, k and v of two heads of 64 in one projection, elements of 2 bytes


@pytest.mark.parametrize("kw", [
    dict(qo=M + 128), dict(qo=M + 2), dict(qo=M - 2), dict(qo=M + 4 * 256 - 2), dict(qo=3 * M), dict(qo=3 * M + 4 * 256 - 2), dict(ko=M), dict(ko=2 * M + 128),
    dict(ko=3 * M + 128), dict(PACKED, k=M + 256, qo=M + 128, qot=384), dict(PACKED, k=M + 256, qo=M + 256, qot=384, ko=4 * M), dict(qo=64), dict(ko=66),
    dict(q=M, qt=0, qo=M + 126, qot=128), dict(qo=M, qot=128, ko=M + 128, kt=128, k=5 * M)])
def test_rope_apply_refuses_overlaps(L, rope, kw):       # noqa: F811
    assert _apply(L, rope, **kw) == INVALID and b"overlap" in L.ace_last_error_message()


@pytest.mark.parametrize("kw", [
    dict(), dict(qo=M), dict(qo=M, ko=3 * M), dict(PACKED, k=M + 256, qo=M, qot=384, ko=M + 256, kot=384), dict(PACKED, k=M + 256, qo=M + 512, qot=384),
    dict(qo=M + 4 * 256), dict(qo=M - 4 * 256), dict(k=M), dict(qt=0, qo=M + 256), dict(heads=0, qo=3 * M), dict(kv_heads=0, ko=M, k=M + 2), dict(T=0, qo=M + 2)])
def test_rope_apply_takes_rows_apart(L, rope, kw):       # noqa: F811
    """What passes the checks ends at the device, which is another than the call's or none."""
    _apply(L, rope, **kw)
    assert b"overlap" not in L.ace_last_error_message()


@pytest.mark.parametrize("kw", [
    dict(qo=M + 128), dict(qo=3 * M), dict(qo=4 * M + 4 * 256 - 2), dict(qo=64), dict(qo=M - 2, q=5 * M, slots=M), dict(qt=384, kt=384, k=M + 256, vt=384, v=M + 512, qot=384, qo=M + 512)])
def test_write_rotated_refuses_overlaps(L, kv, rope, kw):        # noqa: F811
    assert _rotated(L, kv, rope, **kw) == INVALID and b"overlap" in L.ace_last_error_message()


@pytest.mark.parametrize("kw", [
    dict(), dict(qo=M), dict(qt=384, kt=384, k=M + 256, vt=384, v=M + 512, qot=384, qo=M), dict(k=M, v=M), dict(heads=0, qo=3 * M), dict(T=0, qo=M + 2)])
def test_write_rotated_takes_rows_apart(L, kv, rope, kw):        # noqa: F811
    _rotated(L, kv, rope, **kw)
    assert b"overlap" not in L.ace_last_error_message()
