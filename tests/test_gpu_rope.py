"""Rotary positions on the GPU against their formulas in 64 bits, alone and on the way into the cache."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2609_05228_gb300 import ace

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SCALED = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="by_turns", factor=8.0, original_len=8192, low=1.0, high=4.0, base=5e5),
          dict(scaling="by_index", factor=16.0, original_len=4096, low=1.0, high=32.0, magnitude=1.2772588722239782)]
FAR = np.array([0, 1, 2, 7, 1000, 4095, 123457, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -1, -5000, -(1 << 31)])


def _rows(rng, shape, dtype):
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def _freq(rot, kind):
    return S.frequencies(rot, **{k: v for k, v in kind.items() if k != "magnitude"})


def _check(got, want, x, rot, layout, dtype, magnitude=1.0):
    """Sine and cosine: 2^-53 of the angle for the frequency's last place at positions to 2^31 (2^-22 at most), 2 ulp (2^-22) of
    sincospif, the rounding of what it is taken of; two products and a sum, 2^-24 each. In all 6 * 2^-22 of the pair's
    larger element, twice over. bf16 rounds the result besides."""
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    tol = np.zeros_like(x)
    tol[..., a] = tol[..., b] = 12 * 2.0 ** -22 * magnitude * np.maximum(np.abs(x[..., a]), np.abs(x[..., b]))
    tol[..., :rot] += (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want[..., :rot])
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()        # dimensions that are not turned: equal


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot", [(8, 2), (8, 8), (64, 64), (64, 32), (80, 80), (128, 128), (128, 64), (128, 48), (128, 6), (256, 256), (200, 100), (256, 16)])
@pytest.mark.parametrize("kind", range(4))
def test_rotation(dtype, layout, D, rot, kind):
    """Every layout, part and scaling, at near, far and negative positions; the inverse."""
    rng = np.random.default_rng(D + rot)
    T = len(FAR)
    rope = ace.AceRope(D, rot, layout, dtype=dtype, **SCALED[kind])
    m = SCALED[kind].get("magnitude", 1.0)
    q, qd = _rows(rng, (T, 5, D), dtype)
    k, kd = _rows(rng, (T, 2, D), dtype)
    pos = torch.tensor(FAR, dtype=torch.int32, device="cuda")
    f = _freq(rot, SCALED[kind])
    for inverse in (False, True):
        qo, ko = torch.full_like(q, 9), torch.full_like(k, 9)
        rope.apply(pos, q, qo, k, ko, inverse=inverse)
        for got, x in ((qo, qd), (ko, kd)):
            _check(got, S.rotate(x, FAR, f, layout, m, inverse), x, rot, layout, dtype, m)


@pytest.mark.parametrize("T,Hq,H", [(1, 1, 0), (1, 32, 4), (3, 1, 1), (700, 1, 0), (129, 2, 1), (67, 40, 8), (300, 7, 3)])
@pytest.mark.parametrize("D", [64, 128, 256, 72])
def test_rotation_sizes(T, Hq, H, D):
    """Blocks with rows of one token and of many; without k."""
    rng = np.random.default_rng(T)
    rope = ace.AceRope(D, D, "half", dtype="bf16")
    q, qd = _rows(rng, (T, Hq, D), "bf16")
    pos = rng.integers(0, 100000, T)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    qo = torch.full((T + 1, Hq, D), 9.0, dtype=torch.bfloat16, device="cuda")
    f = _freq(D, {})
    if H:
        k, kd = _rows(rng, (T, H, D), "bf16")
        ko = torch.full((T + 1, H, D), 9.0, dtype=torch.bfloat16, device="cuda")
        rope.apply(p, q, qo[:T], k, ko[:T])
        _check(ko[:T], S.rotate(kd, pos, f), kd, D, "half", "bf16")
        assert (ko[T] == 9).all()
    else:
        rope.apply(p, q, qo[:T])
    _check(qo[:T], S.rotate(qd, pos, f), qd, D, "half", "bf16")
    assert (qo[T] == 9).all()
    rope.apply(p[:0], q[:0], qo[:0])
    rope.apply(p, q[:, :0], qo[:T, :0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,D,rot", [("half", 128, 128), ("half", 128, 24), ("interleaved", 64, 32), ("half", 256, 256)])
def test_rotation_strides_and_in_place(dtype, layout, D, rot):
    """Rows inside a fused projection (aligned and not), head-major results, results in the rows' place: all the same bits."""
    rng = np.random.default_rng(rot)
    T, Hq, H = 21, 6, 2
    rope = ace.AceRope(D, rot, layout, dtype=dtype)
    pos = torch.tensor(rng.integers(0, 5000, T), dtype=torch.int32, device="cuda")
    q, _ = _rows(rng, (T, Hq, D), dtype)
    k, _ = _rows(rng, (T, H, D), dtype)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rope.apply(pos, q, qo, k, ko)
    for shift in (0, 3):
        row = torch.zeros(T, (Hq + 2 * H) * D + 8, dtype=DT[dtype], device="cuda")
        heads = row[:, shift: shift + (Hq + 2 * H) * D].unflatten(1, (-1, D))
        qv, kv = heads[:, :Hq], heads[:, Hq: Hq + H]
        qv.copy_(q)
        kv.copy_(k)
        out = torch.empty(Hq, T, D, dtype=DT[dtype], device="cuda").transpose(0, 1)
        k2 = torch.empty_like(k)
        rope.apply(pos, qv, out, kv, k2)
        assert torch.equal(out, qo) and torch.equal(k2, ko)
        rope.apply(pos, qv, qv, kv, kv)
        assert torch.equal(qv, qo) and torch.equal(kv, ko) and heads[:, Hq + H:].count_nonzero() == 0
    # q of one row for all tokens
    one = q[:1].expand(T, Hq, D)
    rope.apply(pos, one, out)
    each = torch.empty_like(q)
    rope.apply(pos, one.contiguous(), each)
    assert torch.equal(out, each)


def test_gradient_against_differences():
    """The inverse of the call is the transpose of its matrix: <g, rotate(x + e) - rotate(x - e)> / 2 = <inverse(g), e>. fp32 sums of
    T Hq D products of N(0, 1), each off by 2^-19 at most (12 * 2^-22 a turn)."""
    rng = np.random.default_rng(3)
    for layout, kind in (("half", 3), ("interleaved", 2)):
        T, Hq, D, rot = 9, 3, 64, 48
        rope = ace.AceRope(D, rot, layout, dtype="f32", **SCALED[kind])
        pos = torch.tensor(rng.integers(0, 100000, T), dtype=torch.int32, device="cuda")
        x, e, g = (_rows(rng, (T, Hq, D), "f32")[0] for _ in range(3))
        up, down, back = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        rope.apply(pos, x + e, up)
        rope.apply(pos, x - e, down)
        rope.apply(pos, g, back, inverse=True)
        left, right = (g.double() * (up.double() - down.double())).sum() / 2, (back.double() * e.double()).sum()
        assert abs(left - right) <= 2.0 ** -18 * (g.abs().double() * (x.abs() + e.abs() + 1).double()).sum()


def test_divisors_divide_the_frequencies():
    rng = np.random.default_rng(4)
    D = 64
    div = np.exp(rng.uniform(0, 3, D // 2))
    rope = ace.AceRope(D, dtype="f32", scaling="linear", factor=2.0, divisors=div)
    pos = np.array([0, 77, 100000])
    q, qd = _rows(rng, (3, 2, D), "f32")
    out = torch.empty_like(q)
    rope.apply(torch.tensor(pos, dtype=torch.int32, device="cuda"), q, out)
    _check(out, S.rotate(qd, pos, S.frequencies(D, scaling="linear", factor=2.0, divisors=div)), qd, D, "half", "f32")


@pytest.mark.parametrize("fmt", ["int4", "fp8", "plain"])
@pytest.mark.parametrize("dtype,D,rot,layout", [("bf16", 128, 128, "half"), ("bf16", 64, 32, "interleaved"), ("bf16", 72, 24, "half"), ("f32", 200, 200, "half"),
                                                ("bf16", 256, 256, "half"), ("f32", 40, 6, "interleaved")])
@pytest.mark.parametrize("T,Hq,H,shift", [(1, 8, 2, 0), (37, 3, 1, 0), (130, 16, 4, 1)])
def test_write_rotated_is_the_two_calls(fmt, dtype, D, rot, layout, T, Hq, H, shift):
    """The same bits in q's results, the pools and the scales as a rotation and a write, from rows of a fused projection; tokens that
    are left out have their q turned."""
    rng = np.random.default_rng(T + D)
    page, n_pages = 16, -(-T // 16) + 2
    rope = ace.AceRope(D, rot, layout, dtype=dtype, **SCALED[2])
    row = torch.empty(T, (Hq + 2 * H) * D + 8, dtype=DT[dtype], device="cuda")
    rows = row[:, shift: shift + (Hq + 2 * H) * D].unflatten(1, (-1, D))
    rows.copy_(_rows(rng, tuple(rows.shape), dtype)[0])
    q, k, v = rows[:, :Hq], rows[:, Hq: Hq + H], rows[:, Hq + H:]
    pos = torch.tensor(rng.integers(0, 70000, T), dtype=torch.int32, device="cuda")
    slots = rng.permutation(n_pages * page)[:T]
    if T > 5:
        slots[[1, 4]] = -1
    slots = torch.from_numpy(slots).cuda()
    a, b = (ace.AceKvCache(H, D, page, n_pages, 2, dtype, fmt) for _ in range(2))
    for kv in (a, b):
        for p in (kv.k_pool, kv.v_pool) + ((kv.k_scale, kv.v_scale) if fmt != "plain" else ()):
            p.view(torch.uint8).fill_(0x21)
    qa, qb, kr = torch.empty(T, Hq, D, dtype=DT[dtype], device="cuda"), torch.empty(T, Hq, D, dtype=DT[dtype], device="cuda"), torch.empty(T, H, D, dtype=DT[dtype], device="cuda")
    rope.apply(pos, q, qa, k, kr)
    a.write(1, kr, v, slots)
    a.sync()
    b.write_rotated(1, rope, pos, q, qb, k, v, slots)
    b.sync()
    assert torch.equal(qa, qb)
    for name in ("k_pool", "v_pool") + (("k_scale", "v_scale") if fmt != "plain" else ()):
        assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8)), name
    # in place, without q, without tokens
    b.write_rotated(0, rope, pos, q[:, :0], qb[:, :0], k, v, slots)
    b.write_rotated(0, rope, pos[:0], q[:0], qb[:0], k[:0], v[:0], slots[:0])
    b.sync()
    assert torch.equal(b.k_pool[0].view(torch.uint8), b.k_pool[1].view(torch.uint8))
    b.write_rotated(0, rope, pos, q, q, k, v, slots)
    b.sync()
    assert torch.equal(q, qa)


def test_write_rotated_reports_slots_outside():
    rope = ace.AceRope(64)
    kv = ace.AceKvCache(2, 64, 16, 2, 1, "bf16", "int4")
    x = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(x)
    kv.write_rotated(0, rope, pos, x, out, x, x, torch.tensor([0, 32, 1 << 40], device="cuda"))
    with pytest.raises(ace.AceError) as err:
        kv.sync()
    assert err.value.status == 1
    kv.sync()
    assert (out != 0).any(-1).all() and kv.v_pool[0, 0, :, 1:].count_nonzero() == 0 and kv.v_pool[0, 1].count_nonzero() == 0


def test_rotation_on_a_stream_and_in_a_graph():
    rng = np.random.default_rng(8)
    rope = ace.AceRope(128)
    q, _ = _rows(rng, (5, 4, 128), "bf16")
    pos = torch.tensor([3, 1, 4, 1, 5], dtype=torch.int32, device="cuda")
    want, out = torch.empty_like(q), torch.empty_like(q)
    rope.apply(pos, q, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rope.apply(pos, q, out)
    side.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rope.apply(pos, q, out)
    pos += 100
    rope.apply(pos, q, want)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
