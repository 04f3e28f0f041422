"""Rows in 4 bits, rotary positions and the cache's pages on the GPU against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as R
from oracle import serving_oracle as S
from paper_2609_05228_gb300 import ace

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}        # a rounding, relative to the value (bf16: half of 2^-7)


def _rows(rng, shape, dtype, scale=1.0):
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def _int(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


# ----------------------------------------------------------------------- rows in 4 bits


@pytest.mark.parametrize("dtype,D", [("bf16", 8), ("bf16", 64), ("bf16", 72), ("bf16", 128), ("bf16", 256), ("f32", 40), ("f32", 96), ("f32", 200)])
@pytest.mark.parametrize("T,H,page", [(1, 1, 16), (37, 3, 32), (300, 2, 128)])
def test_int4_write_and_read_are_exact(dtype, D, T, H, page):
    """Codes, scales and read-back values are the definition's, bit for bit; rows that no token names stay."""
    rng = np.random.default_rng(T + D)
    layers, n_pages = 3, -(-T // page) + 2
    kv = ace.AceKvCache(H, D, page, n_pages, layers, dtype, "int4")
    for pool in (kv.k_pool, kv.v_pool, kv.k_scale, kv.v_scale):
        pool.view(torch.uint8).fill_(0x15)
    k, kd = _rows(rng, (T, H, D), dtype, np.exp(rng.uniform(-30, 30, (T, H, 1))))
    v, vd = _rows(rng, (T, H, D), dtype, np.exp(rng.uniform(-2, 2, (T, H, D))))
    v[0], vd[0] = 0, 0
    slots = rng.permutation(n_pages * page)[:T]
    st = torch.from_numpy(slots).cuda()
    kv.write(1, k, v, st)
    k_out, v_out = torch.empty_like(k), torch.empty_like(v)
    kv.read(1, st, k_out, v_out)
    kv.sync()
    for xd, out, pool, scale in ((kd, k_out, kv.k_pool, kv.k_scale), (vd, v_out, kv.v_pool, kv.v_scale)):
        codes, s, value = S.quantise4(xd)
        assert (pool[1].cpu().numpy()[slots // page, :, slots % page] == codes).all()
        assert (scale[1].view(torch.int16).cpu().numpy().view(np.uint16)[slots // page, :, slots % page] == S.bf16_bits(s)).all()
        assert torch.equal(out.cpu(), torch.from_numpy(value).to(DT[dtype]))
        for p in (pool, scale):
            rest = p.view(torch.uint8).reshape(layers, n_pages, H, page, -1).movedim(2, 3).reshape(layers, n_pages * page, H, -1).cpu()
            keep = np.ones((layers, n_pages * page), bool)
            keep[1, slots] = False
            assert (rest[torch.from_numpy(keep)] == 0x15).all()


def test_int4_values_next_to_a_border():
    """fp32 values one step beside a half of a code, and largest values one step beside 7 scales: no rounding decides them."""
    D = 64
    x = np.zeros((1, 40, D), np.float32)
    s = np.float32(0.8125)
    for i in range(20):
        x[0, i, 0] = 7 * s                          # the group's scale is s
        half = np.arange(-6.5, 7, 1.0)[:14] * float(s)
        x[0, i, 1:15] = half
        x[0, i, 15:29] = np.nextafter(half.astype(np.float32), np.float32(np.inf))
        x[0, i, 32] = np.nextafter(np.float32(7 * (8 + i % 8) * 2.0 ** (i - 10)), np.float32(np.inf if i % 2 else -np.inf))
    for i in range(20, 40):
        x[0, i, :32] = np.nextafter(np.float32((i - 26.5) * 0.1171875), np.float32(-np.inf))
        x[0, i, 31] = 7 * 0.1171875
        x[0, i, 32] = 7 * (8 + i % 8) * 2.0 ** (i - 30)
    kv = ace.AceKvCache(40, D, 16, 1, 1, "f32", "int4")
    t, slot = torch.from_numpy(x).cuda(), torch.zeros(1, dtype=torch.int64, device="cuda")
    kv.write(0, t, t, slot)
    kv.sync()
    codes, scales, _ = S.quantise4(x[0])
    assert (kv.k_scale[0, 0, :, 0].view(torch.int16).cpu().numpy().view(np.uint16) == S.bf16_bits(scales)).all()
    assert (kv.k_pool[0, 0, :, 0].cpu().numpy() == codes).all()


def test_int4_values_that_are_not_finite_and_extremes():
    """A group with a NaN or an infinity is NaN and leaves the others alone; fp32's extremes keep within its scales."""
    D = 96
    x = np.zeros((1, 6, D), np.float32)
    x[0, :, 64:] = 1.0
    x[0, 0, 3], x[0, 1, 40], x[0, 2, 5] = np.nan, np.inf, -np.inf
    x[0, 3, :32] = np.finfo(np.float32).max
    x[0, 4, 5], x[0, 4, 40] = 1e-45, 2.0 ** -126 * 3.5
    x[0, 5, :3], x[0, 5, 32] = [2.0 ** -126 * 7, -(2.0 ** -125), 2.0 ** -127], 2.0 ** -126 * 7.5
    kv = ace.AceKvCache(6, D, 16, 1, 1, "f32", "int4")
    t, slot = torch.from_numpy(x).cuda(), torch.zeros(1, dtype=torch.int64, device="cuda")
    kv.write(0, t, t, slot)
    out = torch.empty(2, 1, 6, D, device="cuda")
    kv.read(0, slot, out[0], out[1])
    kv.sync()
    codes, scales, value = S.quantise4(x[0])
    assert (kv.k_scale[0, 0, :, 0].view(torch.int16).cpu().numpy().view(np.uint16) == S.bf16_bits(scales)).all()
    assert (kv.k_pool[0, 0, :, 0].cpu().numpy() == codes).all()
    assert np.array_equal(out[0, 0].cpu().numpy(), value.astype(np.float32), equal_nan=True)


def test_int4_write_strides_and_left_out_tokens():
    rng = np.random.default_rng(5)
    T, H, D, page = 23, 4, 64, 16
    wide, wd = _rows(rng, (T, 3 * H * D + 5), "bf16")
    k, kd = wide[:, 3: 3 + H * D].unflatten(1, (H, D)), wd[:, 3: 3 + H * D].reshape(T, H, D)
    v0, vd0 = _rows(rng, (H, T, D), "bf16")
    kv = ace.AceKvCache(H, D, page, 4, 1, "bf16", "int4")
    slots = rng.permutation(4 * page)[:T].astype(np.int64)
    slots[[2, 11]] = [-1, -(1 << 40)]
    st = torch.from_numpy(slots).cuda()
    kv.write(0, k, v0.transpose(0, 1), st)
    kv.write(0, k[:0], v0.transpose(0, 1)[:0], st[:0])
    out = torch.empty(2, 1, T, H, D, dtype=torch.bfloat16, device="cuda").fill_(7)
    kv.read(None, st, out[0], out[1])
    kv.sync()
    for xd, got in ((kd, out[0, 0]), (vd0.transpose(1, 0, 2), out[1, 0])):
        want = S.quantise4(xd)[2].copy()
        want[[2, 11]] = 0
        assert (got.double().cpu().numpy() == want).all()
    kv.write(0, k[:1], k[:1], _int([4 * page], torch.int64))
    with pytest.raises(ace.AceError) as err:
        kv.sync()
    assert err.value.status == 1


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 72), ("f32", 200)])
@pytest.mark.parametrize("page", [16, 64])
def test_int4_keep_moves_paths(dtype, D, page):
    """Codes and scales of long paths whose rows overlap the places they move to."""
    rng = np.random.default_rng(D)
    layers, H, n = 3, 2, 200
    lens = np.array([0, 5, page - 1, 130, 77], np.int32)
    paths = [list(range(0, n, 2)), list(range(n)), [3], [], sorted(rng.choice(n, 90, replace=False).tolist())]
    need = [-(-(l + n) // page) for l in lens]
    n_pages = sum(need) + 1
    order = rng.permutation(n_pages)
    table = np.full((5, max(need)), -7, np.int32)
    for b, at in enumerate(np.cumsum([0] + need[:-1])):
        table[b, : need[b]] = order[at: at + need[b]]
    kv = ace.AceKvCache(H, D, page, n_pages, layers, dtype, "int4")
    pools = [p.view(torch.uint8) for p in (kv.k_pool, kv.v_pool, kv.k_scale, kv.v_scale)]
    for p in pools:
        p.copy_(torch.from_numpy(rng.integers(0, 256, tuple(p.shape), np.uint8)))
    before = [p.cpu().numpy() for p in pools]
    path = np.full((5, n), -1, np.int32)
    for b, p in enumerate(paths):
        path[b, : len(p)] = p
    new = torch.empty(5, dtype=torch.int32, device="cuda")
    kv.keep(_int(table), _int(lens), _int(path), _int([len(p) for p in paths]), new)
    kv.sync()
    assert new.tolist() == [l + len(p) for l, p in zip(lens, paths)]
    for p, old in zip(pools, before):
        want = old.copy()
        for b, nodes in enumerate(paths):
            for i, a in enumerate(nodes):
                s, d = lens[b] + a, lens[b] + i
                want[:, table[b, d // page], :, d % page] = old[:, table[b, s // page], :, s % page]
        assert (p.cpu().numpy() == want).all()


class Step:
    """Requests with random rows in a 4-bit cache, and the rows' values in 64 bits. Rows that no call wrote are NaN."""

    def __init__(self, lens, sizes, Hq, H, D, page, dtype="bf16", seed=0, layers=1, layer=0, spare=0, k_scale=1.0, v_scale=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.sizes, self.D, self.dtype, self.page, self.layer, self.rng = list(lens), list(sizes), D, dtype, page, layer, rng
        need = [-(-(l + n) // page) for l, n in zip(lens, sizes)]
        n_pages = sum(need) + 3
        self.kv = ace.AceKvCache(H, D, page, n_pages, layers, dtype, "int4")
        for p in (self.kv.k_pool, self.kv.v_pool, self.kv.k_scale, self.kv.v_scale):
            p.view(torch.uint8).fill_(0xFF)
        order = rng.permutation(n_pages)
        self.table = np.full((len(lens), max(max(need), 1) + spare), -5, np.int32)
        self.k, self.v = [], []
        for b, at in enumerate(np.cumsum([0] + need[:-1])):
            self.table[b, : need[b]] = order[at: at + need[b]]
            L = lens[b] + sizes[b]
            k, kd = _rows(rng, (L, H, D), dtype, k_scale * np.where(np.arange(D) % 17 == 3, 4.0, 1.0))
            v, vd = _rows(rng, (L, H, D), dtype, v_scale)
            self.k.append(np.zeros((L, H, D)))
            self.v.append(np.zeros((L, H, D)))
            self.put(b, np.arange(L), k, kd, v, vd)
        self.off = np.cumsum([0] + list(sizes))
        self.T, self.n_max = int(self.off[-1]), max(max(sizes), 1)
        self.words = -(-self.n_max // 64)
        self.q, self.qd = _rows(rng, (self.T, Hq, D), dtype, 2.0)
        self.sees = [np.tril(np.ones((n, n), bool)) for n in sizes]

    def put(self, b, pos, k, kd, v, vd):
        if len(pos):
            self.kv.write(self.layer, k, v, torch.from_numpy(self.table[b, pos // self.page].astype(np.int64) * self.page + pos % self.page).cuda())
            self.k[b][pos], self.v[b][pos] = S.quantise4(kd)[2], S.quantise4(vd)[2]

    def random_masks(self, p=0.4, empty=()):
        for b, n in enumerate(self.sizes):
            self.sees[b] = self.rng.random((n, n)) < p
            for i in empty:
                if i < n:
                    self.sees[b][i] = False

    def run(self, chain=False, lse=True, stream=None, q=None, scale=None, max_nodes=None):
        out = torch.full((self.T,) + self.q.shape[1:], 7.0, dtype=DT[self.dtype], device="cuda")
        ls = torch.full(self.q.shape[:2], 7.0, device="cuda") if lse else None
        n_max = max_nodes or self.n_max
        mask = None if chain else _int(np.concatenate([R.mask_words(s, -(-n_max // 64)) for s in self.sees]).view(np.int64), torch.int64)
        args = _int(self.table), _int(self.lens), _int(self.off)
        torch.cuda.synchronize()
        self.kv.attend(self.layer, self.q if q is None else q, *args, out, mask, n_max, scale, ls, stream)
        self.kv.sync()
        return out, ls

    def check(self, out, ls, scale=None):
        """Bounds: fp32 sums of D products and of L weights (each a 2^-24 of what is summed); weights rounded to bf16, 2^-8 of
        each at most, and the output (fp32: neither)."""
        scale = self.D ** -0.5 if scale is None else scale
        out = out.double().cpu().numpy()
        bf = self.dtype == "bf16"
        for b, n in enumerate(self.sizes):
            if not n:
                continue
            q = self.qd[self.off[b]: self.off[b] + n]
            want, wl = R.tree_attention(q, self.k[b], self.v[b], self.lens[b], self.sees[b], scale)
            got = out[self.off[b]: self.off[b] + n]
            G, L = q.shape[1] // self.k[b].shape[1], self.lens[b] + n
            k = np.repeat(np.where(np.isfinite(self.k[b]), np.abs(self.k[b]), 0.0), G, 1)
            v = np.repeat(np.where(np.isfinite(self.v[b]), np.abs(self.v[b]), 0.0), G, 1)
            s_abs = np.einsum("nhd,lhd->nhl", np.abs(q), k).max(-1) * abs(scale)
            ds = (self.D + 8) * 2.0 ** -24 * s_abs + 2.0 ** -20
            tol = (2 * ds + (L + 16) * 2.0 ** -24 + (2.0 ** -8 if bf else 0)) * v.max((0, 2))[None, :]
            o_tol = tol[..., None] + EPS[self.dtype] * np.abs(want)
            fine = np.isfinite(want)
            assert np.array_equal(np.isnan(got), np.isnan(want))
            err = np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, want, 0)), 0)
            assert (err <= np.where(fine, o_tol, np.inf)).all(), (b, (err / np.where(fine, o_tol, 1)).max())
            if ls is not None:
                g = ls[self.off[b]: self.off[b] + n].double().cpu().numpy()
                none, nan = np.isneginf(wl), np.isnan(wl)
                assert (np.isneginf(g) == none).all() and (np.isnan(g) == nan).all()
                some = ~none & ~nan
                assert (np.abs(g[some] - wl[some]) <= (ds + (L + 16) * 2.0 ** -24)[some] + 2.0 ** -22 * np.abs(wl[some])).all()


TYPES = [("bf16", 128), ("bf16", 64), ("bf16", 80), ("bf16", 256), ("f32", 64), ("f32", 24)]


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("Hq,H,page", [(8, 2, 16), (4, 4, 64), (5, 1, 128), (16, 1, 32), (24, 1, 256)])
def test_int4_attention_single_tokens(dtype, D, Hq, H, page):
    """Plain decode steps: lengths around pages and tiles, none at all, a request without nodes."""
    s = Step([0, 1, 15, 127, 128, 129, 255, 700, 33, 31, 64], [1, 1, 1, 1, 1, 1, 1, 1, 0, 1, 1], Hq, H, D, page, dtype, seed=D)
    s.check(*s.run(chain=True))


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("Hq,H,sizes", [(8, 2, [1, 3, 2, 4]), (8, 2, [1, 17, 64, 5]), (6, 2, [65, 3, 130, 100]), (16, 1, [256, 31, 2, 8])])
def test_int4_attention_trees(dtype, D, Hq, H, sizes):
    """Any masks, rows that see no node (none at all where the prefix is empty too), several row blocks a head."""
    s = Step([0, 250, 97, 1025], sizes, Hq, H, D, 32, dtype, seed=D + Hq)
    s.random_masks(empty=(0, 3))
    s.check(*s.run())


@pytest.mark.parametrize("dtype,D", TYPES)
def test_int4_attention_chain_is_the_lower_triangle(dtype, D):
    for sizes in ([70, 9], [4, 2], [12, 7]):
        s = Step([40, 500], sizes, 4, 2, D, 16, dtype, seed=2)
        a, b = s.run(chain=True), s.run()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        s.check(*a)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("nodes", [3, 9, 40])
def test_int4_attention_long_and_ragged(dtype, D, nodes):
    """One request's keys spread over all SMs and joined; beside it short ones. The same call gives the same bits."""
    s = Step([20000, 3, 0, 4000], [nodes, 2, 1, nodes], 8, 2, D, 64, dtype, seed=3)
    s.random_masks(0.7)
    first, again = s.run(), s.run()
    s.check(*first)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("most", [1, 2, 5])
def test_int4_attention_many_requests(D, most):
    """More requests than a block keeps shapes of, many without nodes or without a prefix, a few long ones far apart."""
    rng = np.random.default_rng(D + most)
    lens = rng.integers(0, 40, 700)
    lens[[0, 255, 256, 257, 511, 699]] = [900, 1700, 640, 0, 2500, 300]
    sizes = rng.integers(0, most + 1, 700)
    sizes[[0, 255, 256, 511, 699]] = most
    s = Step(lens.tolist(), sizes.tolist(), 8, 2, D, 16, seed=5)
    s.random_masks(0.6)
    s.check(*s.run())


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("nodes,length", [(2, 0), (3, 63), (12, 0), (12, 90), (12, 126), (30, 126), (70, 5)])
def test_int4_attention_masked_rows_never_matter(dtype, D, nodes, length):
    """Drafted rows of NaN and infinities reach exactly the nodes that see them; unwritten rows reach none."""
    s = Step([length, 40], [nodes, 2], 8, 2, D, 16, dtype, seed=length + 1)
    s.random_masks(0.5)
    bad = [0, nodes - 1]
    s.sees[0][:, bad] = False
    s.sees[0][0, nodes - 1] = True
    k, _ = _rows(s.rng, (2, 2, D), dtype)
    v, _ = _rows(s.rng, (2, 2, D), dtype)
    k[0], v[0, :, 3], v[0, :, 4] = float("nan"), float("inf"), float("nan")
    v[1, :, 5], v[1, 1, D - 1] = float("nan"), float("-inf")
    s.put(0, length + np.array(bad), k, k.double().cpu().numpy(), v, v.double().cpu().numpy())
    out, ls = s.run()
    nan = torch.isnan(out[:nodes]).any(-1).any(-1).cpu().numpy()
    assert nan.tolist() == [i == 0 for i in range(nodes)]
    s.check(out, ls)


@pytest.mark.parametrize("dtype,D", TYPES)
def test_int4_attention_not_finite_in_the_prefix(dtype, D):
    """A NaN of K in the prefix makes the rows of its head NaN, one of V its dimensions, even where its weight is nothing."""
    s = Step([300, 300], [2, 9], 4, 2, D, 16, dtype, seed=6)
    for b in (0, 1):
        k, _ = _rows(s.rng, (2, 2, D), dtype)
        v, _ = _rows(s.rng, (2, 2, D), dtype)
        k[0, 0, 1] = float("nan")
        v[1, 1, D - 1] = float("inf")
        k[1] = -60 * torch.sign(s.q[s.off[b], 2])       # hardly any weight for the first row of kv head 1
        s.put(b, np.array([17, 150]), k, k.double().cpu().numpy(), v, v.double().cpu().numpy())
    s.check(*s.run())


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("nodes", [2, 8, 40])
def test_int4_attention_sharp_and_wide_scores(dtype, D, nodes):
    """Scores in the hundreds (the running maximum moves), all alike, and turned round."""
    s = Step([3000], [nodes], 4, 2, D, 64, dtype, seed=9)
    for scale in (3.0, 0.0, -1.0):
        s.check(*s.run(scale=scale), scale=scale)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("nodes", [1, 8, 40])
def test_int4_attention_rows_of_many_sizes(dtype, D, nodes):
    """V rows that differ by 2^40 along the keys, q rows by 2^30, K rows of 2^-20: exact codes know no unit."""
    L = 600
    s = Step([L], [nodes], 4, 1, D, 32, dtype, seed=8)
    size = 2.0 ** s.rng.integers(-20, 21, L)
    v, _ = _rows(s.rng, (L, 1, D), dtype)
    v = (v.float() * torch.from_numpy(size).float().cuda()[:, None, None]).to(DT[dtype])
    k, _ = _rows(s.rng, (L, 1, D), dtype)
    k = (k.float() * 2.0 ** -20).to(DT[dtype])
    s.put(0, np.arange(L), k, k.double().cpu().numpy(), v, v.double().cpu().numpy())
    up = torch.from_numpy(2.0 ** s.rng.integers(-10, 20, (nodes, 4, 1))).cuda()
    s.q = (s.q.double() * up).to(DT[dtype])
    s.qd = s.q.double().cpu().numpy()
    s.check(*s.run())


@pytest.mark.parametrize("size", [1e5, 1e17])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("nodes", [1, 3, 6, 15, 50])
def test_int4_attention_equal_scores_of_any_size(nodes, sign, size):
    """Rows of one key score alike however large the score, so the output is the mean of V: codes of 1 to 7 and their sums are
    exact, a weight's rounding is at most 2^-8 of it, the output's too."""
    rng = np.random.default_rng(nodes)
    H, G, D, page, length = 1, 4, 128, 16, 333
    total = length + nodes
    v = torch.from_numpy(rng.integers(1, 8, (total, H, D)).astype(np.float32)).bfloat16()
    v[..., ::32] = 7
    kv = ace.AceKvCache(H, D, page, 24, 1, "bf16", "int4")
    kv.write(0, torch.full((total, H, D), size, dtype=torch.bfloat16, device="cuda"), v.cuda(), torch.arange(total, device="cuda"))
    q = torch.full((nodes, H * G, D), sign * size, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    kv.attend(0, q, torch.arange(24, dtype=torch.int32, device="cuda")[None], _int([length]), _int([0, nodes]), out, None, nodes)
    kv.sync()
    sums = v.double().numpy().cumsum(0)
    want = np.stack([sums[length + i] / (length + i + 1) for i in range(nodes)])
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -7 * want).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 80)])
def test_int4_attention_strides_layers_streams_and_graphs(dtype, D):
    """q inside a wider projection at an odd offset, another layer of the cache, another stream, replays with changed inputs."""
    s = Step([130, 45, 700], [5, 1, 3], 8, 2, D, 16, dtype, seed=11, layers=3, layer=2)
    s.random_masks(0.6)
    wide = torch.empty(s.T, 8 * D + 3, dtype=DT[dtype], device="cuda")
    q = wide[:, 3:].unflatten(1, (8, D))
    q.copy_(s.q)
    want = s.run()
    s.check(*want)
    side = torch.cuda.Stream()
    got = s.run(q=q, stream=side)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    out, ls = torch.empty_like(s.q), torch.empty(s.T, 8, device="cuda")
    mask = _int(np.concatenate([R.mask_words(x, 1) for x in s.sees]).view(np.int64), torch.int64)
    args = _int(s.table), _int(s.lens), _int(s.off)
    qg = s.q.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.kv.attend(2, qg, *args, out, mask, s.n_max, lse=ls)
    for scale in (1.0, -0.5):
        qg.copy_(s.q * scale)
        g.replay()
        torch.cuda.synchronize()
        s.q, s.qd = qg.clone(), qg.double().cpu().numpy()
        s.check(out, ls)
    s.kv.sync()


def test_int4_pages_that_do_not_exist_are_reported_and_read_as_zeros():
    """As in the other formats, by each of the kernels."""
    for dtype, D, nodes in (("bf16", 128, 1), ("bf16", 64, 3), ("bf16", 128, 30), ("f32", 64, 2)):
        s = Step([100, 60], [nodes, 1], 4, 2, D, 16, dtype, seed=21)
        s.table[0, 2] = 1 << 20
        s.k[0][32:48], s.v[0][32:48] = 0, 0
        out = torch.empty_like(s.q)
        s.kv.attend(0, s.q, _int(s.table), _int(s.lens), _int(s.off), out, None, s.n_max)
        with pytest.raises(ace.AceError) as err:
            s.kv.sync()
        assert err.value.status == 1
        s.check(out, None)


def test_int4_offsets_past_2_32():
    """A cache of more than 2^32 bytes a pool: rows behind them are written, read and attended to."""
    H, D, page, n_pages = 8, 128, 256, 33000
    kv = ace.AceKvCache(H, D, page, n_pages, 1, "bf16", "int4")
    assert kv.k_pool.numel() > 1 << 32
    rng = np.random.default_rng(1)
    k, kd = _rows(rng, (300, H, D), "bf16")
    v, vd = _rows(rng, (300, H, D), "bf16")
    table = np.array([[n_pages - 1, n_pages - 3]], np.int32)
    pos = np.arange(300)
    kv.write(0, k, v, torch.from_numpy(table[0, pos // page].astype(np.int64) * page + pos % page).cuda())
    for n in (1, 5, 40):
        q, qd = _rows(rng, (n, H, D), "bf16")
        out = torch.empty_like(q)
        kv.attend(0, q, _int(table), _int([300 - n]), _int([0, n]), out, None, n)
        kv.sync()
        want, _ = R.tree_attention(qd, S.quantise4(kd)[2], S.quantise4(vd)[2], 300 - n, np.tril(np.ones((n, n), bool)), D ** -0.5)
        assert np.abs(out.double().cpu().numpy() - want).max() <= 2.0 ** -7 * np.abs(vd).max()
