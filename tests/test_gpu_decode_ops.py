"""The speculative decode step's operators on the GPU against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as R
from paper_2609_05228_gb300 import ace

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows(rng, shape, dtype, scale=1.0):
    """Random rows of the storage type, on the device, and the same in fp64."""
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(DT[dtype])
    return t.cuda(), t.double().numpy()


# ----------------------------------------------------------------------- the cache


@pytest.mark.parametrize("fmt", ["fp8", "plain"])
@pytest.mark.parametrize("dtype,D", [("bf16", 8), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 40), ("f32", 80), ("f32", 200)])
@pytest.mark.parametrize("T,H,page", [(1, 1, 16), (37, 3, 32), (300, 2, 128)])
def test_write_and_read_are_exact(fmt, dtype, D, T, H, page):
    """Codes, scale bytes and read-back values are the definition's, bit for bit; a layer of several; unnamed rows stay."""
    rng = np.random.default_rng(T + D)
    layers, n_pages = 3, -(-T // page) + 2
    kv = ace.AceKvCache(H, D, page, n_pages, layers, dtype, fmt)
    for pool in (kv.k_pool, kv.v_pool):
        pool.view(torch.uint8).fill_(0x15)
    spread = np.exp(rng.uniform(-30, 30, (T, H, 1)))
    k, kd = _rows(rng, (T, H, D), dtype, spread)
    v, vd = _rows(rng, (T, H, D), dtype)
    v[0], vd[0] = 0, 0                              # a row of zeros
    slots = rng.permutation(n_pages * page)[:T]
    st = torch.from_numpy(slots).cuda()
    kv.write(1, k, v, st)
    k_out, v_out = torch.empty_like(k), torch.empty_like(v)
    kv.read(1, st, k_out, v_out)
    kv.sync()
    for x, xd, out, pool, scale in ((k, kd, k_out, kv.k_pool, kv.k_scale), (v, vd, v_out, kv.v_pool, kv.v_scale)):
        got = pool.view(torch.uint8 if fmt == "fp8" else x.dtype)[1].cpu()[slots // page, :, slots % page]
        if fmt == "fp8":
            code, byte, value = R.quantise_rows(xd)
            assert (scale[1].cpu().numpy()[slots // page, :, slots % page] == byte).all()
            # the sign of a zero is the input's
            assert (got.numpy() == code).all()
            want = torch.from_numpy(value).to(DT[dtype])
        else:
            assert (got.view(torch.uint8) == x.cpu().view(torch.uint8)).all()
            want = x.cpu()
        assert torch.equal(out.cpu(), want)
        rest = pool.view(torch.uint8).reshape(layers, n_pages, H, page, -1).movedim(2, 3).reshape(layers, n_pages * page, H, -1).cpu()
        keep = np.ones((layers, n_pages * page), bool)
        keep[1, slots] = False
        assert (rest[torch.from_numpy(keep)] == 0x15).all()


@pytest.mark.parametrize("fmt", ["fp8", "plain"])
def test_write_strides_and_left_out_tokens(fmt):
    """Head-major rows, rows inside a wider projection at an odd element offset, negative slots, no tokens."""
    rng = np.random.default_rng(5)
    T, H, D, page = 23, 4, 64, 16
    wide, wd = _rows(rng, (T, 3 * H * D + 5), "bf16")
    k = wide[:, 3: 3 + H * D].unflatten(1, (H, D))
    kd = wd[:, 3: 3 + H * D].reshape(T, H, D)
    v0, vd0 = _rows(rng, (H, T, D), "bf16")
    v, vd = v0.transpose(0, 1), vd0.transpose(1, 0, 2)
    kv = ace.AceKvCache(H, D, page, 4, 1, "bf16", fmt)
    slots = rng.permutation(4 * page)[:T].astype(np.int64)
    slots[[2, 11]] = [-1, -(1 << 40)]
    st = torch.from_numpy(slots).cuda()
    kv.write(0, k, v, st)
    kv.write(0, k[:0], v[:0], st[:0])
    out = torch.empty(2, 1, T, H, D, dtype=torch.bfloat16, device="cuda").fill_(7)
    kv.read(None, st, out[0], out[1])
    kv.sync()
    for xd, got in ((kd, out[0, 0]), (vd, out[1, 0])):
        want = (R.quantise_rows(xd)[2] if fmt == "fp8" else xd).copy()
        want[[2, 11]] = 0
        assert (got.double().cpu().numpy() == want).all()


def test_write_of_values_that_are_not_finite():
    """NaN and infinities become e4m3's NaN and leave the scale to the finite ones; the extremes of fp32 are in range."""
    D = 32
    x = np.zeros((1, 6, D), np.float32)
    x[0, 0, :4] = [np.nan, np.inf, -np.inf, 3.0]
    x[0, 1] = np.finfo(np.float32).max
    x[0, 2, 5] = 1e-45
    x[0, 3, :3] = [448.0, 448.0001, -2.0]
    x[0, 4] = np.nan
    x[0, 5, :2] = [2.0 ** -126 * 448, -(2.0 ** -130)]
    kv = ace.AceKvCache(6, D, 16, 1, 1, "f32", "fp8")
    t = torch.from_numpy(x).cuda()
    slot = torch.zeros(1, dtype=torch.int64, device="cuda")
    kv.write(0, t, t, slot)
    out = torch.empty(2, 1, 6, D, device="cuda")
    kv.read(0, slot, out[0], out[1])
    kv.sync()
    code, byte, value = R.quantise_rows(x[0])
    assert (kv.k_scale[0, 0, :, 0].cpu().numpy() == byte).all()
    assert (kv.k_pool.view(torch.uint8)[0, 0, :, 0].cpu().numpy() == code).all()
    # a row's largest float32 rounds up to the code of 2^128, which no float32 is
    with np.errstate(over="ignore"):
        assert np.array_equal(out[0, 0].cpu().numpy(), value.astype(np.float32), equal_nan=True)


def test_slots_outside_the_cache_are_left_out_and_reported():
    kv = ace.AceKvCache(2, 64, 16, 2, 2, "bf16", "fp8")
    x = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([0, 32, 31, 1 << 40], device="cuda")
    kv.write(0, x, x, slots)
    with pytest.raises(ace.AceError) as err:
        kv.sync()
    assert err.value.status == 1
    kv.sync()                                       # reported once
    assert kv.k_pool.view(torch.uint8)[1].count_nonzero() == 0
    out = torch.full((2, 4, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    kv.read(0, slots, out[0], out[1])
    with pytest.raises(ace.AceError):
        kv.sync()
    assert (out[:, [0, 2]] == 1).all() and (out[:, [1, 3]] == 0).all()


@pytest.mark.parametrize("fmt,dtype,D", [("fp8", "bf16", 128), ("plain", "bf16", 64), ("plain", "f32", 72), ("fp8", "f32", 40)])
@pytest.mark.parametrize("page", [16, 64])
def test_keep_moves_paths(fmt, dtype, D, page):
    """Long paths whose rows overlap the places they move to, the whole tree, one node, none."""
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
    kv = ace.AceKvCache(H, D, page, n_pages, layers, dtype, fmt)
    g = torch.Generator(device="cuda").manual_seed(3)
    pools = [kv.k_pool, kv.v_pool] + ([kv.k_scale, kv.v_scale] if fmt == "fp8" else [])
    for p in pools:
        p.view(torch.uint8).copy_(torch.randint(0, 256, p.view(torch.uint8).shape, generator=g, device="cuda", dtype=torch.uint8))
    before = [p.view(torch.uint8).cpu().numpy() for p in pools]
    path = np.full((5, n), -1, np.int32)
    for b, p in enumerate(paths):
        path[b, : len(p)] = p
    keep = np.array([len(p) for p in paths], np.int32)
    new = torch.empty(5, dtype=torch.int32, device="cuda")
    cu = [torch.from_numpy(a).cuda() for a in (table, lens, path, keep)]
    kv.keep(*cu, new)
    kv.sync()
    assert (new.cpu().numpy() == lens + keep).all()
    for p, old in zip(pools, before):
        want = old.copy()
        for b, nodes in enumerate(paths):
            for i, a in enumerate(nodes):
                s, d = lens[b] + a, lens[b] + i
                want[:, table[b, d // page], :, d % page] = old[:, table[b, s // page], :, s % page]
        assert (p.view(torch.uint8).cpu().numpy() == want).all()


def test_keep_leaves_out_paths_that_are_wrong():
    kv = ace.AceKvCache(1, 64, 16, 4, 1, "bf16", "plain")
    kv.k_pool.copy_(torch.arange(64, device="cuda").view(1, 4, 1, 16, 1).expand_as(kv.k_pool))
    before = kv.k_pool.clone()
    table = torch.tensor([[0, 1], [2, 9], [3, 1]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([4, 14, 30], dtype=torch.int32, device="cuda")
    path = torch.tensor([[2, 1, -1], [0, 3, -1], [0, 5, -1]], dtype=torch.int32, device="cuda")
    n_keep = torch.tensor([2, 2, 2], dtype=torch.int32, device="cuda")      # not increasing; a page of no pool; past the table
    new = torch.zeros(3, dtype=torch.int32, device="cuda")
    kv.keep(table, lens, path, n_keep, new)
    with pytest.raises(ace.AceError):
        kv.sync()
    assert torch.equal(kv.k_pool, before) and torch.equal(new, lens)


# ----------------------------------------------------------------------- masks


@pytest.mark.parametrize("n_max", [1, 7, 64, 65, 200, 256])
def test_tree_mask(n_max):
    rng = np.random.default_rng(n_max)
    sizes = [n_max, 0, 1, max(1, n_max // 2)]
    parents = []
    for n in sizes:
        parents.append(np.array([-1] + [rng.integers(-1, i) for i in range(1, n)], np.int32)[:n])
    if n_max > 3:
        parents[0][3] = 3                           # not below its node: none
        parents[0][2] = 1 << 30
    off = torch.tensor(np.cumsum([0] + sizes), dtype=torch.int32, device="cuda")
    words = -(-n_max // 64)
    mask = torch.full((sum(sizes), words), -1, dtype=torch.int64, device="cuda")
    depth = torch.full((sum(sizes),), -1, dtype=torch.int32, device="cuda")
    ace.ace_tree_mask(torch.from_numpy(np.concatenate(parents)).cuda(), off, len(sizes), n_max, mask, depth)
    sees = [R.ancestors(p) for p in parents]
    want = np.concatenate([R.mask_words(s, words) for s in sees])
    assert (mask.cpu().numpy().view(np.uint64) == want).all()
    assert (depth.cpu().numpy() == np.concatenate([s.sum(1) - 1 for s in sees])).all()


# ----------------------------------------------------------------------- attention


class Step:
    """A batch of requests with random cached rows: device tensors, and the rows as values in 64 bits."""

    def __init__(self, lens, sizes, Hq, H, D, page, fmt, dtype, seed=0, layers=1, layer=0, extra_pages=3, spare=0):
        rng = np.random.default_rng(seed)
        self.lens, self.sizes, self.D = list(lens), list(sizes), D
        self.rng, self.fmt, self.dtype, self.page, self.layer = rng, fmt, dtype, page, layer
        B = len(lens)
        need = [-(-(l + n) // page) for l, n in zip(lens, sizes)]
        n_pages = sum(need) + extra_pages
        self.kv = ace.AceKvCache(H, D, page, n_pages, layers, dtype, fmt)
        # what no call wrote is NaN
        for p in (self.kv.k_pool, self.kv.v_pool):
            p.view(torch.uint8).fill_(0xFF)
        order = rng.permutation(n_pages)
        self.table = np.full((B, max(max(need), 1) + spare), -5, np.int32)
        self.k, self.v = [], []
        for b, at in enumerate(np.cumsum([0] + need[:-1])):
            self.table[b, : need[b]] = order[at: at + need[b]]
            L = lens[b] + sizes[b]
            k, kd = _rows(rng, (L, H, D), dtype, np.where(np.arange(D) % 17 == 3, 4.0, 1.0))
            v, vd = _rows(rng, (L, H, D), dtype)
            pos = np.arange(L)
            slots = torch.from_numpy(self.table[b, pos // page].astype(np.int64) * page + pos % page).cuda()
            self.kv.write(layer, k, v, slots)
            self.k.append(R.quantise_rows(kd)[2] if fmt == "fp8" and L else kd)
            self.v.append(R.quantise_rows(vd)[2] if fmt == "fp8" and L else vd)
        self.off = np.cumsum([0] + list(sizes))
        self.T = int(self.off[-1])
        self.n_max = max(max(sizes), 1)
        self.words = -(-self.n_max // 64)
        self.q, self.qd = _rows(rng, (self.T, Hq, D), dtype, 2.0)
        self.sees = [np.tril(np.ones((n, n), bool)) for n in sizes]

    def random_masks(self, p=0.4, empty=()):
        for b, n in enumerate(self.sizes):
            self.sees[b] = self.rng.random((n, n)) < p
            for i in empty:
                if i < n:
                    self.sees[b][i] = False

    def mask(self):
        return torch.from_numpy(np.concatenate([R.mask_words(s, self.words) for s in self.sees]).view(np.int64)).cuda()

    def run(self, chain=False, lse=True, stream=None, q=None, scale=None, T=None):
        out = torch.full((self.T,) + self.q.shape[1:], 7.0, dtype=DT[self.dtype], device="cuda")
        ls = torch.full(self.q.shape[:2], 7.0, device="cuda") if lse else None
        args = [torch.from_numpy(np.asarray(a, np.int32)).cuda() for a in (self.table, self.lens, self.off)]
        torch.cuda.synchronize()
        self.kv.attend(self.layer, self.q if q is None else q, *args, out, None if chain else self.mask(), self.n_max, scale, ls, stream)
        self.kv.sync()
        return out, ls

    def check(self, out, ls, scale=None):
        """Bounds: fp32 sums of D products and of L weights (each a 2^-24 of what is summed), the weights' rounding
        (2^-9 bf16 cache, 2^-12 fp8 cache; none in fp32), the output's."""
        scale = self.D ** -0.5 if scale is None else scale
        out = out.double().cpu().numpy()
        for b, n in enumerate(self.sizes):
            if not n:
                continue
            q = self.qd[self.off[b]: self.off[b] + n]
            want, wl = R.tree_attention(q, self.k[b], self.v[b], self.lens[b], self.sees[b], scale)
            got = out[self.off[b]: self.off[b] + n]
            L = self.lens[b] + n
            G = q.shape[1] // self.k[b].shape[1]
            k = np.repeat(np.where(np.isfinite(self.k[b]), np.abs(self.k[b]), 0.0), G, 1)
            v = np.repeat(np.where(np.isfinite(self.v[b]), np.abs(self.v[b]), 0.0), G, 1)
            s_abs = np.einsum("nhd,lhd->nhl", np.abs(q), k).max(-1) * abs(scale)       # sum of |products| of a score
            ds = (self.D + 8) * 2.0 ** -24 * s_abs + 2.0 ** -20                      # a score's error, exp2's included
            v_max = v.max((0, 2))[None, :]
            w = 0.0 if self.dtype == "f32" else 2.0 ** -9 if self.fmt == "plain" else 2.0 ** -12
            tol = (2 * ds + (L + 16) * 2.0 ** -24 + w) * v_max
            o_tol = tol[..., None] + (0 if self.dtype == "f32" else 2.0 ** -8) * np.abs(want)
            assert np.isfinite(got).all() == np.isfinite(want).all()
            fine = np.isfinite(want)
            assert np.array_equal(np.isnan(got), np.isnan(want))
            err = np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, want, 0)), 0)
            assert (err <= np.where(fine, o_tol, np.inf)).all(), (b, (err / np.where(fine, o_tol, 1)).max())
            if ls is not None:
                g = ls[self.off[b]: self.off[b] + n].double().cpu().numpy()
                none = np.isneginf(wl)
                assert (np.isneginf(g) == none).all()
                assert (np.abs(np.where(none, 0, g) - np.where(none, 0, wl)) <= ds + (L + 16) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(none, 0, wl))).all()


TYPES = [("fp8", "bf16", 128), ("plain", "bf16", 128), ("fp8", "bf16", 64), ("plain", "bf16", 64), ("plain", "bf16", 256),
         ("fp8", "bf16", 80), ("plain", "f32", 64), ("fp8", "f32", 128), ("plain", "f32", 24)]


@pytest.mark.parametrize("fmt,dtype,D", TYPES)
@pytest.mark.parametrize("Hq,H,page", [(8, 2, 16), (4, 4, 64), (5, 1, 128), (16, 1, 32)])
def test_attention_single_tokens(fmt, dtype, D, Hq, H, page):
    """Plain decode steps: lengths around pages and tiles, none at all, a request without nodes."""
    s = Step([0, 1, 15, 127, 128, 129, 255, 700, 33], [1, 1, 1, 1, 1, 1, 1, 1, 0], Hq, H, D, page, fmt, dtype, seed=D)
    s.check(*s.run(chain=True))


@pytest.mark.parametrize("fmt,dtype,D", TYPES)
@pytest.mark.parametrize("Hq,H,sizes", [(8, 2, [1, 17, 64, 5]), (6, 2, [65, 3, 130, 100]), (16, 1, [256, 31, 2, 8])])
def test_attention_trees(fmt, dtype, D, Hq, H, sizes):
    """Any masks, rows that see no node (none at all where the prefix is empty too), several row blocks a head."""
    s = Step([0, 250, 97, 1025], sizes, Hq, H, D, 32, fmt, dtype, seed=D + Hq)
    s.random_masks(empty=(0, 3))
    s.check(*s.run())


@pytest.mark.parametrize("fmt,dtype,D", TYPES)
def test_attention_chain_is_the_lower_triangle(fmt, dtype, D):
    s = Step([40, 500], [70, 9], 4, 2, D, 16, fmt, dtype, seed=2)
    a = s.run(chain=True)
    b = s.run(chain=False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    s.check(*a)


@pytest.mark.parametrize("fmt,dtype,D", TYPES)
def test_attention_long_and_ragged(fmt, dtype, D):
    """One request's keys spread over all SMs and joined; beside it short ones."""
    s = Step([20000, 3, 0, 4000], [3, 2, 1, 9], 8, 2, D, 64, fmt, dtype, seed=3)
    s.random_masks(0.7)
    first = s.run()
    s.check(*first)
    again = s.run()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("fmt,dtype,D", TYPES)
@pytest.mark.parametrize("length", [0, 90, 126])
def test_attention_masked_rows_never_matter(fmt, dtype, D, length):
    """Drafted rows of NaN and infinities reach exactly the nodes that see them; unwritten rows reach none."""
    s = Step([length, 40], [12, 6], 8, 2, D, 16, fmt, dtype, seed=length + 1)
    s.random_masks(0.5)
    bad = [2, 7]
    s.sees[0][:, bad] = False
    s.sees[0][[4, 9], 7] = True                     # two nodes see one of the poisoned rows
    pos = length + np.array(bad)
    slots = torch.from_numpy(s.table[0, pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
    k, kd = _rows(s.rng, (2, 2, D), dtype)
    v, vd = _rows(s.rng, (2, 2, D), dtype)
    k[0], v[0, :, 3], v[0, :, 4] = float("nan"), float("inf"), float("nan")
    v[1, :, 5], v[1, :, D - 1] = float("nan"), float("nan")
    k[1, :, 0] = 0.5
    s.kv.write(0, k, v, slots)
    kd, vd = k.double().cpu().numpy(), v.double().cpu().numpy()
    s.k[0][pos] = R.quantise_rows(kd)[2] if fmt == "fp8" else kd
    s.v[0][pos] = R.quantise_rows(vd)[2] if fmt == "fp8" else vd
    out, ls = s.run()
    nan = torch.isnan(out[:12]).any(-1).any(-1).cpu().numpy()
    assert nan.tolist() == [i in (4, 9) for i in range(12)]
    s.check(out, ls)


@pytest.mark.parametrize("fmt,dtype,D", [("plain", "bf16", 128), ("fp8", "bf16", 128), ("plain", "f32", 64)])
def test_attention_sharp_and_wide_scores(fmt, dtype, D):
    """Scores in the hundreds that grow along the keys (the running maximum moves in every tile), and one key that
    takes nearly all beside thousands that share the rest."""
    s = Step([3000], [2], 4, 2, D, 64, fmt, dtype, seed=9)
    s.check(*s.run(scale=3.0), scale=3.0)
    s.check(*s.run(scale=0.0), scale=0.0)
    s.check(*s.run(scale=-1.0), scale=-1.0)


@pytest.mark.parametrize("size", [1e5, 1e17])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("fmt", ["fp8", "plain"])
@pytest.mark.parametrize("nodes", [1, 3, 6, 15, 30, 50])
def test_attention_equal_scores_of_any_size(fmt, nodes, sign, size):
    """Rows of one key score alike however large the score, so the output is the mean of V: values of an eighth from 1 to 2
    have exact codes and sums, and a weight's rounding is at most 2^-8 of it, as the output's."""
    rng = np.random.default_rng(nodes)
    H, G, D, page, length = 1, 4, 128, 16, 333
    total = length + nodes
    v = torch.from_numpy(1 + rng.integers(0, 8, (total, H, D)) / 8.0).bfloat16()
    kv = ace.AceKvCache(H, D, page, 24, 1, "bf16", fmt)
    kv.write(0, torch.full((total, H, D), size, dtype=torch.bfloat16, device="cuda"), v.cuda(), torch.arange(total, device="cuda"))
    q = torch.full((nodes, H * G, D), sign * size, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    kv.attend(0, q, torch.arange(24, dtype=torch.int32, device="cuda")[None], torch.tensor([length], dtype=torch.int32, device="cuda"),
              torch.tensor([0, nodes], dtype=torch.int32, device="cuda"), out, None, nodes)
    kv.sync()
    sums = v.double().numpy().cumsum(0)
    want = np.stack([sums[length + i] / (length + i + 1) for i in range(nodes)])
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -7 * want).all()


def test_attention_sink_beside_many_small_weights():
    """A first key with weight e^12 of the others': 30000 weights of 6e-6 still sum to their share of the output."""
    L, D = 30000, 128
    s = Step([L], [1], 2, 1, D, 64, "fp8", "bf16", seed=4)
    k = torch.zeros(L, 1, D, dtype=torch.bfloat16, device="cuda")
    k[0, 0, 0] = 12.0
    v = torch.ones(L, 1, D, dtype=torch.bfloat16, device="cuda")
    v[0] = -1.0
    pos = np.arange(L)
    s.kv.write(0, k, v, torch.from_numpy(s.table[0, pos // 64].astype(np.int64) * 64 + pos % 64).cuda())
    s.k[0][:L], s.v[0][:L] = R.quantise_rows(k.double().cpu().numpy())[2], R.quantise_rows(v.double().cpu().numpy())[2]
    s.q.zero_()
    s.q[..., 0] = 1.0
    s.qd = s.q.double().cpu().numpy()
    s.check(*s.run(scale=1.0), scale=1.0)


@pytest.mark.parametrize("fmt", ["fp8", "plain"])
def test_attention_values_of_many_sizes(fmt):
    """Rows of V whose scales differ by 2^40 along the keys, rows of q that differ by 2^30."""
    D, L = 64, 600
    s = Step([L], [4], 4, 1, D, 32, fmt, "bf16", seed=8)
    size = 2.0 ** s.rng.integers(-20, 21, L)
    v, _ = _rows(s.rng, (L, 1, D), "bf16")
    v = (v.float() * torch.from_numpy(size).float().cuda()[:, None, None]).bfloat16()
    k, kd = _rows(s.rng, (L, 1, D), "bf16")
    pos = np.arange(L)
    s.kv.write(0, k, v, torch.from_numpy(s.table[0, pos // 32].astype(np.int64) * 32 + pos % 32).cuda())
    vd = v.double().cpu().numpy()
    s.k[0][:L], s.v[0][:L] = (R.quantise_rows(kd)[2], R.quantise_rows(vd)[2]) if fmt == "fp8" else (kd, vd)
    s.q.mul_((2.0 ** torch.tensor([-30.0, -10.0, 0.0, 1.0], device="cuda"))[:, None, None])
    s.qd = s.q.double().cpu().numpy()
    s.check(*s.run())


@pytest.mark.parametrize("fmt,dtype,D", [("fp8", "bf16", 128), ("plain", "bf16", 64), ("plain", "f32", 40)])
def test_attention_strided_queries_layers_and_spare_pages(fmt, dtype, D):
    """q inside a wider projection, head-major and at odd offsets; the last of three layers; a table wider than used."""
    s = Step([33, 200], [5, 20], 8, 2, D, 16, fmt, dtype, seed=6, layers=3, layer=2, spare=4)
    want = s.run(chain=True)
    s.check(*want)
    wide = torch.zeros(s.T, 8 * D + 11, dtype=DT[dtype], device="cuda")
    wide[:, 3: 3 + 8 * D] = s.q.reshape(s.T, -1)
    heads = s.q.transpose(0, 1).contiguous().transpose(0, 1)
    for q in (wide[:, 3: 3 + 8 * D].unflatten(1, (8, D)), heads):
        got = s.run(chain=True, q=q)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    none = s.run(chain=True, lse=False)
    assert torch.equal(none[0], want[0])


def test_attention_past_32_bit_offsets():
    """Rows of a pool whose byte and element offsets pass 2^32."""
    H, D, page = 8, 128, 64
    n_pages = (1 << 32) // (H * page * D) + 40
    kv = ace.AceKvCache(H, D, page, n_pages, 1, "bf16", "plain")
    rng = np.random.default_rng(0)
    L = 300
    table = torch.tensor([[n_pages - 1 - i for i in range(5)]], dtype=torch.int32, device="cuda")
    k, kd = _rows(rng, (L, H, D), "bf16")
    v, vd = _rows(rng, (L, H, D), "bf16")
    pos = torch.arange(L, device="cuda")
    kv.write(0, k, v, table[0, pos // page].long() * page + pos % page)
    q, qd = _rows(rng, (1, H, D), "bf16")
    out = torch.empty_like(q)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    kv.attend(0, q, table, one * (L - 1), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), out)
    kv.sync()
    want, _ = R.tree_attention(qd, kd, vd, L - 1, np.ones((1, 1), bool), D ** -0.5)
    assert np.abs(out.double().cpu().numpy() - want).max() < 2.0 ** -8 * np.abs(vd).max()


def test_attention_reports_bad_tables_and_lengths():
    s = Step([100, 50], [2, 2], 4, 2, 64, 16, "plain", "bf16", seed=1)
    good, _ = s.run(chain=True)
    for name, b, i, value in (("table", 1, 1, 1 << 20), ("table", 1, 2, -1), ("lens", 1, None, -4), ("lens", 1, None, 1 << 30)):
        old = s.table.copy(), list(s.lens)
        if name == "table":
            s.table[b, i] = value
        else:
            s.lens[b] = value
        with pytest.raises(ace.AceError) as err:
            s.run(chain=True)
        assert err.value.status == 1
        s.table, s.lens = old[0], old[1]
    again, _ = s.run(chain=True)
    assert torch.equal(good, again)


@pytest.mark.parametrize("fmt,dtype,D", [("fp8", "bf16", 128), ("plain", "f32", 40)])
def test_attention_on_other_streams_and_in_graphs(fmt, dtype, D):
    s = Step([1000, 20], [6, 3], 8, 2, D, 64, fmt, dtype, seed=12)
    want, _ = s.run(chain=True)
    side = torch.cuda.Stream()
    got, _ = s.run(chain=True, stream=side)
    assert torch.equal(got, want)
    args = [torch.from_numpy(np.asarray(a, np.int32)).cuda() for a in (s.table, s.lens, s.off)]
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        s.kv.attend(0, s.q, *args, out, None, s.n_max, stream=side)
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    args[1][0] = 400                                # other lengths, same graph
    s.lens[0] = 400
    g.replay()
    torch.cuda.synchronize()
    fresh, _ = s.run(chain=True)
    assert torch.equal(out, fresh)


# ----------------------------------------------------------------------- verification


def _trees(rng, sizes, kids=3):
    parents = []
    for n in sizes:
        p = [-1]
        for i in range(1, n):
            ok = [j for j in range(i) if p.count(j) < kids]
            p.append(int(ok[min(len(ok) - 1, int(rng.exponential(2.0)))]))
        parents.append(p[:n])
    return parents


def _verify_case(rng, sizes, V, dtype, draft, kids=3, temps=None, pad=0, sharp=3.0):
    T, B = sum(sizes), len(sizes)
    parents = _trees(rng, sizes, kids)
    z = rng.standard_normal((T, V + pad)) * sharp
    logits = torch.from_numpy(z.astype(np.float32)).to(DT[dtype]).cuda()[:, :V]
    probs = np.exp(z[:, :V] + rng.standard_normal((T, V)))
    probs = (probs / probs.sum(1, keepdims=True)).astype(np.float32)
    off = np.cumsum([0] + list(sizes))
    tokens = np.zeros(T, np.int32)
    for b, ps in enumerate(parents):
        for i in range(len(ps)):
            mine = [j for j in range(len(ps)) if ps[j] == i]
            if mine:
                x = rng.choice(V, min(V, len(mine)), replace=False, p=probs[off[b] + i] / probs[off[b] + i].sum(dtype=np.float64)) \
                    if draft else np.argsort(-probs[off[b] + i])[: len(mine)]
                tokens[off[b] + np.array(mine[: len(x)])] = x
    u = rng.random(T).astype(np.float32)
    noise = np.maximum(rng.exponential(size=(B, V + pad)), 1e-30).astype(np.float32)
    temps = np.array(temps if temps is not None else rng.choice([0.0, 0.7, 1.0, 1.3], B), np.float32)
    return dict(parents=parents, logits=logits, probs=probs, tokens=tokens, u=u, noise=noise, temps=temps, off=off, sizes=sizes,
                draft=draft)


def _run_verify(c, n_max, stream=None):
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()     # noqa: E731
    B, V = len(c["sizes"]), c["logits"].shape[1]
    path = torch.full((B, n_max), 77, dtype=torch.int32, device="cuda")
    keep = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    nxt = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    flat = np.array([p for ps in c["parents"] for p in ps], np.int32)
    args = (c["logits"], cu(c["tokens"]), cu(flat), cu(c["off"].astype(np.int32)), n_max, cu(c["u"]), cu(c["noise"])[:, :V],
            path, keep, nxt, cu(c["probs"]) if c["draft"] else None, cu(c["temps"]))
    torch.cuda.synchronize()
    ace.ace_verify_tree(*args, stream=stream)
    torch.cuda.synchronize()
    return path.cpu().numpy(), keep.cpu().numpy(), nxt.cpu().numpy()


def _check_verify(c, got, n_max):
    path, keep, nxt = got
    z, V = c["logits"].double().cpu().numpy(), c["logits"].shape[1]
    for b, n in enumerate(c["sizes"]):
        o = c["off"][b]
        want, token = R.verify(z[o: o + n], c["tokens"][o: o + n], c["parents"][b], c["probs"][o: o + n] if c["draft"] else None,
                               float(c["temps"][b]), c["u"][o: o + n], c["noise"][b, :V].astype(np.float64))
        assert keep[b] == len(want) and path[b, : len(want)].tolist() == want and (path[b, len(want):] == -1).all()
        assert nxt[b] == token, (b, nxt[b], token)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("sizes,V,pad", [([8], 32000, 0), ([1, 5, 0, 17, 30], 1003, 5), ([6] * 40, 2048, 0), ([3] * 170, 257, 1),
                                         ([256, 2], 600, 0), ([9, 4, 4], 1, 0), ([4, 7], 5, 3)])
def test_verify(dtype, draft, sizes, V, pad):
    rng = np.random.default_rng(V + len(sizes))
    c = _verify_case(rng, sizes, V, dtype, draft, pad=pad)
    n_max = max(sizes)
    _check_verify(c, _run_verify(c, n_max), n_max)


@pytest.mark.parametrize("draft", [True, False])
def test_verify_many_children(draft):
    """Up to 40 children of a node, most of them rejected."""
    rng = np.random.default_rng(4)
    c = _verify_case(rng, [120, 60, 90], 300, "f32", draft, kids=40, temps=[1.0, 0.5, 2.0], sharp=0.5)
    c["u"][:] = np.maximum(c["u"], 0.5)
    _check_verify(c, _run_verify(c, 128), 128)


def test_verify_filtered_and_broken_rows():
    """-inf filters tokens (all but one, all but the drafted ones); NaN, +inf and rows of -inf end a walk with -1;
    drafted tokens outside the vocabulary; rows where nothing is left after a rejection."""
    rng = np.random.default_rng(6)
    sizes = [4] * 8
    c = _verify_case(rng, sizes, 500, "f32", True, temps=[1.0, 0.0, 1.0, 0.0, 0.8, 1.0, 1.0, 1.0])
    z = c["logits"]
    z[0] = float("-inf")
    z[0, 77] = 2.0
    z[4, 9] = float("nan")
    z[8] = float("-inf")
    z[12, 3] = float("inf")
    z[16, 100:] = float("-inf")
    c["tokens"][21:24] = [500, -3, 1 << 30]
    c["probs"][24] = 0.0                            # nothing is subtracted: r(x) > 0 is accepted
    # the target's row is the draft's and the child is rejected by u * q > r alone (u above one): the residual is empty
    z[28] = torch.log(torch.from_numpy(c["probs"][28])).cuda()
    c["u"][28:32] = 3.0
    _check_verify(c, _run_verify(c, 4), 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("V", [20000, 20003])
def test_verify_few_requests_with_small_trees(dtype, draft, V):
    """Trees on both sides of a node a CTA; a NaN in a row that no walk visits is nothing to the others."""
    rng = np.random.default_rng(V)
    sizes = [2, 8, 1, 0, 5, 9, 7, 8]
    c = _verify_case(rng, sizes, V, dtype, draft, temps=[1.0, 0.8, 1.0, 1.0, 0.0, 1.2, 0.0, 1.0])
    c["parents"][7] = [-1, 0, 1, 2, 3, 4, 0, 0]
    o = c["off"][7]
    c["tokens"][o + 1] = -1                         # never accepted, so nodes 2 to 5 are not visited
    c["logits"][o + 2, 11] = float("nan")
    c["logits"][o + 4] = float("-inf")
    _check_verify(c, _run_verify(c, 9), 9)


def test_verify_is_lossless():
    """The first token after the root follows the target's distribution whatever the draft is: 20000 walks over
    12 tokens, each frequency within five standard deviations."""
    rng = np.random.default_rng(1)
    B, V = 20000, 12
    z = rng.standard_normal(V).astype(np.float32)
    q = rng.random(V).astype(np.float32) ** 2
    q /= q.sum()
    kids = np.argsort(rng.exponential(size=(B, V)) / q, 1)[:, :3]      # three draws without replacement
    parents = [[-1, 0, 0, 0]] * B
    tokens = np.concatenate([np.zeros((B, 1), int), kids], 1).astype(np.int32).reshape(-1)
    c = dict(parents=parents, logits=torch.from_numpy(np.tile(z, (4 * B, 1))).cuda(), probs=np.tile(q, (4 * B, 1)), tokens=tokens,
             u=rng.random(4 * B).astype(np.float32), noise=rng.exponential(size=(B, V)).astype(np.float32),
             temps=np.ones(B, np.float32), off=np.arange(B + 1) * 4, sizes=[4] * B, draft=True)
    path, keep, nxt = _run_verify(c, 4)
    first = np.where(keep > 1, tokens.reshape(B, 4)[np.arange(B), np.maximum(path[:, 1], 0)], nxt)
    p = np.exp(z.astype(float))
    p /= p.sum()
    freq = np.bincount(first, minlength=V) / B
    assert (keep > 1).mean() > 0.5
    assert (np.abs(freq - p) <= 5 * np.sqrt(p * (1 - p) / B)).all()


def test_verify_repeats_and_other_streams():
    rng = np.random.default_rng(2)
    c = _verify_case(rng, [12, 9, 16], 40000, "bf16", True, temps=[1.0, 0.9, 0.8])
    a = _run_verify(c, 16)
    b = _run_verify(c, 16, stream=torch.cuda.Stream())
    assert all((x == y).all() for x, y in zip(a, b))
