"""The measured cases of what a server does around a decoder's attention: rotary positions, a key/value cache held in 4
bits and the attention that reads it, and the life of the cache's pages.

A case's "kind" says which operator one pass runs:

  rope    q and k are rotated by their positions, or gradients are rotated back
  enter   q and k are rotated, and k and v are written into the cache as it quantises them; the rows are read back
  attend  every node of every request's tree attends to the request's cached prefix and its ancestors, the cache in 4 bits
  beam    requests are forked after a step of a search over beams and reserve pages for the next tokens: pages that
          are shared and about to be written are copied
  compact the live pages move to the front of the pool

Formulas (own and plain form alike):

  Rotary positions. With R = rot, t_i = base^(-2 i / R), i = 0 .. R / 2 - 1, and L = original, the angle of dimension pair i at
  position p is p f_i:
    none      f_i = t_i
    linear    f_i = t_i / factor
    by_turns  g = clamp((L t_i / 2 pi - low) / (high - low), 0, 1), f_i = t_i (g + (1 - g) / factor)
    by_index  c(b) = R ln(L / (2 pi b)) / (2 ln base), a = max(floor(c(high)), 0), z = min(ceil(c(low)), R - 1) (a + 0.001 where
              that is a), g = 1 - clamp((i - a) / (z - a), 0, 1), f_i as by_turns
  (x, y) -> magnitude (x cos - y sin, x sin + y cos), pairs (i, i + R / 2) in layout "half" and (2 i, 2 i + 1) in
  "interleaved"; dimensions R and on stay. Gradients: the same with the angles' signs turned.

  Pools [layer, page, head, row, ..]; slot = page * page_size + row. Format "plain" keeps rows, "fp8" e4m3 codes and a byte
  E = e + 127 a row (e the smallest integer >= -126 with max |x| <= 448 2^e). "int4" takes a row in groups of 32 (the last may be
  shorter), each with a scale s in bf16: the smallest number of 4 significant bits with max |x| <= 7 s, within 2^-126 and
  1.125 * 2^125; NaN for a group that is not finite. An element's code is x / s rounded to nearest even, kept as code + 8 in 4
  bits, two a byte, the first in the lower half. k is rounded to the storage type after the rotation.

  refs[page] counts the rows of page tables that name the page. beam: row b of the new tables has the pages of row parents[b]
  for its lens tokens and -1 beyond (no parent: empty); refs lose the old rows' pages and gain the new rows'. Then each row is
  to have pages for grow[b] more tokens. Its partly filled page, where others hold it too, is replaced by a copy of its rows (the
  last row of those that hold it keeps it where all of them grow); entries of -1 are filled. Pages come from those with
  refs 0 at the start of the call, ascending, row by row. compact: with n live pages, the i-th live page at n or above moves
  to the i-th free one below n; tables and refs follow.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32


# ----------------------------------------------------------------------- cases


def _rope(name, T, heads, kv_heads, dim, rot, layout="half", scaling="none", dtype="bf16", far=4096, back=False):
    return {"name": name, "kind": "rope", "tokens": T, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot,
            "layout": layout, "scaling": scaling, "dtype": dtype, "far": far, "back": back}


def _enter(name, T, heads, kv_heads, dim, fmt="int4", rot=0, layout="half", scaling="none", page=64, far=8192):
    return {"name": name, "kind": "enter", "tokens": T, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot or dim,
            "layout": layout, "scaling": scaling, "dtype": "bf16", "format": fmt, "page": page, "far": far}


def _attend(name, B, length, nodes, heads, kv_heads, dim, dtype="bf16", page=64, shape="tree"):
    return {"name": name, "kind": "attend", "batch": B, "length": length, "nodes": nodes, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "dtype": dtype, "format": "int4", "page": page, "shape": shape}


def _beam(name, requests, beams, length, grow, layers, kv_heads, dim, fmt="int4", page=64):
    return {"name": name, "kind": "beam", "requests": requests, "beams": beams, "length": length, "grow": grow, "layers": layers,
            "kv_heads": kv_heads, "dim": dim, "dtype": "bf16", "format": fmt, "page": page}


def _compact(name, batch, length, pages, layers, kv_heads, dim, fmt="int4", page=64):
    return {"name": name, "kind": "compact", "batch": batch, "length": length, "pages": pages, "layers": layers,
            "kv_heads": kv_heads, "dim": dim, "dtype": "bf16", "format": fmt, "page": page}


def listed():
    return [
        # one user's next token: the smallest call
        _rope("rope_1", 1, 32, 4, 128, 128),
        # a batch of long prompts, half of each head rotated, frequencies scaled for a context of 8 times the trained one
        _rope("rope_16384", 16384, 64, 8, 128, 64, "interleaved", "by_turns", far=65536),
        # gradients of q and k in the fp32 used to develop a model
        _rope("rope_back_2048", 2048, 32, 8, 128, 128, "half", "by_index", "f32", far=32768, back=True),
        # a decode step of 64 users: their rows enter the cache
        _enter("enter_64", 64, 32, 4, 128),
        # prompts enter the cache
        _enter("enter_8192", 8192, 32, 8, 128, rot=64, layout="interleaved"),
        # one user's next token after a short conversation
        _attend("attend_1", 1, 2048, 1, 32, 4, 128, shape="chain"),
        # a busy server's plain decode step, ragged lengths
        _attend("attend_64", 64, 8192, 1, 32, 4, 128, shape="chain"),
        # a speculative step, 16-node trees
        _attend("attend_tree_24", 24, 4096, 16, 64, 8, 128, page=16),
        # one user with a very long context and a chain of drafted tokens: split over the long axis
        _attend("attend_long", 1, 262144, 5, 64, 8, 128, shape="chain", page=128),
        # large trees, where the products and not the cache decide
        _attend("attend_wide_8", 8, 16384, 128, 64, 8, 128),
        # a step of a beam search, 32 requests of 4 beams
        _beam("beam_32", 32, 4, 1024, 1, 16, 4, 128),
        # a pool of which a third is in use moves to its front
        _compact("compact_64", 64, 2048, 6000, 16, 4, 128),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choices(["rope", "enter", "attend", "beam", "compact"], [2, 2, 6, 2, 1])[0]
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8, 8])
    page = rng.choice([16, 32, 64, 128])
    layout, scaling = rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "by_turns", "by_index"])
    far = _log_int(rng, 16, 1 << 20)
    if kind == "rope":
        dim = rng.choice([64, 128, 128, 8 * rng.randint(2, 32)])
        c = _rope("", _log_int(rng, 1, 16384), kv_heads * group, kv_heads, dim, rng.choice([dim, dim, dim // 2 // 2 * 2]), layout, scaling,
                  rng.choice(["bf16", "bf16", "f32"]), far, rng.random() < 0.3)
        while c["tokens"] * (c["heads"] + c["kv_heads"]) * dim * (1 if c["dtype"] == "bf16" else 2) > 16384 * 72 * 128:
            c["tokens"] = int(c["tokens"] * 0.7)
    elif kind == "enter":
        dim = rng.choice([64, 128, 128, 8 * rng.randint(2, 32)])
        c = _enter("", _log_int(rng, 1, 8192), kv_heads * group, kv_heads, dim, rng.choice(["int4", "int4", "int4", "fp8", "plain"]),
                   rng.choice([dim, dim, dim // 2 // 2 * 2]), layout, scaling, page, far)
        while c["tokens"] * (c["heads"] + c["kv_heads"]) * dim > 8192 * 40 * 128:
            c["tokens"] = int(c["tokens"] * 0.7)
    elif kind == "attend":
        nodes = 1 if rng.random() < 0.4 else _log_int(rng, 2, 128)
        if rng.random() < 0.15:                 # the CUDA-core sizes: fp32 or an odd head size
            c = _attend("", _log_int(rng, 1, 16), _log_int(rng, 1, 2048), min(nodes, 32), 2 * min(kv_heads, 4), min(kv_heads, 4),
                        8 * rng.randint(4, 32), rng.choice(["f32", "f32", "bf16"]), page, rng.choice(["tree", "chain"]))
        else:
            c = _attend("", _log_int(rng, 1, 128), _log_int(rng, 1, 65536), nodes, kv_heads * group, kv_heads, rng.choice([64, 128, 128]),
                        "bf16", page, rng.choice(["tree", "chain"]))
        while _attend_cost(c) > 1.0:
            if c["batch"] > 1:
                c["batch"] = max(1, int(c["batch"] * 0.7))
            else:
                c["length"] = int(c["length"] * 0.7)
    elif kind == "beam":
        c = _beam("", _log_int(rng, 1, 64), rng.choice([1, 2, 3, 4, 8]), _log_int(rng, 1, 1024), rng.choice([1, 1, rng.randint(2, 40)]),
                  _log_int(rng, 1, 24), kv_heads, rng.choice([64, 128, 72]), rng.choice(["int4", "int4", "fp8", "plain"]), page)
        while c["requests"] > 1 and _pool_rows(c) > 32 << 20:
            c["requests"] = int(c["requests"] * 0.7)
    else:
        c = _compact("", _log_int(rng, 1, 64), _log_int(rng, 1, 2048), 0, _log_int(rng, 1, 24), kv_heads, rng.choice([64, 128, 72]),
                     rng.choice(["int4", "int4", "fp8", "plain"]), page)
        most = c["batch"] * -(-c["length"] // page)
        c["pages"] = max(most + 1, int(most * rng.uniform(1.05, 3.0)))
        while c["pages"] * c["page"] * c["layers"] * c["kv_heads"] * c["dim"] * {"int4": 1, "fp8": 2, "plain": 4}[c["format"]] > 6000 * 64 * 16 * 4 * 128:
            c["pages"], c["length"] = int(c["pages"] * 0.7), int(c["length"] * 0.7)
            c["pages"] = max(c["pages"], c["batch"] * -(-c["length"] // page) + 1)
            if c["length"] < 4:
                c["layers"] = max(1, c["layers"] // 2)
                c["length"] = 4
    del c["name"]
    return c


def _attend_cost(c):
    """Of the costliest listed case: cached bytes, products and padded fp32 intermediates of the plain form."""
    n, L = c["nodes"], c["length"] + c["nodes"]
    rows = c["batch"] * L * c["kv_heads"] * c["dim"]
    scores = c["batch"] * c["heads"] * n * L
    return max(rows / (8 * 16512 * 8 * 128 * 2.0), scores / (8 * 64 * 128 * 16512.0),
               scores * c["dim"] / (8 * 64 * 128 * 16512 * 128.0 * (1.0 if c["dtype"] == "bf16" and c["dim"] in (64, 128) else 0.01)))


def _pool_rows(c):
    """Cache rows of a beam case, all layers and heads, of 128 4-bit values' size."""
    pages = c["requests"] * (c["beams"] + 1) * (-(-(c["length"] + c["grow"]) // c["page"]) + 1)
    return pages * c["page"] * c["layers"] * c["kv_heads"] * c["dim"] / 128 * {"int4": 1, "fp8": 2, "plain": 4}[c["format"]]


# ----------------------------------------------------------------------- inputs


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + tag) & 0x7FFFFFFFFFFF)
    return g


def _randn(shape, seed, tag):
    return torch.randn(shape, generator=_gen(seed, tag), device="cuda")


def _keys(shape, dim, seed, tag):
    """Rows like keys: N(0, 1) with a few channels of several times the size."""
    x = _randn(shape, seed, tag)
    big = torch.ones(dim, device="cuda")
    big[torch.randperm(dim, generator=_gen(seed, tag + 50), device="cuda")[: max(1, dim // 32)]] = 4.0
    return x.mul_(big)


class _State:
    """What a serving program holds."""

    def __init__(self, case):
        self.case = case


def _rope_args(c):
    return {"none": {}, "linear": {"factor": 4.0}, "by_turns": {"factor": 8.0, "original_len": 8192, "low": 1.0, "high": 4.0},
            "by_index": {"factor": 16.0, "original_len": 4096, "low": 1.0, "high": 32.0, "magnitude": 0.1 * math.log(16.0) + 1.0}}[c["scaling"]]


def _base(c):
    return 500000.0 if c["scaling"] == "by_turns" else 10000.0


def _frequencies(c):
    """f_i in 64 bits, on the GPU."""
    a, R, base = _rope_args(c), c["rot"], _base(c)
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    t = base ** (-2.0 * i / R)
    if c["scaling"] == "none":
        return t
    if c["scaling"] == "linear":
        return t / a["factor"]
    L = a["original_len"]
    if c["scaling"] == "by_turns":
        g = ((L * t / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
    else:
        lo = max(math.floor(R * math.log(L / (2 * math.pi * a["high"])) / (2 * math.log(base))), 0)
        hi = min(math.ceil(R * math.log(L / (2 * math.pi * a["low"])) / (2 * math.log(base))), R - 1)
        g = 1 - ((i - lo) / ((hi if hi != lo else lo + 0.001) - lo)).clamp(0, 1)
    return t * (g + (1 - g) / a["factor"])


def _handles(st, c, layers=None, n_pages=None):
    """The plans and handles that a program which uses the kernels keeps beside its data."""
    from paper_2609_05228_gb300 import ace
    if "rot" in c:
        st.rope = ace.AceRope(c["dim"], c["rot"], c["layout"], _base(c), c["scaling"], dtype=c["dtype"], **_rope_args(c))
    if "format" in c:
        st.kv = ace.AceKvCache(c["kv_heads"], c["dim"], c["page"], n_pages, layers, c["dtype"], c["format"], st.k_pool, st.v_pool,
                               st.k_scale, st.v_scale)


def _shapes(c, layers, n_pages):
    """(pool shape, pool type, scale shape, scale type)."""
    rows = (layers, n_pages, c["kv_heads"], c["page"])
    D = c["dim"]
    return {"plain": (rows + (D,), DT[c["dtype"]], None, None), "fp8": (rows + (D,), torch.float8_e4m3fn, rows, torch.uint8),
            "int4": (rows + (D // 2,), torch.uint8, rows + (-(-D // GROUP),), torch.bfloat16)}[c["format"]]


def _new_pools(st, c, layers, n_pages):
    shape, dt, scale, scale_dt = _shapes(c, layers, n_pages)
    st.k_pool, st.v_pool = torch.zeros(shape, dtype=dt, device="cuda"), torch.zeros(shape, dtype=dt, device="cuda")
    st.k_scale = st.v_scale = None
    if scale:
        st.k_scale, st.v_scale = torch.zeros(scale, dtype=scale_dt, device="cuda"), torch.zeros(scale, dtype=scale_dt, device="cuda")


def _bytes(t):
    return t.view(torch.uint8) if t.dtype != torch.uint8 else t


def _pools(st, c):
    return [t for t in (st.k_pool, st.v_pool, st.k_scale, st.v_scale) if t is not None]


def _fill(st, c, seed):
    """Any bytes: what moves them does not look at them."""
    for i, t in enumerate(_pools(st, c)):
        b = _bytes(t)
        b.copy_(torch.randint(0, 256, b.shape, generator=_gen(seed, 30 + i), device="cuda", dtype=torch.uint8))


def _positions(c, seed):
    """Sequences that end anywhere up to `far`, a request's tokens one after another."""
    T = c["tokens"]
    run = max(1, T // 8)
    start = torch.randint(0, max(1, c["far"] - run), (-(-T // run),), generator=_gen(seed, 20), device="cuda")
    return (start[:, None] + torch.arange(run, device="cuda")).reshape(-1)[:T].int().contiguous()


def _parents(c, sizes, rng):
    """Parents (index in the request, -1 for node 0) of every node, drafted breadth first."""
    parents = []
    for n in sizes:
        if c["shape"] == "chain":
            parents += list(range(-1, n - 1))
        else:
            kids = np.zeros(n, int)
            of = [-1]
            for i in range(1, n):
                ok = np.nonzero(kids[:i] < 4)[0]
                p = int(ok[min(len(ok) - 1, int(rng.exponential(3.0)))])
                kids[p] += 1
                of.append(p)
            parents += of
    return parents


def _prepare_attend(st, c, seed):
    rng = np.random.default_rng(seed)
    B, n, page = c["batch"], c["nodes"], c["page"]
    sizes = np.full(B, n)
    if B > 1 and n > 1:
        sizes = np.random.default_rng(1000 * B + n).integers(max(1, n // 2), n + 1, B)
        sizes[B // 2] = n
    st.sizes, st.total = sizes, int(sizes.sum())
    off = np.concatenate([[0], np.cumsum(sizes)])
    st.offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    st.parents_host = _parents(c, sizes, rng)
    # ancestors' masks, as a program has them from the trees that it drafted
    words = -(-n // 64)
    mask = np.zeros((st.total, words), np.uint64)
    for b in range(B):
        for i in range(sizes[b]):
            t, p = off[b] + i, st.parents_host[off[b] + i]
            if p >= 0:
                mask[t] = mask[off[b] + p]
            mask[t, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    st.mask = torch.from_numpy(mask.view(np.int64)).cuda()
    lens = np.full(B, c["length"]) if B == 1 else rng.integers(c["length"] // 4, c["length"] + 1, B)
    # pages scattered over the pool, as after many requests have come and gone
    need = (lens + sizes + page - 1) // page
    n_pages = int(need.sum()) + 3
    order = rng.permutation(n_pages)
    table = np.zeros((B, int(need.max())), np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    for b in range(B):
        table[b, : need[b]] = order[at[b]: at[b + 1]]
    st.table, st.lens = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    st.max_len = int((lens + sizes).max())
    _new_pools(st, c, 1, n_pages)
    rows = (1, n_pages, c["kv_heads"], page, c["dim"])
    for pool, scale, x in ((st.k_pool, st.k_scale, _keys(rows, c["dim"], seed, 1)), (st.v_pool, st.v_scale, _randn(rows, seed, 2))):
        codes, s = _encode4(x)
        pool.copy_(codes)
        scale.copy_(s)
    st.q = _randn((st.total, c["heads"], c["dim"]), seed, 7).to(DT[c["dtype"]])
    st.out = torch.empty_like(st.q)
    st.lse = torch.empty(st.total, c["heads"], device="cuda")
    return n_pages


def _prepare_beam(st, c, seed):
    """Rows of a request share the pages of its prompt and have pages of their own behind it."""
    rng = np.random.default_rng(seed)
    Q, K, page = c["requests"], c["beams"], c["page"]
    B = Q * K
    shape = np.random.default_rng(17 * B + c["length"])         # lengths from the case: the work is the same for every seed
    lens = np.repeat(shape.integers(max(1, c["length"] // 4), c["length"] + 1, Q), K)
    prompt = (lens * shape.uniform(0.3, 0.9, B).reshape(Q, K)[:, :1].repeat(K, 1).reshape(-1)).astype(int) // page
    need = -(-lens // page)
    st.max_pages = int((-(-(lens + c["grow"]) // page)).max()) + 1
    used = int(sum(prompt[q * K] + (need - prompt)[q * K: q * K + K].sum() for q in range(Q)))
    n_pages = used + 2 * B + B * -(-c["grow"] // page) + 3
    order = rng.permutation(n_pages)
    table = np.full((B, st.max_pages), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    at = 0
    for b in range(B):
        first = b // K * K
        if b == first:
            table[b, : prompt[b]] = order[at: at + prompt[b]]
            at += prompt[b]
        else:
            table[b, : prompt[b]] = table[first, : prompt[b]]
        table[b, prompt[b]: need[b]] = order[at: at + need[b] - prompt[b]]
        at += need[b] - prompt[b]
        np.add.at(refs, table[b, : need[b]], 1)
    # the search keeps the better beams more than once, and some requests have ended
    parents = np.arange(B) // K * K + np.minimum(shape.integers(0, K, B), shape.integers(0, K, B))
    parents[(np.arange(B) // K) % 16 == 15] = -1
    st.table0, st.lens0, st.refs0 = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (table, lens, refs))
    st.parents = torch.tensor(parents, dtype=torch.int32, device="cuda")
    st.grow = torch.full((B,), c["grow"], dtype=torch.int32, device="cuda")
    st.grow[st.parents < 0] = 0
    st.refs, st.table, st.lens = torch.empty_like(st.refs0), torch.empty_like(st.table0), torch.empty_like(st.lens0)
    st.missing = torch.empty(1, dtype=torch.int32, device="cuda")
    _new_pools(st, c, c["layers"], n_pages)
    _fill(st, c, seed)
    return n_pages


def _prepare_compact(st, c, seed):
    rng = np.random.default_rng(seed)
    B, page, n_pages = c["batch"], c["page"], c["pages"]
    lens = np.random.default_rng(31 * B + c["length"]).integers(max(1, c["length"] // 4), c["length"] + 1, B)
    need = -(-lens // page)
    order = rng.permutation(n_pages)
    table = np.full((B, int(need.max()) + 1), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    at = 0
    for b in range(B):
        share = int(need[b]) // 3 if b % 4 == 3 else 0           # every fourth request was forked from the one before
        share = min(share, int(need[b - 1])) if share else 0
        table[b, :share] = table[b - 1, :share]
        table[b, share: need[b]] = order[at: at + need[b] - share]
        at += int(need[b]) - share
        np.add.at(refs, table[b, : need[b]], 1)
    st.table0, st.refs0 = torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda()
    st.table, st.refs = torch.empty_like(st.table0), torch.empty_like(st.refs0)
    st.new_page = torch.empty(n_pages, dtype=torch.int32, device="cuda")
    st.used = torch.empty(1, dtype=torch.int32, device="cuda")
    _new_pools(st, c, c["layers"], n_pages)
    _fill(st, c, seed)
    return n_pages


def prepare(case, seed):
    c = case
    st = _State(c)
    layers, n_pages = c.get("layers", 1), None
    if c["kind"] in ("rope", "enter"):
        T, H, K, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        dt = DT[c["dtype"]]
        # q, k and v as a fused projection leaves them: [T, heads of q, k, v] rows
        row = torch.cat([_randn((T, H, D), seed, 3), _keys((T, K, D), D, seed, 4), _randn((T, K, D), seed, 5)], 1).to(dt)
        st.q, st.k, st.v = row[:, :H], row[:, H: H + K], row[:, H + K:]
        st.positions = _positions(c, seed)
        st.q_out, st.k_out = torch.empty(T, H, D, dtype=dt, device="cuda"), torch.empty(T, K, D, dtype=dt, device="cuda")
        if c["kind"] == "enter":
            n_pages = -(-T // c["page"]) + 5
            _new_pools(st, c, 1, n_pages)
            st.slots = torch.randperm(n_pages * c["page"], generator=_gen(seed, 6), device="cuda")[:T].contiguous()
            st.v_out = torch.empty(T, K, D, dtype=dt, device="cuda")
    else:
        n_pages = {"attend": _prepare_attend, "beam": _prepare_beam, "compact": _prepare_compact}[c["kind"]](st, c, seed)
    if own:
        _handles(st, c, layers, n_pages)
    torch.cuda.empty_cache()
    return st


# ----------------------------------------------------------------------- one pass


def run(state):
    st, c = state, state.case
    if c["kind"] == "beam":         # the search's state before the step
        st.refs.copy_(st.refs0)
    elif c["kind"] == "compact":
        st.refs.copy_(st.refs0)
        st.table.copy_(st.table0)
    if not own:
        return {"rope": _plain_rope, "enter": _plain_enter, "attend": _plain_attend, "beam": _plain_beam,
                "compact": _plain_compact}[c["kind"]](st, c)
    if c["kind"] == "rope":
        st.rope.apply(st.positions, st.q, st.q_out, st.k, st.k_out, inverse=c["back"])
        return st.q_out, st.k_out
    if c["kind"] == "enter":
        st.kv.write_rotated(0, st.rope, st.positions, st.q, st.q_out, st.k, st.v, st.slots)
        st.kv.read(0, st.slots, st.k_out, st.v_out)
        return st.q_out, st.k_out, st.v_out
    if c["kind"] == "attend":
        st.kv.attend(0, st.q, st.table, st.lens, st.offsets, st.out, st.mask, c["nodes"], lse=st.lse)
        return st.out, st.lse
    if c["kind"] == "beam":
        st.kv.fork(st.table0, st.lens0, st.parents, st.refs, st.table, st.lens)
        st.kv.reserve(st.table, st.lens, st.grow, st.refs, st.missing)
        return (st.table, st.lens, st.refs, st.missing) + tuple(_bytes(t) for t in _pools(st, c))
    st.kv.compact(st.table, st.refs, st.used, st.new_page)
    return (st.table, st.refs, st.used, st.new_page) + tuple(_bytes(t) for t in _pools(st, c))


def _rotate(x, positions, c, back=False):
    """fp32 rows [T, heads, D] rotated; angles in 64 bits, as far positions want them."""
    R, m = c["rot"], _rope_args(c).get("magnitude", 1.0)
    a = positions.double()[:, None] * _frequencies(c)
    cos, sin = (a.cos() * m).float()[:, None], (a.sin() * m).float()[:, None]
    if back:
        sin = -sin
    x = x.float()
    if c["layout"] == "half":
        u, w = x[..., : R // 2], x[..., R // 2: R]
        turned = torch.cat([u * cos - w * sin, u * sin + w * cos], -1)
    else:
        u, w = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_rope(st, c):
    dt = DT[c["dtype"]]
    return _rotate(st.q, st.positions, c, c["back"]).to(dt), _rotate(st.k, st.positions, c, c["back"]).to(dt)


def _pow2(e):
    """2^e in 64 bits for whole e, exactly (exp2 and pow may be a bit off)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _encode8(x):
    """fp32 rows [..., D] -> (e4m3 codes, scale bytes)."""
    m, ex = torch.frexp(x.abs().amax(-1))                        # amax = m 2^ex, 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, ex - 8, ex - 9)
    e = torch.where(m > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    return (x * _pow2(-e[..., None])).float().to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _encode4(x):
    """fp32 rows [..., D] -> (two codes a byte, bf16 scales). Quotients in 64 bits: a value may lie next to a half."""
    D = x.shape[-1]
    pad = -D % GROUP
    g = torch.nn.functional.pad(x, (0, pad)).unflatten(-1, (-1, GROUP))
    m, ex = torch.frexp(g.abs().amax(-1).double() / 7)
    s = (torch.ceil(m * 16) * _pow2(ex - 4)).clamp(2.0 ** -126, 1.125 * 2.0 ** 125)
    code = torch.round(g / s[..., None]).clamp(-7, 7).to(torch.int16).flatten(-2)[..., :D] + 8
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), s.to(torch.bfloat16)


def _decode4(codes, scale):
    x = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8
    return x * scale.float().repeat_interleave(GROUP, -1)[..., : x.shape[-1]]


def _decode(st, c, pool, scale):
    if c["format"] == "int4":
        return _decode4(pool, scale)
    return (pool.float() * _pow2(scale.to(torch.int32)[..., None] - 127)).float() if c["format"] == "fp8" else pool.float()


def _plain_enter(st, c):
    dt = DT[c["dtype"]]
    at = (0, st.slots // c["page"], slice(None), st.slots % c["page"])
    out = []
    for x, pool, scale in ((_rotate(st.k, st.positions, c).to(dt), st.k_pool, st.k_scale), (st.v, st.v_pool, st.v_scale)):
        if c["format"] == "plain":
            pool[at] = x
            out.append(pool[at].clone())
            continue
        codes, s = (_encode4 if c["format"] == "int4" else _encode8)(x.float())
        _bytes(pool)[at] = _bytes(codes)
        scale[at] = s
        out.append(_decode(st, c, pool[at], scale[at]).to(dt))
    return _rotate(st.q, st.positions, c).to(dt), out[0], out[1]


def _plain_attend(st, c):
    n, H, G, D, B = c["nodes"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], c["batch"]
    off = st.offsets.long()
    t = torch.arange(st.total, device="cuda")
    req = torch.searchsorted(off, t, right=True) - 1
    idx = t - off[req]
    m = torch.arange(n, device="cuda")
    at = off[:-1, None] + m
    ok = at < off[1:, None]
    at = torch.where(ok, at, torch.zeros_like(at))
    sees = (((st.mask[at][..., m // 64] >> (m % 64)) & 1) == 1) & ok[..., None]
    pos = torch.arange(st.max_len, device="cuda")
    lens = st.lens.long()
    here = pos < (lens + (off[1:] - off[:-1]))[:, None]
    page = st.table[:, (pos // c["page"]).clamp(max=st.table.shape[1] - 1)].long()
    slot = torch.where(here, page * c["page"] + pos % c["page"], torch.zeros_like(page))
    cell = (0, slot // c["page"], slice(None), slot % c["page"])
    k, v = _decode4(st.k_pool[cell], st.k_scale[cell]), _decode4(st.v_pool[cell], st.v_scale[cell])      # [B, L, H, D]
    i = (pos - lens[:, None]).clamp(min=0, max=n - 1)
    mask = (pos < lens[:, None])[:, None] | (torch.gather(sees, 2, i[:, None].expand(B, n, -1)) & here[:, None])   # [B, n, L]
    q = st.q.float()[at].view(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(D)).view(B, H, n, G, -1)
    s.masked_fill_(~mask[:, None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, H, n * G, -1), v.transpose(1, 2)).view(B, H, n, G, D) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log())[..., 0]
    o = o.permute(0, 2, 1, 3, 4).reshape(B, n, H * G, D)[req, idx]
    return o.to(st.q.dtype), lse.permute(0, 2, 1, 3).reshape(B, n, H * G)[req, idx]


def _plain_beam(st, c):
    P, n_pages = c["page"], st.refs.shape[0]
    entry = torch.arange(st.max_pages, device="cuda")
    # fork
    old = entry < ((st.lens0 + P - 1) // P)[:, None]
    named = (st.table0 >= 0)
    parent = st.parents.long().clamp(min=0)
    there = (st.parents >= 0)[:, None]
    table = torch.where(old[parent] & there, st.table0[parent], torch.full_like(st.table0, -1))
    lens = torch.where(st.parents >= 0, st.lens0[parent], torch.zeros_like(st.lens0))
    ones = torch.ones_like(st.table0)
    refs = st.refs.index_add(0, st.table0.clamp(min=0).flatten().long(), -(ones * named).flatten())
    refs = refs.index_add(0, table.clamp(min=0).flatten().long(), (ones * (table >= 0)).flatten())
    # reserve: the partly filled page of a row that grows
    B = table.shape[0]
    row = torch.arange(B, device="cuda")
    part = ((lens % P) > 0) & (st.grow > 0)
    cell = (lens // P).long().clamp(max=st.max_pages - 1)
    page = table[row, cell].long().clamp(min=0)
    holders = torch.zeros_like(refs).index_add(0, page, part.int())
    last = torch.full_like(refs, -1).scatter_reduce(0, page, torch.where(part, row, torch.full_like(row, -1)).int(), "amax")
    copy = part & (refs[page] > 1) & ~((holders[page] == refs[page]) & (last[page] == row))
    need = -(-(lens + st.grow) // P)
    want = (entry < need[:, None]) & (table < 0) & (st.grow > 0)[:, None]
    want[row, cell] |= copy
    order = want.flatten().long().cumsum(0) - 1
    free = torch.sort(torch.where(refs == 0, torch.arange(n_pages, device="cuda"), n_pages)).values
    total, have = want.sum(), (refs == 0).sum()
    fresh = torch.where(want, free[order.clamp(0, n_pages - 1)].view_as(want).int(), table)
    enough = total <= have
    src = torch.where(copy, page, torch.zeros_like(page))
    dst = torch.where(copy & enough, fresh[row, cell].long(), src)
    # the rows before the row's length move; a row that copies nothing writes its first page to itself
    moved = (torch.arange(P, device="cuda") < (lens % P)[:, None]) & (copy & enough)[:, None]        # [B, P]
    b, r = moved.nonzero(as_tuple=True)
    for t in _pools(st, c):
        y = _bytes(t)
        y[:, dst[b], :, r] = y[:, src[b], :, r]
    new = torch.where(want & enough, ones, torch.zeros_like(ones))
    refs = refs.index_add(0, page, -(copy & enough).int()).index_add(0, fresh.clamp(min=0).flatten().long(), new.flatten())
    table = torch.where(enough, fresh, table)
    missing = (total - have).clamp(min=0).int()[None]
    return (table, lens, refs, missing) + tuple(_bytes(t) for t in _pools(st, c))


def _plain_compact(st, c):
    n_pages = st.refs.shape[0]
    live = st.refs > 0
    n = live.sum()
    page = torch.arange(n_pages, device="cuda")
    high, low = live & (page >= n), ~live & (page < n)           # as many of the one as of the other
    src, dst = high.nonzero()[:, 0], low.nonzero()[:, 0]
    new = torch.where(live, page, torch.full_like(page, -1))
    new[src] = dst
    for t in _pools(st, c):
        y = _bytes(t)
        y[:, dst] = y[:, src]
    table = torch.where(st.table >= 0, new[st.table.clamp(min=0).long()].int(), st.table)
    refs = st.refs.clone()
    refs[dst] = refs[src]
    refs[src] = 0
    return (table, refs, n.int()[None], new.int()) + tuple(_bytes(t) for t in _pools(st, c))


# ----------------------------------------------------------------------- what a pass needs


def _row_bytes(c):
    D = c["dim"]
    return {"plain": D * (2 if c["dtype"] == "bf16" else 4), "fp8": D + 1, "int4": D // 2 + 2 * -(-D // GROUP)}[c["format"]]


def work(case):
    c = case
    D = c["dim"]
    E = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        n = c["tokens"] * (c["heads"] + c["kv_heads"])
        return {"bytes": float(2 * n * D * E + 4 * c["tokens"]), "flops": float(3 * n * c["rot"])}
    if c["kind"] == "enter":      # q in and out; k and v in, codes out; codes in, rows out
        n = c["tokens"]
        return {"bytes": float(n * (2 * c["heads"] * D * E + 2 * c["kv_heads"] * (2 * D * E + 2 * _row_bytes(c)) + 12)),
                "flops": float(3 * n * (c["heads"] + c["kv_heads"]) * c["rot"])}
    if c["kind"] == "attend":
        many = c["batch"] > 1
        n = c["nodes"] * (0.75 if many and c["nodes"] > 1 else 1.0)
        L = c["length"] * (0.625 if many else 1.0) + n
        B = c["batch"]
        return {"bytes": float(B * (2 * c["kv_heads"] * L * _row_bytes(c) + 2 * n * c["heads"] * D * E + n * c["heads"] * 4)),
                "flops": float(4 * B * c["heads"] * n * L * D)}
    page_row = 2 * c["layers"] * c["kv_heads"] * _row_bytes(c)     # K and V of a position
    if c["kind"] == "beam":       # about 0.4 of the rows copy half a page; tables in and out, refs in and out
        B = c["requests"] * c["beams"]
        need = 0.625 * c["length"] / c["page"] + 1
        shared = 0.4 if c["beams"] > 1 else 0.0
        return {"bytes": float(2 * shared * B * c["page"] / 2 * page_row + 4 * (2 * B * need + 2 * B * need * 0.7)), "flops": 0.0}
    live = c["batch"] * (0.625 * c["length"] / c["page"] + 0.5) * 0.92
    moved = live * max(0.0, 1 - live / c["pages"])
    return {"bytes": float(2 * moved * c["page"] * page_row + 8 * c["pages"] + 8 * live), "flops": 0.0}


# ----------------------------------------------------------------------- the same in 64 bits


def exact(case, seed):
    c = case
    if c["kind"] in ("beam", "compact"):
        return None                 # whole numbers, compared as such
    if c["kind"] == "attend" and 4.0 * c["batch"] * c["heads"] * c["nodes"] * (c["length"] + c["nodes"]) * c["dim"] > 6e12:
        return None
    st = prepare(c, seed)
    return {"rope": _exact_rope, "enter": _exact_enter, "attend": _exact_attend}[c["kind"]](st, c)


def _exact_turned(x, positions, c, sign):
    """Rotation as a product of complex numbers."""
    R, a, base = c["rot"], _rope_args(c), _base(c)
    f = []
    for i in range(R // 2):
        t = math.pow(base, -2.0 * i / R)
        s, L = a.get("factor", 1.0), a.get("original_len", 0)
        if c["scaling"] == "none":
            keep = 1.0
        elif c["scaling"] == "linear":
            keep = 0.0
        elif c["scaling"] == "by_turns":
            keep = min(1.0, max(0.0, (L * t / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])))
        else:
            at = [R / 2 * math.log(L / (2 * math.pi * b)) / math.log(base) for b in (a["high"], a["low"])]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
            hi = lo + 0.001 if hi == lo else hi
            keep = 1.0 - min(1.0, max(0.0, (i - lo) / (hi - lo)))
        f.append(t * keep + t / s * (1.0 - keep))
    turn = torch.polar(torch.full((1,), a.get("magnitude", 1.0), dtype=torch.float64, device="cuda"),
                       sign * positions.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda"))[:, None]
    y = x.double().clone()
    first, second = (slice(0, R // 2), slice(R // 2, R)) if c["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
    z = torch.complex(y[..., first].clone(), y[..., second].clone()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rope(st, c):
    sign = -1.0 if c["back"] else 1.0
    return _exact_turned(st.q, st.positions, c, sign), _exact_turned(st.k, st.positions, c, sign)


def _exact_values8(x):
    power = torch.tensor([2.0 ** k for k in range(-200, 201)], dtype=torch.float64, device=x.device)
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(amax, -126, dtype=torch.int64)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):                  # the largest e whose 448 * 2^e is too little, and one more
        e = torch.where(amax > 448.0 * power[(e + step).clamp(max=200) + 200], e + step, e)
    e = torch.where(amax > 448.0 * power[e + 200], e + 1, e)
    y = x / power[e + 200]
    step = power[torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).long() - 3 + 200]
    return torch.round(y / step) * step * power[e + 200]


def _exact_values4(x):
    """Group by group: the least 4-bit number times a power of two that is enough, and the nearest multiple of it."""
    power = torch.tensor([2.0 ** k for k in range(-200, 201)], dtype=torch.float64, device=x.device)
    out = []
    for g in x.split(GROUP, -1):
        amax = g.abs().amax(-1, keepdim=True)
        p = power[torch.floor(torch.log2((amax / 7).clamp(min=2.0 ** -140))).long() - 3 + 200]       # 8 .. 16 times it, or a step off
        s = torch.full_like(amax, math.inf)
        for u in (18, 16, 15, 14, 13, 12, 11, 10, 9, 8, 7.5, 7):
            s = torch.where(7 * u * p >= amax, u * p, s)
        s = s.clamp(2.0 ** -126, 1.125 * 2.0 ** 125)
        out.append(torch.round(g / s).clamp(-7, 7) * s)
    return torch.cat(out, -1)


def _exact_enter(st, c):
    # k is kept as a number of the storage type, whatever the cache makes of it then
    k = _exact_turned(st.k, st.positions, c, 1.0).to(DT[c["dtype"]]).double()
    f = {"plain": lambda x: x, "fp8": _exact_values8, "int4": _exact_values4}[c["format"]]
    return _exact_turned(st.q, st.positions, c, 1.0), f(k), f(st.v.double())


def _exact_attend(st, c):
    off, lens = st.offsets.tolist(), st.lens.tolist()
    G, D = c["heads"] // c["kv_heads"], c["dim"]
    out = torch.zeros(st.total, c["heads"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((st.total, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    group = torch.arange(D, device="cuda") // GROUP
    for b in range(c["batch"]):
        n, L = off[b + 1] - off[b], lens[b]
        sees = np.zeros((n, n), bool)
        for i in range(n):
            m = i
            while m >= 0:
                sees[i, m] = True
                m = st.parents_host[off[b] + m]
        mask = torch.cat([torch.ones(n, L, dtype=torch.bool), torch.from_numpy(sees)], 1).cuda()
        pages = st.table[b, : -(-(L + n) // c["page"])].long()
        for h in range(c["kv_heads"]):
            kv = []
            for x in ("k", "v"):
                codes = getattr(st, x + "_pool")[0, pages, h].flatten(0, 1)[: L + n]
                y = torch.empty(L + n, D, dtype=torch.float64, device="cuda")
                y[:, 0::2], y[:, 1::2] = (codes % 16).double() - 8, (codes // 16).double() - 8
                kv.append(y * getattr(st, x + "_scale")[0, pages, h].flatten(0, 1)[: L + n].double()[:, group])
            for g in range(G):
                s = st.q[off[b]: off[b + 1], h * G + g].double() @ kv[0].T / math.sqrt(D)
                s = s.masked_fill(~mask, -math.inf)
                lse[off[b]: off[b + 1], h * G + g] = torch.logsumexp(s, 1)
                out[off[b]: off[b + 1], h * G + g] = torch.softmax(s, 1) @ kv[1]
    return out, lse
