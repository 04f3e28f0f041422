"""The measured cases of the speculative decode step's operators: the key/value cache that is quantised as
it is written, attention for a tree of drafted tokens over it, and the verification of the drafted tokens.

A case's "kind" says which operator one pass runs:

  cache   the K and V rows of new tokens are written into the paged cache and read back
  keep    the accepted nodes' rows of all layers move to the front of their trees and are read back
  attend  every node of every request's tree attends to the request's cached prefix and to its ancestors
  verify  the walk down the trees that accepts drafted tokens and picks each request's next token

Layouts and formulas (own and plain form alike):

  pool[layer, page, head, row, D]; slot = page * page_size + row. Format "plain" keeps the rows as they
  come. Format "fp8" keeps e4m3 codes and a byte per (token, head), E = e + 127, where e is the smallest
  integer >= -126 with max |x| <= 448 * 2^e over the row; a code stands for code * 2^e.

  Request b has lens[b] committed rows and the nodes node_offsets[b] .. node_offsets[b + 1] - 1, whose
  rows are at positions lens[b] + i. Bit m of mask[t] says that node t sees node m of its request.

  Verification: node 0 is the last committed token, parents say the tree. At a node r = softmax(logits /
  temperature) and q = its draft row; children in index order: accepted if r(x) > 0 and u * q(x) <= r(x),
  else r becomes max(r - q, 0) and q loses x, both renormalised. Where no child is left the next token is
  argmax r(v) / noise(v). Without draft rows q is a point mass at the child. Temperature 0 is greedy.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
VOCAB_SHARP = 2.5          # standard deviation of the logits beside each row's likely token


# ----------------------------------------------------------------------- cases


def _cache(name, T, heads, dim, fmt="fp8", dtype="bf16", page=64):
    return {"name": name, "kind": "cache", "tokens": T, "kv_heads": heads, "dim": dim, "format": fmt, "dtype": dtype,
            "page": page}


def _keep(name, B, nodes, layers, heads, dim, fmt="fp8", page=64, length=512):
    return {"name": name, "kind": "keep", "batch": B, "nodes": nodes, "layers": layers, "kv_heads": heads, "dim": dim,
            "format": fmt, "dtype": "bf16", "page": page, "length": length, "shape": "tree"}


def _attend(name, B, length, nodes, heads, kv_heads, dim, fmt="fp8", dtype="bf16", page=64, shape="tree", fresh=False):
    return {"name": name, "kind": "attend", "batch": B, "length": length, "nodes": nodes, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "format": fmt, "dtype": dtype, "page": page, "shape": shape, "fresh": fresh}


def _verify(name, B, nodes, vocab, dtype="bf16", draft="probs", shape="tree", temp="mixed"):
    return {"name": name, "kind": "verify", "batch": B, "nodes": nodes, "vocab": vocab, "dtype": dtype, "draft": draft,
            "shape": shape, "temp": temp}


def listed():
    return [
        # a decode step's K and V rows for 64 users: latency
        _cache("cache_64", 64, 4, 128),
        # a batch of prompts enters the cache
        _cache("cache_16384", 16384, 8, 128),
        # 32 users keep the accepted rows of a 16-node tree in every layer
        _keep("keep_32", 32, 16, 16, 4, 128),
        # a busy server with large trees and an unquantised cache
        _keep("keep_128_plain", 128, 64, 48, 8, 128, fmt="plain", length=256),
        # one user's next token after a short conversation, unquantised: the smallest call
        _attend("attend_1", 1, 2048, 1, 32, 4, 128, fmt="plain", shape="chain"),
        # a busy server's plain decode step, ragged lengths
        _attend("attend_64", 64, 8192, 1, 32, 4, 128, shape="chain"),
        # a speculative step: 16-node trees that the drafter draws anew each step, ragged
        _attend("attend_tree_24", 24, 4096, 16, 64, 8, 128, page=16, fresh=True),
        # one user with a very long context and a chain of drafted tokens: split over the long axis
        _attend("attend_long", 1, 262144, 5, 64, 8, 128, shape="chain", page=128),
        # large trees, where the products and not the cache decide
        _attend("attend_wide_8", 8, 16384, 128, 64, 8, 128, fmt="plain"),
        # the fp32 layer used to develop and check a model, an odd head size
        _attend("attend_f32", 4, 777, 6, 8, 2, 80, dtype="f32", page=16),
        # one user, a chain of 7 drafted tokens
        _verify("verify_1", 1, 8, 32000, shape="chain"),
        # a busy server, trees
        _verify("verify_64", 64, 16, 128000),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choices(["cache", "keep", "attend", "verify"], [2, 1, 6, 2])[0]
    fmt = rng.choice(["fp8", "fp8", "plain"])
    page = rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 16])
    dim = rng.choice([64, 128, 128])
    if kind == "cache":
        f32 = rng.random() < 0.25
        dim = 8 * rng.randint(4, 32) if f32 else dim
        c = _cache("", _log_int(rng, 1, 16384), kv_heads, dim, fmt, "f32" if f32 else "bf16", page)
        while c["tokens"] * c["kv_heads"] * c["dim"] > 16384 * 1024:
            c["tokens"] = int(c["tokens"] * 0.7)
    elif kind == "keep":
        c = _keep("", _log_int(rng, 1, 128), _log_int(rng, 4, 64), _log_int(rng, 1, 48), min(kv_heads, 8), dim, fmt, page,
                  _log_int(rng, 1, 512))
    elif kind == "attend":
        nodes = 1 if rng.random() < 0.3 else _log_int(rng, 2, 128)
        if rng.random() < 0.15:                 # the CUDA-core sizes: fp32 or an odd head size
            c = _attend("", _log_int(rng, 1, 16), _log_int(rng, 1, 2048), min(nodes, 32), 2 * min(kv_heads, 4),
                        min(kv_heads, 4), 8 * rng.randint(4, 32), fmt, rng.choice(["f32", "f32", "bf16"]), page,
                        rng.choice(["tree", "chain"]))
        else:
            group = rng.choice([1, 2, 4, 5, 8, 8, 16])
            c = _attend("", _log_int(rng, 1, 128), _log_int(rng, 1, 65536), nodes, kv_heads * group, kv_heads, dim, fmt,
                        "bf16", page, rng.choice(["tree", "chain"]), rng.random() < 0.3)
        while _attend_cost(c) > 1.0:
            if c["batch"] > 1:
                c["batch"] = max(1, int(c["batch"] * 0.7))
            else:
                c["length"] = int(c["length"] * 0.7)
    else:
        c = _verify("", _log_int(rng, 1, 64), _log_int(rng, 2, 32), _log_int(rng, 1000, 128000),
                    rng.choice(["bf16", "f32"]), rng.choice(["probs", "probs", "none"]), rng.choice(["tree", "chain"]),
                    rng.choice(["mixed", "one"]))
    del c["name"]
    return c


def _attend_cost(c):
    """Of the costliest listed case: cached bytes, products and padded fp32 intermediates of the plain form."""
    n, L = c["nodes"], c["length"] + c["nodes"]
    rows = c["batch"] * L * c["kv_heads"] * c["dim"]
    scores = c["batch"] * c["heads"] * n * L
    return max(rows / (8 * 16512 * 8 * 128 * 2.0), scores / (8 * 64 * 128 * 16512.0),
               scores * c["dim"] / (8 * 64 * 128 * 16512 * 128.0 * (1.0 if c["dtype"] == "bf16" and c["dim"] in (64, 128) else 0.01)))


# ----------------------------------------------------------------------- inputs


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + tag) & 0x7FFFFFFFFFFF)
    return g


def _randn(shape, seed, tag):
    return torch.randn(shape, generator=_gen(seed, tag), device="cuda")


def _rand(shape, seed, tag):
    return torch.rand(shape, generator=_gen(seed, tag), device="cuda")


def _keys(shape, dim, seed, tag):
    """Rows like keys after a rotary embedding: N(0, 1) with a few channels of several times the size."""
    x = _randn(shape, seed, tag)
    big = torch.ones(dim, device="cuda")
    big[torch.randperm(dim, generator=_gen(seed, tag + 50), device="cuda")[: max(1, dim // 32)]] = 4.0
    return x.mul_(big)


def _encode(x):
    """fp32 rows [..., D] -> (e4m3 codes, scale bytes): the format's definition."""
    fine = torch.isfinite(x)
    amax = torch.where(fine, x.abs(), torch.zeros_like(x)).amax(-1)
    m, ex = torch.frexp(amax)                                   # amax = m * 2^ex, 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, ex - 8, ex - 9)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    code = torch.where(fine, torch.ldexp(x, -e[..., None]), torch.full_like(x, math.nan)).to(torch.float8_e4m3fn)
    return code, (e + 127).to(torch.uint8)


def _decode(code, scale):
    return torch.ldexp(code.float(), scale.to(torch.int32)[..., None] - 127)


def _pools(st, c, layers, n_pages, seed, filled):
    """The cache's memory, owned by the program: as a server holds it after some hours (`filled`), or new."""
    shape = (layers, n_pages, c["kv_heads"], c["page"], c["dim"])
    fp8 = c["format"] == "fp8"
    st.k_scale = st.v_scale = None
    if not filled:
        dt = torch.float8_e4m3fn if fp8 else DT[c["dtype"]]
        st.k_pool, st.v_pool = torch.zeros(shape, dtype=dt, device="cuda"), torch.zeros(shape, dtype=dt, device="cuda")
        if fp8:
            st.k_scale = torch.zeros(shape[:-1], dtype=torch.uint8, device="cuda")
            st.v_scale = torch.zeros(shape[:-1], dtype=torch.uint8, device="cuda")
    else:
        k, v = _keys(shape, c["dim"], seed, 1), _randn(shape, seed, 2)
        if fp8:
            st.k_pool, st.k_scale = _encode(k)
            st.v_pool, st.v_scale = _encode(v)
        else:
            st.k_pool, st.v_pool = k.to(DT[c["dtype"]]), v.to(DT[c["dtype"]])
    if own:      # the same inputs either way; a program that uses the kernels keeps a handle of its cache too
        from paper_2609_05228_gb300 import ace
        st.kv = ace.AceKvCache(c["kv_heads"], c["dim"], c["page"], n_pages, layers, c["dtype"], c["format"], st.k_pool,
                               st.v_pool, st.k_scale, st.v_scale)


class _State:
    """What a serving program holds."""

    def __init__(self, case):
        self.case = case


def _parents(c, sizes, rng):
    """Parents (index in the request, -1 for node 0) of every node, drafted breadth first."""
    parents = []
    for n in sizes:
        if c["shape"] == "chain":
            parents += list(range(-1, n - 1))
        else:
            kids = np.zeros(n, int)
            own_parents = [-1]
            for i in range(1, n):
                ok = np.nonzero(kids[:i] < 4)[0]
                p = int(ok[min(len(ok) - 1, int(rng.exponential(3.0)))])
                kids[p] += 1
                own_parents.append(p)
            parents += own_parents
    return parents


def _requests(st, c, seed):
    """Node counts (ragged but for a single request, and the case's own), offsets, parents."""
    rng = np.random.default_rng(seed)
    B, n = c["batch"], c["nodes"]
    sizes = np.full(B, n)
    if B > 1 and n > 1:
        sizes = np.random.default_rng(1000 * B + n).integers(max(1, n // 2), n + 1, B)
        sizes[B // 2] = n
    st.sizes = sizes
    st.offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    st.total = int(sizes.sum())
    st.parents_host = _parents(c, sizes, rng)
    depth = []
    for i, p in enumerate(st.parents_host):
        depth.append(1 if p < 0 else depth[root + p] + 1)
        root = i if p < 0 else root
    st.max_depth = max(depth)
    st.parents = torch.tensor(st.parents_host, dtype=torch.int32, device="cuda")
    return rng


def _tables(st, c, lens, rng):
    """Pages scattered over the pool, as after many requests have come and gone."""
    need = (lens + st.sizes + c["page"] - 1) // c["page"]
    st.n_pages = int(need.sum()) + 3
    order = rng.permutation(st.n_pages)
    table = np.zeros((len(lens), int(need.max())), np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    for b in range(len(lens)):
        table[b, : need[b]] = order[at[b]: at[b + 1]]
    st.table = torch.from_numpy(table).cuda()
    st.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    st = _State(c)
    dt = DT[c["dtype"]]
    if c["kind"] == "cache":
        T, H, D = c["tokens"], c["kv_heads"], c["dim"]
        n_pages = -(-T // c["page"]) + 5
        _pools(st, c, 1, n_pages, seed, False)
        # K and V as a fused projection leaves them: [T, heads of q, k, v] rows
        row = torch.cat([_randn((T, 2 * H, D), seed, 3), _keys((T, H, D), D, seed, 4), _randn((T, H, D), seed, 5)], 1).to(dt)
        st.k, st.v = row[:, 2 * H: 3 * H], row[:, 3 * H:]
        st.slots = torch.randperm(n_pages * c["page"], generator=_gen(seed, 6), device="cuda")[:T].contiguous()
        st.k_out, st.v_out = torch.empty(1, T, H, D, dtype=dt, device="cuda"), torch.empty(1, T, H, D, dtype=dt, device="cuda")
    elif c["kind"] == "keep":
        rng = _requests(st, c, seed)
        B, n = c["batch"], c["nodes"]
        _tables(st, c, rng.integers(max(1, c["length"] // 2), c["length"] + 1, B), rng)
        _pools(st, c, c["layers"], st.n_pages, seed, True)
        # accepted paths: increasing nodes after the root; the moved rows lie past the places they move to
        some = np.random.default_rng(1000 * B + n + 1)
        keep = np.array([1 + some.integers(0, max(1, int(math.sqrt(s)))) for s in st.sizes])
        path = np.full((B, n), -1, np.int32)
        for b in range(B):
            path[b, 0] = 0
            path[b, 1: keep[b]] = np.sort(rng.choice(np.arange(keep[b], st.sizes[b]), keep[b] - 1, replace=False))
        st.path = torch.from_numpy(path).cuda()
        st.n_keep = torch.tensor(keep, dtype=torch.int32, device="cuda")
        st.new_lens = torch.empty_like(st.lens)
        pos = np.concatenate([np.arange(keep[b]) for b in range(B)])
        req = np.repeat(np.arange(B), keep)
        st.req, st.pos = torch.from_numpy(req).cuda(), torch.from_numpy(pos).cuda()
        at = st.lens[st.req].long() + st.pos
        st.slots = st.table[st.req, at // c["page"]].long() * c["page"] + at % c["page"]
        shape = (c["layers"], len(pos), c["kv_heads"], c["dim"])
        st.k_out, st.v_out = torch.empty(shape, dtype=dt, device="cuda"), torch.empty(shape, dtype=dt, device="cuda")
    elif c["kind"] == "attend":
        rng = _requests(st, c, seed)
        B = c["batch"]
        lens = np.full(B, c["length"]) if B == 1 else rng.integers(c["length"] // 4, c["length"] + 1, B)
        _tables(st, c, lens, rng)
        _pools(st, c, 1, st.n_pages, seed, True)
        st.q = _randn((st.total, c["heads"], c["dim"]), seed, 7).to(dt)
        st.max_len = int((lens + st.sizes).max())
        words = -(-c["nodes"] // 64)
        st.mask = torch.zeros(st.total, words, dtype=torch.int64, device="cuda")
        if not c["fresh"]:
            st.mask.copy_(_pack(_ancestors(st), words))
        st.out = torch.empty_like(st.q)
        st.lse = torch.empty(st.total, c["heads"], device="cuda")
    else:
        _requests(st, c, seed)
        B, V = c["batch"], c["vocab"]
        # the drafter is a smaller model: its logits are the target's and an error
        z = _randn((st.total, V), seed, 8) * VOCAB_SHARP
        # one likely token a row, of a probability between a tenth and nine tenths mostly
        likely = (_rand((st.total, 1), seed, 13) * V).long().clamp_(max=V - 1)
        z.scatter_(1, likely, math.log(V) + VOCAB_SHARP ** 2 / 2 + 1.0 + 1.5 * _randn((st.total, 1), seed, 14))
        draft = z + 0.35 * VOCAB_SHARP * _randn((st.total, V), seed, 9)
        st.logits = z.to(dt)
        probs = torch.softmax(draft, 1)
        del z
        # children: distinct tokens drawn from the parent's draft row
        st.tokens = torch.zeros(st.total, dtype=torch.int32, device="cuda")
        race = probs / torch.empty_like(probs).exponential_(generator=_gen(seed, 10))
        top = torch.topk(race, min(V, 4), 1).indices.int()
        off = np.repeat(np.concatenate([[0], np.cumsum(st.sizes)])[:-1], st.sizes)
        par = np.array(st.parents_host)
        at = np.nonzero(par >= 0)[0]
        owner = off[at] + par[at]
        rank = np.zeros(len(at), int)
        seen = {}
        for i, o in enumerate(owner):
            rank[i] = seen.get(o, 0)
            seen[o] = rank[i] + 1
        st.tokens[torch.from_numpy(at).cuda()] = top[torch.from_numpy(owner).cuda(), torch.from_numpy(rank).cuda()]
        st.max_kids = max(seen.values(), default=0)
        st.draft = probs if c["draft"] == "probs" else None
        st.temp = torch.ones(B, device="cuda")
        if c["temp"] == "mixed":
            st.temp = torch.tensor([0.8, 1.0, 0.0, 0.6], device="cuda").repeat(-(-B // 4))[:B].contiguous()
        st.u = _rand((st.total,), seed, 11)
        st.noise = torch.empty(B, V, device="cuda").exponential_(generator=_gen(seed, 12)).clamp_(min=1e-30)
        st.path = torch.empty(B, c["nodes"], dtype=torch.int32, device="cuda")
        st.n_keep = torch.empty(B, dtype=torch.int32, device="cuda")
        st.next = torch.empty(B, dtype=torch.int32, device="cuda")
        del draft, probs, race, top
    torch.cuda.empty_cache()
    return st


# ----------------------------------------------------------------------- one pass


def run(state):
    st, c = state, state.case
    if not own:
        return {"cache": _plain_cache, "keep": _plain_keep, "attend": _plain_attend, "verify": _plain_verify}[c["kind"]](st, c)
    from paper_2609_05228_gb300 import ace
    if c["kind"] == "cache":
        st.kv.write(0, st.k, st.v, st.slots)
        st.kv.read(None, st.slots, st.k_out, st.v_out)
        return st.k_out, st.v_out
    if c["kind"] == "keep":
        st.kv.keep(st.table, st.lens, st.path, st.n_keep, st.new_lens)
        st.kv.read(None, st.slots, st.k_out, st.v_out)
        return st.k_out, st.v_out, st.new_lens
    if c["kind"] == "attend":
        if c["fresh"]:
            ace.ace_tree_mask(st.parents, st.offsets, c["batch"], c["nodes"], st.mask)
        st.kv.attend(0, st.q, st.table, st.lens, st.offsets, st.out, st.mask, c["nodes"], lse=st.lse)
        return st.out, st.lse
    ace.ace_verify_tree(st.logits, st.tokens, st.parents, st.offsets, c["nodes"], st.u, st.noise, st.path, st.n_keep,
                        st.next, st.draft, st.temp)
    return st.path, st.n_keep, st.next


def _rows(st, c, layer, slots):
    """(k, v) fp32 rows at `slots` (layer None: of all layers)."""
    at = (slice(None) if layer is None else layer, slots // c["page"], slice(None), slots % c["page"])
    # indices apart by a slice put their axis first: [..., layers, heads, D] -> [layers, ..., heads, D]
    k, v = st.k_pool[at], st.v_pool[at]
    if c["format"] == "fp8":
        k, v = _decode(k, st.k_scale[at]), _decode(v, st.v_scale[at])
    k, v = k.float(), v.float()
    if layer is None:
        k, v = k.movedim(-3, 0), v.movedim(-3, 0)
    return k, v


def _plain_cache(st, c):
    at = (0, st.slots // c["page"], slice(None), st.slots % c["page"])
    if c["format"] == "fp8":
        kc, ks = _encode(st.k.float())
        vc, vs = _encode(st.v.float())
        st.k_scale[at], st.v_scale[at] = ks, vs
        st.k_pool.view(torch.uint8)[at], st.v_pool.view(torch.uint8)[at] = kc.view(torch.uint8), vc.view(torch.uint8)
    else:
        st.k_pool[at], st.v_pool[at] = st.k, st.v
    k, v = _rows(st, c, None, st.slots)
    return k.to(DT[c["dtype"]]), v.to(DT[c["dtype"]])


def _plain_keep(st, c):
    src = st.lens[st.req].long() + st.path[st.req, st.pos].long()
    src = st.table[st.req, src // c["page"]].long() * c["page"] + src % c["page"]
    a = (slice(None), src // c["page"], slice(None), src % c["page"])
    b = (slice(None), st.slots // c["page"], slice(None), st.slots % c["page"])
    if c["format"] == "fp8":
        st.k_scale[b], st.v_scale[b] = st.k_scale[a], st.v_scale[a]
        kp, vp = st.k_pool.view(torch.uint8), st.v_pool.view(torch.uint8)
    else:
        kp, vp = st.k_pool, st.v_pool
    kp[b], vp[b] = kp[a], vp[a]
    k, v = _rows(st, c, None, st.slots)
    return k.to(DT[c["dtype"]]), v.to(DT[c["dtype"]]), st.lens + st.n_keep


def _node_index(st):
    """(request, index in the request) of every node, and [B, n_max] packed indices with a validity mask."""
    off = st.offsets.long()
    t = torch.arange(st.total, device="cuda")
    req = torch.searchsorted(off, t, right=True) - 1
    i = torch.arange(st.case["nodes"], device="cuda")
    at = off[:-1, None] + i
    ok = at < off[1:, None]
    return req, t - off[req], torch.where(ok, at, torch.zeros_like(at)), ok


def _ancestors(st):
    """[B, n, n] bool: node i sees node m, itself and its ancestors. With A the matrix of parents,
    (I - A)^-1 = I + A + A^2 + ..., which holds a one for each ancestor."""
    n = st.case["nodes"]
    _, _, at, ok = _node_index(st)
    par = st.parents[at].long()
    A = (par[..., None] == torch.arange(n, device="cuda")) & ok[..., None]
    eye = torch.eye(n, device="cuda")
    return (torch.linalg.solve_triangular(eye - A.float(), eye, upper=False, unitriangular=True) > 0.5) & ok[..., None]


def _pack(sees_all, words):
    """[B, n, n] bool -> the present nodes' mask words [total, words] int64."""
    B, n, _ = sees_all.shape
    bits = torch.zeros(B, n, words * 64, dtype=torch.int64, device="cuda")
    bits[..., :n] = sees_all
    weight = torch.ones((), dtype=torch.int64, device="cuda") << torch.arange(64, device="cuda")
    packed = (bits.view(B, n, words, 64) * weight).sum(-1)
    return packed[sees_all.diagonal(dim1=1, dim2=2)]          # every present node sees itself


def _plain_attend(st, c):
    n, H, G, D = c["nodes"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    req, idx, at, ok = _node_index(st)
    if c["fresh"]:
        sees = _ancestors(st)
    else:
        m = torch.arange(n, device="cuda")
        sees = (((st.mask[at][..., m // 64] >> (m % 64)) & 1) == 1) & ok[..., None]
    B = c["batch"]
    pos = torch.arange(st.max_len, device="cuda")
    lens = st.lens.long()
    here = pos < (lens + (st.offsets[1:] - st.offsets[:-1]))[:, None]
    page = st.table[:, (pos // c["page"]).clamp(max=st.table.shape[1] - 1)].long()
    k, v = _rows(st, c, 0, torch.where(here, page * c["page"] + pos % c["page"], torch.zeros_like(page)))   # [B, L, H, D]
    m = (pos - lens[:, None]).clamp(min=0, max=n - 1)
    mask = (pos < lens[:, None])[:, None] | (torch.gather(sees, 2, m[:, None].expand(B, n, -1)) & here[:, None])   # [B, n, L]
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


def _plain_verify(st, c):
    """The walk for all requests side by side; its steps depend on one another, so depth and children are loops."""
    B, V, n = c["batch"], c["vocab"], c["nodes"]
    req, idx, at, ok = _node_index(st)
    par = torch.where(ok, st.parents[at].long(), torch.full_like(at, -2))             # [B, n]
    off = st.offsets[:-1].long()
    greedy = (st.temp == 0)[:, None]
    b = torch.arange(B, device="cuda")
    node = torch.zeros(B, dtype=torch.int64, device="cuda")
    live = ok[:, 0].clone()
    path = torch.full((B, n), -1, dtype=torch.int32, device="cuda")
    keep = torch.zeros(B, dtype=torch.int64, device="cuda")
    token = torch.full((B,), -1, dtype=torch.int64, device="cuda")
    for _ in range(st.max_depth):
        path[b, keep.clamp(max=n - 1)] = torch.where(live, node.int(), path[b, keep.clamp(max=n - 1)])
        keep = keep + live
        z = st.logits[off + node].float()
        r = (z / torch.where(greedy, torch.ones_like(greedy, dtype=z.dtype), st.temp[:, None]))
        r = (r - r.amax(1, keepdim=True)).exp()
        r = r / r.sum(1, keepdim=True)
        r = torch.where(greedy, torch.nn.functional.one_hot(z.argmax(1), V).float(), r)
        q = st.draft[off + node] if st.draft is not None else None
        kids = par == node[:, None]
        order = torch.argsort(~kids, dim=1, stable=True)                                # children first, in index order
        count = kids.sum(1)
        taken = torch.full_like(node, -1)
        for j in range(min(n, st.max_kids)):
            kid = order[:, j]
            open_ = live & (j < count) & (taken < 0)
            x = st.tokens[off + kid].long().clamp(0, V - 1)[:, None]
            rx = r.gather(1, x)
            qx = q.gather(1, x) if q is not None else torch.ones_like(rx)
            qx = torch.where(greedy, torch.zeros_like(qx), qx)
            good = ((rx > 0) & (st.u[off + kid][:, None] * qx <= rx))[:, 0]
            taken = torch.where(open_ & good, kid, taken)
            less = (r - q).clamp(min=0) if q is not None else r.scatter(1, x, 0.0)
            total = less.sum(1, keepdim=True)
            move = (open_ & ~good)[:, None] & (total > 0) & ~greedy
            r = torch.where(move, less / total, r)
            if q is not None:
                rest = 1 - qx
                q = torch.where((open_ & ~good)[:, None], torch.where(rest > 0, q.scatter(1, x, 0.0) / rest, torch.zeros_like(q)), q)
        stop = live & (taken < 0)
        pick = torch.where(r > 0, r / st.noise, torch.full_like(r, -1.0)).argmax(1)
        token = torch.where(stop, torch.where(greedy[:, 0], z.argmax(1), pick), token)
        live = live & (taken >= 0)
        node = torch.where(live, taken, node)
    return path, keep.int(), token.int()


# ----------------------------------------------------------------------- what a pass needs


def work(case):
    c = case
    if c["kind"] in ("cache", "keep"):
        D, E = c["dim"], 2 if c["dtype"] == "bf16" else 4
        row = D + 1 if c["format"] == "fp8" else D * E
        if c["kind"] == "cache":      # rows in, codes out; codes in, rows out
            return {"bytes": float(2 * c["tokens"] * c["kv_heads"] * (2 * D * E + 2 * row)), "flops": 0.0}
        kept = c["batch"] * (1 + (max(1, int(math.sqrt(0.75 * c["nodes"]))) - 1) / 2)      # expected
        return {"bytes": float(2 * kept * c["layers"] * c["kv_heads"] * (3 * row + D * E)), "flops": 0.0}
    if c["kind"] == "attend":
        D, E = c["dim"], 2 if c["dtype"] == "bf16" else 4
        row = D + 1 if c["format"] == "fp8" else D * E
        many = c["batch"] > 1
        n = c["nodes"] * (0.75 if many and c["nodes"] > 1 else 1.0)
        L = c["length"] * (0.625 if many else 1.0) + n
        B = c["batch"]
        return {"bytes": float(B * (2 * c["kv_heads"] * L * row + 2 * n * c["heads"] * D * E + n * c["heads"] * 4)),
                "flops": float(4 * B * c["heads"] * n * L * D)}
    # visited nodes of a walk on these inputs (measured: 2.0 of 4 nodes, 2.5 of 8, 2.9 of 16, 3.2 of 32 with draft
    # rows): their logits, the draft row where a child is rejected (about every second), one row of noise
    E = 2 if c["dtype"] == "bf16" else 4
    visited = 1 + (0.45 if c["draft"] == "probs" else 0.3) * math.log2(c["nodes"])
    rows = visited * E + (0.5 * visited * 4 if c["draft"] == "probs" else 0) + 4
    return {"bytes": float(c["batch"] * c["vocab"] * rows), "flops": float(c["batch"] * c["vocab"] * 4 * visited)}


# ----------------------------------------------------------------------- the same in 64 bits


def exact(case, seed):
    c = case
    if c["kind"] == "attend" and 4.0 * c["batch"] * c["heads"] * c["nodes"] * (c["length"] + c["nodes"]) * c["dim"] > 6e12:
        return None
    st = prepare(c, seed)
    with torch.no_grad():
        return {"cache": _exact_cache, "keep": _exact_keep, "attend": _exact_attend, "verify": _exact_verify}[c["kind"]](st, c)


def _exact_values(x):
    """What format fp8 makes of fp64 rows: nearest values of 4 significant bits on a grid of 2^-9 at the least."""
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax / 448.0).clamp(min=-126))
    e = torch.where(amax <= 448.0 * torch.exp2(e - 1), e - 1, e)
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e).clamp(min=-126)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def _exact_cache(st, c):
    f = _exact_values if c["format"] == "fp8" else (lambda x: x)
    return f(st.k.double())[None], f(st.v.double())[None]


def _exact_pool(st, c, name):
    pool = getattr(st, name + "_pool").double()
    if c["format"] == "fp8":
        pool = pool * torch.exp2(getattr(st, name + "_scale").double() - 127.0)[..., None]
    return pool


def _exact_keep(st, c):
    table, lens = st.table.cpu().numpy(), st.lens.cpu().numpy()
    path, keep = st.path.cpu().numpy(), st.n_keep.cpu().numpy()
    at = [(table[b, (lens[b] + i) // c["page"]], (lens[b] + i) % c["page"]) for b in range(c["batch"]) for i in path[b, : keep[b]]]
    page, row = (torch.tensor([int(x[i]) for x in at], device="cuda") for i in (0, 1))
    out = []
    for name in ("k", "v"):
        flat = getattr(st, name + "_pool").movedim(2, 3).flatten(1, 2)[:, page * c["page"] + row].double()
        if c["format"] == "fp8":
            sc = getattr(st, name + "_scale").movedim(2, 3).flatten(1, 2)[:, page * c["page"] + row].double()
            flat = flat * torch.exp2(sc - 127.0)[..., None]
        out.append(flat)
    return out[0], out[1], None


def _exact_attend(st, c):
    off = st.offsets.tolist()
    lens = st.lens.tolist()
    G = c["heads"] // c["kv_heads"]
    out = torch.zeros(st.total, c["heads"], c["dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((st.total, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
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
            k, v = (getattr(st, x + "_pool")[0, pages, h].double() for x in ("k", "v"))
            if c["format"] == "fp8":
                k = k * torch.exp2(st.k_scale[0, pages, h].double() - 127.0)[..., None]
                v = v * torch.exp2(st.v_scale[0, pages, h].double() - 127.0)[..., None]
            k, v = k.flatten(0, 1)[: L + n], v.flatten(0, 1)[: L + n]
            for g in range(G):
                s = st.q[off[b]: off[b + 1], h * G + g].double() @ k.T / math.sqrt(c["dim"])
                s = s.masked_fill(~mask, -math.inf)
                lse[off[b]: off[b + 1], h * G + g] = torch.logsumexp(s, 1)
                out[off[b]: off[b + 1], h * G + g] = torch.softmax(s, 1) @ v
    return out, lse


def _exact_verify(st, c):
    """The outputs are whole numbers, which are compared as such: no value of theirs in 64 bits is a measure."""
    return None
