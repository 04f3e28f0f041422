"""The life of the cache's pages on the GPU against a plain account of it, row by row."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2609_05228_gb300 import ace

pytestmark = pytest.mark.gpu

FORMATS = [("int4", "bf16", 128), ("int4", "bf16", 72), ("fp8", "bf16", 64), ("plain", "bf16", 128), ("plain", "f32", 40), ("fp8", "f32", 8)]


def _int(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def _cache(fmt, dtype, D, page, n_pages, layers=2, H=3, seed=0):
    kv = ace.AceKvCache(H, D, page, n_pages, layers, dtype, fmt)
    g = torch.Generator(device="cuda").manual_seed(seed)
    pools = [p.view(torch.uint8) for p in (kv.k_pool, kv.v_pool, kv.k_scale, kv.v_scale) if p is not None]
    pools = [p.view(layers, n_pages, H, page, -1) for p in pools]
    for p in pools:
        p.copy_(torch.randint(0, 256, p.shape, generator=g, device="cuda", dtype=torch.uint8))
    return kv, pools


def _requests(rng, B, page, n_pages, longest, max_pages=None, share=0.5):
    """Tables of requests that share the pages of prompts, and the pages' counts."""
    lens = rng.integers(0, longest + 1, B)
    lens[rng.random(B) < 0.2] //= page
    max_pages = max_pages or -(-longest // page) + 3
    table, refs = np.full((B, max_pages), -1, np.int32), np.zeros(n_pages, np.int32)
    free = list(rng.permutation(n_pages))
    for b in range(B):
        n = -(-int(lens[b]) // page)
        at = 0
        if b and rng.random() < share:
            p = int(rng.integers(0, b))
            at = min(n, -(-int(lens[p]) // page))
            if rng.random() < 0.5:
                at = int(rng.integers(0, at + 1))
            table[b, :at] = table[p, :at]
        for i in range(at, n):
            table[b, i] = free.pop()
        np.add.at(refs, table[b, :n], 1)
    return table, lens.astype(np.int32), refs


def _moved(before, moves):
    """The pools after (from, to, rows) moves, side by side."""
    out = [p.copy() for p in before]
    for p, o in zip(out, before):
        for a, b, rows in moves:
            p[:, b, :, :rows] = o[:, a, :, :rows]
    return out


def _same(pools, want):
    for p, w in zip(pools, want):
        assert (p.cpu().numpy() == w).all()


@pytest.mark.parametrize("B,B_out", [(1, 1), (5, 9), (200, 130), (3, 0), (0, 2)])
@pytest.mark.parametrize("page", [16, 256])
def test_fork(B, B_out, page):
    """Requests kept once, several times, not at all; pages reserved beyond a request's tokens go back."""
    rng = np.random.default_rng(B + page)
    n_pages = 4000
    kv, pools = _cache("int4", "bf16", 64, page, n_pages, 1, 1)
    table, lens, refs = _requests(rng, B, page, n_pages, 300)
    for b in range(0, B, 2):                        # a page reserved, and not in use yet
        n = -(-int(lens[b]) // page)
        if n < table.shape[1]:
            table[b, n] = int(np.nonzero(refs == 0)[0][0])
            refs[table[b, n]] = 1
    parents = rng.integers(-1, B, B_out) if B else np.full(B_out, -1)
    want = S.fork(table, lens, parents, refs, page)
    t, r = _int(table), _int(refs)
    nt, nl = torch.full((B_out, table.shape[1]), 99, dtype=torch.int32, device="cuda"), torch.full((B_out,), 99, dtype=torch.int32, device="cuda")
    kv.fork(t, _int(lens), _int(parents), r, nt, nl)
    kv.sync()
    for got, w in zip((nt, nl, r), want):
        assert (got.cpu().numpy() == w).all()
    assert (t.cpu().numpy() == table).all()
    assert (r.cpu().numpy() == np.bincount(want[0][want[0] >= 0], minlength=n_pages)).all()


@pytest.mark.parametrize("fmt,dtype,D", FORMATS)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("most", [1, 50])
def test_reserve(fmt, dtype, D, page, most):
    """Fresh pages and copies of shared ones, with their rows alone and in all layers, as one request after another gets them."""
    rng = np.random.default_rng(D + page + most)
    n_pages, B = 400, 40
    kv, pools = _cache(fmt, dtype, D, page, n_pages)
    table, lens, refs = _requests(rng, B, page, n_pages, 100)
    grow = rng.integers(0, most + 1, B)
    before = [p.cpu().numpy() for p in pools]
    want_t, want_r, missing, moves = S.reserve(table, lens, grow, refs, page)
    assert missing == 0 and len(moves) > 0
    t, r, m = _int(table), _int(refs), _int([77])
    for again in range(2):                          # the second time there is nothing to do
        kv.reserve(t, _int(lens), _int(grow), r, m)
        kv.sync()
        assert (t.cpu().numpy() == want_t).all() and (r.cpu().numpy() == want_r).all() and m.item() == 0
        _same(pools, _moved(before, moves))


@pytest.mark.parametrize("B", [1, 33, 1025, 8192])
def test_reserve_batches_and_large_pools(B):
    """Many requests, rows of thousands of pages, a pool of several rounds of the search for free pages."""
    rng = np.random.default_rng(B)
    n_pages, page = 70000, 16
    kv, pools = _cache("fp8", "bf16", 8, page, n_pages, 1, 1)
    refs = (rng.random(n_pages) < 0.6).astype(np.int32)
    taken = np.nonzero(refs)[0]
    max_pages = 9000 if B == 1 else 5
    lens = rng.integers(0, 33, B).astype(np.int32)
    table = np.full((B, max_pages), -1, np.int32)
    at = 0
    for b in range(B):
        n = -(-int(lens[b]) // page)
        table[b, :n] = taken[at: at + n]
        at += n
    grow = rng.integers(0, 40, B)
    if B == 1:
        lens[0], table[0, 0], grow[0] = 5, taken[0], 140000
    want_t, want_r, missing, moves = S.reserve(table, lens, grow, refs, page)
    t, r, m = _int(table), _int(refs), _int([77])
    kv.reserve(t, _int(lens), _int(grow), r, m)
    kv.sync()
    assert missing == 0 == m.item()
    assert (t.cpu().numpy() == want_t).all() and (r.cpu().numpy() == want_r).all()


def test_reserve_says_what_is_missing_and_changes_nothing():
    rng = np.random.default_rng(3)
    page, n_pages = 16, 40
    kv, pools = _cache("int4", "bf16", 64, page, n_pages)
    table, lens, refs = _requests(rng, 6, page, n_pages, 60)
    before = [p.cpu().numpy() for p in pools]
    table = np.concatenate([table, np.full((6, 60), -1, np.int32)], 1)
    grow = np.array([1, 300, 0, 400, 5, 100])
    want = S.reserve(table, lens, grow, refs, page)
    assert want[2] > 0
    t, r, m = _int(table), _int(refs), _int([77])
    kv.reserve(t, _int(lens), _int(grow), r, m)
    kv.sync()
    assert m.item() == want[2]
    assert (t.cpu().numpy() == table).all() and (r.cpu().numpy() == refs).all()
    _same(pools, before)
    # exactly as many as there are
    less = int((refs == 0).sum())
    grow = np.array([0, 0, 0, 0, 0, 0])
    grow[0] = less * page - (page - int(lens[0]) % page) % page - (page if refs[table[0, int(lens[0]) // page]] > 1 and lens[0] % page else 0)
    grow[0] += (page - int(lens[0]) % page) % page
    want = S.reserve(np.concatenate([table, np.full((6, 60), -1, np.int32)], 1), lens, grow, refs, page)
    t = _int(np.concatenate([table, np.full((6, 60), -1, np.int32)], 1))
    kv.reserve(t, _int(lens), _int(grow), r, m)
    kv.sync()
    assert m.item() == want[2] and (t.cpu().numpy() == want[0]).all() and (r.cpu().numpy() == want[1]).all()


def test_reserve_and_fork_leave_out_what_is_wrong():
    page, n_pages = 16, 20
    kv, pools = _cache("int4", "bf16", 64, page, n_pages)
    before = [p.cpu().numpy() for p in pools]
    table = np.array([[0, 1, -1], [2, -1, -1], [99, -1, -1], [3, 4, 5], [6, -1, -1]], np.int32)
    lens = np.array([20, -1, 5, 47, 3], np.int32)
    grow = np.array([-2, 4, 4, 2, 20], np.int32)        # backwards; no length; no such page; past its row; fine
    refs = np.zeros(n_pages, np.int32)
    refs[:7] = 1
    t, r, m = _int(table), _int(refs), _int([77])
    kv.reserve(t, _int(lens), _int(grow), r, m)
    with pytest.raises(ace.AceError) as err:
        kv.sync()
    assert err.value.status == 1
    kv.sync()
    table[4, 1], refs[7] = 7, 1
    assert (t.cpu().numpy() == table).all() and (r.cpu().numpy() == refs).all() and m.item() == 0
    _same(pools, before)
    nt, nl = _int(np.zeros((4, 3))), _int(np.zeros(4))
    kv.fork(t, _int([20, -1, 5, 50, 3]), _int([0, 1, 5, 3]), r, nt, nl)
    with pytest.raises(ace.AceError):
        kv.sync()
    assert nt.tolist() == [[0, 1, -1], [-1, -1, -1], [-1, -1, -1], [-1, -1, -1]] and nl.tolist() == [20, 0, 0, 0]
    assert r.tolist() == [1, 1] + [0] * 18


@pytest.mark.parametrize("page", [16, 128])
def test_release(page):
    rng = np.random.default_rng(page)
    n_pages, B = 900, 60
    kv, pools = _cache("plain", "bf16", 8, page, n_pages, 1, 1)
    table, lens, refs = _requests(rng, B, page, n_pages, 200)
    ended = (rng.random(B) < 0.5).astype(np.int32) * 5
    t, l, r = _int(table), _int(lens), _int(refs)
    kv.release(t, l, _int(ended), r)
    kv.sync()
    table[ended != 0], lens[ended != 0] = -1, 0
    assert (t.cpu().numpy() == table).all() and (l.cpu().numpy() == lens).all()
    assert (r.cpu().numpy() == np.bincount(table[table >= 0], minlength=n_pages)).all()
    kv.release(t, l, _int(np.ones(B)), r)
    kv.sync()
    assert r.count_nonzero() == 0


@pytest.mark.parametrize("fmt,dtype,D", FORMATS)
@pytest.mark.parametrize("page,n_pages,B", [(16, 700, 50), (64, 64, 6), (16, 40000, 30)])
def test_compact(fmt, dtype, D, page, n_pages, B):
    rng = np.random.default_rng(D + n_pages)
    kv, pools = _cache(fmt, dtype, D, page, n_pages)
    table, lens, refs = _requests(rng, B, page, n_pages, 150)
    before = [p.cpu().numpy() for p in pools]
    want_t, want_r, n, at, moves = S.compact(table, refs)
    t, r, u, where = _int(table), _int(refs), _int([99]), _int(np.full(n_pages, 99))
    kv.compact(t, r, u, where)
    kv.sync()
    assert (t.cpu().numpy() == want_t).all() and (r.cpu().numpy() == want_r).all() and u.item() == n and (where.cpu().numpy() == at).all()
    _same(pools, _moved(before, [(a, b, page) for a, b in moves]))
    kv.compact(t, r, u)                             # nothing is left to move
    kv.sync()
    assert (t.cpu().numpy() == want_t).all() and u.item() == n
    # no requests: places alone; entries of free pages are reported
    kv.compact(t[:0], r, u, where)
    kv.sync()
    assert where.tolist() == [x if x < n else -1 for x in range(n_pages)]
    wrong = _int([[0, n, n_pages + 3]])
    kv.compact(wrong, r, u)
    with pytest.raises(ace.AceError):
        kv.sync()
    assert wrong.tolist() == [[0, -1, -1]]


@pytest.mark.parametrize("fmt,dtype,D", FORMATS)
def test_copy_pages(fmt, dtype, D):
    rng = np.random.default_rng(D)
    n_pages = 3000
    kv, pools = _cache(fmt, dtype, D, 16, n_pages)
    order = rng.permutation(n_pages)
    src, dst = order[:1100], order[1500:2600].copy()
    src[5] = src[6]                                 # one page to two places
    before = [p.cpu().numpy() for p in pools]
    kv.copy_pages(_int(src), _int(dst))
    kv.sync()
    _same(pools, _moved(before, [(a, b, 16) for a, b in zip(src, dst)]))
    before = [p.cpu().numpy() for p in pools]
    # a page to itself is nothing; two to one place, a place that is copied from, pages outside are left out and reported
    kv.copy_pages(_int([1, 7]), _int([1, 8]))
    kv.sync()
    kv.copy_pages(_int([10, 11, 12, 13, -1, 15, 16]), _int([20, 20, 13, 21, 22, n_pages, 23]))
    with pytest.raises(ace.AceError) as err:
        kv.sync()
    assert err.value.status == 1
    _same(pools, _moved(before, [(7, 8, 16), (13, 21, 16), (16, 23, 16)]))
    kv.copy_pages(_int([]), _int([]))
    kv.copy_pages(_int([12]), _int([13]))           # nothing of the calls before is remembered
    kv.sync()


def test_pages_past_2_32_bytes():
    """Moves to and from pages behind 2^32 bytes of a pool."""
    kv = ace.AceKvCache(8, 128, 256, 33000, 1, "bf16", "int4")
    last = 32999
    kv.k_pool[0, last], kv.v_scale[0, last], kv.v_pool[0, 1] = 37, 2.5, 11
    kv.copy_pages(_int([last, 1]), _int([3, last - 1]))
    kv.sync()
    assert (kv.k_pool[0, 3] == 37).all() and (kv.v_scale[0, 3] == 2.5).all() and (kv.v_pool[0, last - 1] == 11).all()
    assert kv.k_pool[0, 4].count_nonzero() == 0 and kv.k_pool[0, 2].count_nonzero() == 0
    refs = torch.zeros(33000, dtype=torch.int32, device="cuda")
    refs[last] = 2
    table, used = _int([[last], [last]]), _int([0])
    kv.compact(table, refs, used)
    kv.sync()
    assert table.tolist() == [[0], [0]] and used.item() == 1 and refs[0] == 2 and (kv.k_pool[0, 0] == 37).all()


def test_empty_calls_and_requests_that_do_not_grow():
    """No requests, no pages, and requests with a grow of 0 whose lengths and rows are not looked at."""
    kv, pools = _cache("int4", "bf16", 64, 16, 10)
    before = [p.cpu().numpy() for p in pools]
    refs = np.zeros(10, np.int32)
    refs[[2, 3]] = 1
    r, none, m, empty = _int(refs), _int(np.zeros((0, 3))), _int([77]), _int([])
    kv.reserve(none, empty, empty, r, m)
    assert m.item() == 0
    kv.release(none, empty, empty, r)
    kv.fork(none, empty, empty, r, none.clone(), empty.clone())
    kv.copy_pages(empty, empty)
    kv.sync()
    assert (r.cpu().numpy() == refs).all()
    table = _int([[99, -7, 5], [2, -1, -1], [3, 3, 3]])
    kv.reserve(table, _int([-3, 4, 1000]), _int([0, 20, 0]), r, m)
    kv.sync()
    assert table.tolist() == [[99, -7, 5], [2, 0, -1], [3, 3, 3]] and m.item() == 0
    refs[0] = 1
    assert (r.cpu().numpy() == refs).all()
    _same(pools, before)
    kv.compact(none, r, m, new := _int(np.zeros(10)))
    kv.sync()
    assert m.item() == 3 and new.tolist() == [0, -1, 2, 1] + [-1] * 6
    assert r.tolist() == [1, 1, 1] + [0] * 7
    _same(pools, _moved(before, [(3, 1, 16)]))


def test_graphs_of_one_cache_replayed_in_turn():
    """Two captured graphs share a cache's workspace: each leaves what the other's plan needs as it found it."""
    page, n_pages = 16, 12
    kv, pools = _cache("int4", "bf16", 64, page, n_pages)
    table, refs = np.array([[0, -1, -1, -1], [0, -1, -1, -1]], np.int32), np.zeros(n_pages, np.int32)
    refs[0] = 2
    lens, grow = np.array([5, 9], np.int32), np.array([20, 1], np.int32)
    t, l, g, r, m = _int(table), _int(lens), _int(grow), _int(refs), _int([77])
    src, dst = _int([0, 0]), _int([11, 10])
    grows, copies = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(grows):
        kv.reserve(t, l, g, r, m)
    with torch.cuda.graph(copies):
        kv.copy_pages(src, dst)
    before = [p.cpu().numpy() for p in pools]
    for _ in range(3):
        t.copy_(_int(table)), r.copy_(_int(refs))
        for p, b in zip(pools, before):
            p.copy_(torch.from_numpy(b))
        copies.replay()
        grows.replay()
        copies.replay()
        kv.sync()
        want = S.reserve(table, lens, grow, refs, page)
        assert (t.cpu().numpy() == want[0]).all() and (r.cpu().numpy() == want[1]).all() and m.item() == 0
        fresh = int(t[0, 0])
        assert fresh != 0 and int(t[1, 0]) == 0
        _same(pools, _moved(before, [(0, 11, page), (0, 10, page), (0, fresh, 5)]))


def test_a_beam_search_keeps_its_books():
    """Steps of forks and reserves in one captured graph, against the account; the rows that a beam wrote are the rows that it reads."""
    rng = np.random.default_rng(12)
    page, n_pages, B, H, D = 16, 64, 8, 2, 64
    kv = ace.AceKvCache(H, D, page, n_pages, 1, "bf16", "plain")
    table, lens, refs = np.full((B, 8), -1, np.int32), np.zeros(B, np.int32), np.zeros(n_pages, np.int32)
    t, l, r, m = _int(table), _int(lens), _int(refs), _int([0])
    nt, nl = torch.empty_like(t), torch.empty_like(l)
    parents, grow = _int(np.arange(B)), _int(np.ones(B))
    rows = torch.zeros(B, H, D, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(B, dtype=torch.int64, device="cuda")

    def step():
        kv.fork(t, l, parents, r, nt, nl)
        kv.reserve(nt, nl, grow, r, m)
        t.copy_(nt)
        slots.copy_(t.gather(1, (nl // page).long()[:, None])[:, 0].long() * page + nl % page)
        kv.write(0, rows, rows, slots)
        l.copy_(nl + 1)
    step()
    kv.sync()
    table, lens, refs = S.fork(table, lens, np.arange(B), refs, page)
    table, refs, _, _ = S.reserve(table, lens, np.ones(B, int), refs, page)
    lens = lens + 1
    said = [[0] for _ in range(B)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(1, 60):
        p = rng.integers(0, B, B)
        parents.copy_(_int(p))
        rows.copy_((torch.arange(B, device="cuda") + 8 * i).view(B, 1, 1).expand(B, H, D))
        g.replay()
        torch.cuda.synchronize()
        table, lens, refs = S.fork(table, lens, p, refs, page)
        table, refs, missing, _ = S.reserve(table, lens, np.ones(B, int), refs, page)
        lens = lens + 1
        said = [said[x] + [b + 8 * i] for b, x in enumerate(p)]
        assert missing == 0 == m.item()
        assert (t.cpu().numpy() == table).all() and (l.cpu().numpy() == lens).all() and (r.cpu().numpy() == refs).all()
    kv.sync()
    for b in range(B):
        pos = np.arange(lens[b])
        at = torch.from_numpy(table[b, pos // page].astype(np.int64) * page + pos % page).cuda()
        k, v = torch.empty(len(pos), H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(len(pos), H, D, dtype=torch.bfloat16, device="cuda")
        kv.read(0, at, k, v)
        # bf16 holds whole numbers up to 256 exactly
        want = torch.tensor(said[b], dtype=torch.float32).bfloat16()
        assert torch.equal(k[:, 1, 5].cpu(), want) and torch.equal(v[:, 0, 0].cpu(), want)


# ----------------------------------------------------------------------- all of it together, as the example's decoder runs it


@pytest.fixture(scope="module")
def example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decode.py")
    spec = importlib.util.spec_from_file_location("speculative_decode", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _alone(decoder):
    """Skipping by ratio looks at the whole batch, so that a token's experts would depend on its company."""
    for layer in decoder.moe:
        layer.forward = lambda x, y, T, mode, value, plain=layer.forward: plain(x, y, T, "threshold", 0.15)
    return decoder


def test_speculation_over_a_4_bit_cache_is_plain_decoding(example):
    first = torch.arange(4, device="cuda") * 7
    torch.manual_seed(1)
    plain, steps = example.generate(_alone(example.Decoder("f32", "int4")), first, 40, 0.0, drafted=False)
    torch.manual_seed(2)
    d = _alone(example.Decoder("f32", "int4"))
    fast, fewer = example.generate(d, first, 40, 0.0)
    assert steps == 40 and fewer <= steps
    assert [o[:40] for o in fast] == [o[:40] for o in plain]
    # the pages in use are those that the requests' rows name
    named = d.pages[d.pages >= 0]
    assert torch.equal(torch.bincount(named, minlength=d.refs.shape[0]).int(), d.refs) and d.refs.max() == 1
    assert int(named.numel()) >= int(((d.lens + example.PAGE - 1) // example.PAGE).sum())


@pytest.mark.parametrize("dtype,fmt", [("bf16", "int4"), ("f32", "plain")])
def test_forked_requests_go_on_as_the_one_that_they_come_from(example, dtype, fmt):
    """One request's tokens are run; it is forked into all places, and its copies, which share its pages until they write, have the
    logits that requests with pages of their own have."""
    d, own = (_alone(example.Decoder(dtype, fmt, seed=5)) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(9)
    chain = torch.tensor([-1], dtype=torch.int32, device="cuda")

    def step(decoder, tokens):
        B = decoder.lens.shape[0]
        logits = decoder.forward(tokens, chain.repeat(B), torch.arange(B + 1, dtype=torch.int32, device="cuda"), 1)
        path = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
        decoder.keep(path, torch.ones(B, dtype=torch.int32, device="cuda"))
        return logits

    for i in range(37):                             # two pages and a part of the third
        tokens = torch.randint(0, example.VOCAB, (4,), generator=g, device="cuda").int()
        step(d, tokens)
        step(own, tokens[2].repeat(4))
    d.reorder(_int([2, 2, 2, 2]))
    assert d.refs.max() == 4 and int((d.refs > 0).sum()) == 3
    for i in range(20):
        tokens = torch.randint(0, example.VOCAB, (4,), generator=g, device="cuda").int()
        assert torch.equal(step(d, tokens), step(own, tokens))
    assert torch.equal(torch.bincount(d.pages[d.pages >= 0], minlength=d.refs.shape[0]).int(), d.refs) and int((d.refs == 4).sum()) == 2
    d.reorder(_int([-1, -1, -1, -1]))
    assert d.refs.count_nonzero() == 0 and d.lens.count_nonzero() == 0
    d.kv.sync()
