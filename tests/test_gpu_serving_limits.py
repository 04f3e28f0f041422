"""Attention over 4-bit caches where its number formats and its tables of pages end."""
import numpy as np
import pytest
import torch

from paper_2609_05228_gb300 import ace

from test_gpu_serving_ops import DT, Step, _int

pytestmark = pytest.mark.gpu

LARGEST = float(torch.finfo(torch.bfloat16).max)


@pytest.mark.parametrize("size", [2.0 ** 120, 2.0 ** 121, 1e38, LARGEST])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("scale", [128 ** -0.5, 4.0])
@pytest.mark.parametrize("nodes", [1, 2, 4, 15, 50])
def test_int4_attention_equal_scores_of_the_largest_q(nodes, scale, sign, size):
    """Rows of one key score alike for q to bf16's largest (scores of 4e9 to 5e12, all of one sign), so the output is the mean of V:
    codes of 1 to 7 and their sums are exact, a weight's rounding is at most 2^-8 of it, the output's too. lse: the score, a sum of
    128 products in fp32, four factors (2^-24 each)."""
    rng = np.random.default_rng(nodes)
    H, G, D, page, length = 1, 4, 128, 16, 333
    total = length + nodes
    v = torch.from_numpy(rng.integers(1, 8, (total, H, D)).astype(np.float32)).bfloat16()
    v[..., ::32] = 7
    kv = ace.AceKvCache(H, D, page, 24, 1, "bf16", "int4")
    key = 7 * 2.0 ** -96
    kv.write(0, torch.full((total, H, D), key, dtype=torch.bfloat16, device="cuda"), v.cuda(), torch.arange(total, device="cuda"))
    q = torch.full((nodes, H * G, D), sign * size, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(nodes, H * G, device="cuda")
    kv.attend(0, q, torch.arange(24, dtype=torch.int32, device="cuda")[None], _int([length]), _int([0, nodes]), out, None, nodes, scale, lse)
    kv.sync()
    sums = v.double().numpy().cumsum(0)
    want = np.stack([sums[length + i] / (length + i + 1) for i in range(nodes)])
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -7 * want).all()
    score = q[0, 0, 0].item() * key * D * scale
    assert (np.abs(lse.double().cpu().numpy() - score) <= 140 * 2.0 ** -24 * abs(score)).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 80), ("f32", 64)])
@pytest.mark.parametrize("p", [60, 110, 118, 121, 124])
@pytest.mark.parametrize("nodes", [1, 2, 4, 5, 20])
def test_int4_attention_large_q_and_small_keys(dtype, D, p, nodes):
    """q of 2^p and K of 2^-p score as both of 1 do. (At p = 124 the sums of products lie among fp32's subnormals: four roundings of 2^-150
    to a row whose largest is 2^(e - 127) are 2^(e - 265) scale of a score, an eighth of the bound's 136 * 2^-24 |q| |k| scale and
    less, as |k| is 2^-122 somewhere.)"""
    s = Step([333, 70], [nodes, 1], 4, 1, D, 16, dtype, seed=p, k_scale=2.0 ** -p)
    s.q = (s.q.double() * 2.0 ** p).to(DT[dtype])
    s.qd = s.q.double().cpu().numpy()
    assert np.isfinite(s.qd).all() and (p < 124 or dtype == "f32" or np.abs(s.qd).max() > 2.0 ** 125)
    s.check(*s.run())


def _longest_share(lens, nodes, kv_heads, ctas, keys, start):
    """Tiles of the longest part of a unit that one block walks: units of start + tiles places on a line that the blocks share alike."""
    tiles = [-(-(n + nodes) // keys) for n in lens]
    line = sum(start + t for t in tiles) * kv_heads
    longest, at = 0, 0
    for t in tiles:
        for _ in range(kv_heads):
            first = at + start
            for c in range(first * ctas // line, min((first + t) * ctas // line + 1, ctas)):
                longest = max(longest, min((c + 1) * line // ctas, first + t) - max(c * line // ctas, first))
            at = first + t
    return longest


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes,G,requests,length,keys,start,batch,per_sm", [
    (1, 8, 20, 16600, 256, 2, 16, 2), (2, 4, 20, 16600, 256, 2, 16, 2), (4, 4, 20, 12500, 96, 3, 32, 2), (5, 4, 10, 8300, 128, 7, 16, 1),
    (10, 8, 10, 8300, 128, 7, 16, 1), (32, 4, 10, 8300, 128, 7, 16, 1), (40, 4, 10, 8300, 128, 7, 16, 1)])
def test_int4_attention_walks_of_many_batches_of_pages(nodes, G, requests, length, keys, start, batch, per_sm, D):
    """Blocks that walk more tiles of a unit than three batches of page-table entries hold: every batch is taken over and filled again.
    Every query row has a key of its own, somewhere in a request's scattered pages, that takes nearly all of its weight, so a tile
    read from another page shows. Bounds as in test_gpu_serving_ops.py (weights and outputs rounded to bf16, 2^-8 each)."""
    H, page, n_pages = 16, 16, 700
    rng = np.random.default_rng(D + nodes)
    lens = [length - int(x) for x in rng.integers(0, 100, requests)]
    ctas = torch.cuda.get_device_properties(0).multi_processor_count * per_sm
    assert _longest_share(lens, nodes, H, ctas, keys, start) > 3 * batch
    kv = ace.AceKvCache(H, D, page, n_pages, 1, "bf16", "int4")
    g = torch.Generator(device="cuda").manual_seed(D + nodes)
    k, v = (torch.randn(n_pages * page, H, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    slots = torch.arange(n_pages * page, device="cuda")
    kv.write(0, k, v, slots)
    kv.read(0, slots, k, v)
    table = torch.randint(0, n_pages, (requests, -(-(length + nodes) // page)), generator=g, device="cuda", dtype=torch.int32)
    q = torch.empty(requests * nodes, H * G, D, dtype=torch.bfloat16, device="cuda")
    at = []
    for b, n in enumerate(lens):
        pos = torch.arange(n + nodes, device="cuda")
        at.append(table[b, pos // page].long() * page + pos % page)
        needle = torch.randint(0, n, (nodes, H * G), generator=g, device="cuda")
        head = torch.arange(H * G, device="cuda") // G
        q[b * nodes: (b + 1) * nodes] = 4 * k[at[b][needle], head]
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    kv.attend(0, q, table, _int(lens), _int(range(0, requests * nodes + 1, nodes)), out, None, nodes, lse=lse)
    kv.sync()
    for b, n in enumerate(lens):
        kd, vd = (x[at[b]].double().movedim(0, 1) for x in (k, v))
        qd = q[b * nodes: (b + 1) * nodes].double().view(nodes, H, G, D).movedim(1, 0).reshape(H, nodes * G, D)
        s = qd @ kd.mT * D ** -0.5
        s_abs = qd.abs().amax((1, 2)) * kd.abs().sum(-1).amax(-1) * D ** -0.5
        hidden = torch.arange(n + nodes, device="cuda")[None, :] > n + torch.arange(nodes, device="cuda").repeat_interleave(G)[:, None]
        s.masked_fill_(hidden, float("-inf"))
        want, wl = torch.softmax(s, -1) @ vd, torch.logsumexp(s, -1)
        got = out[b * nodes: (b + 1) * nodes].double().view(nodes, H, G, D).movedim(1, 0).reshape(H, nodes * G, D)
        ds = ((D + 8) * 2.0 ** -24 * s_abs + 2.0 ** -20)[:, None]
        tol = (2 * ds + (n + nodes + 16) * 2.0 ** -24 + 2.0 ** -8) * vd.abs().amax((1, 2))[:, None]
        assert ((got - want).abs() <= tol[..., None] + 2.0 ** -8 * want.abs()).all(), b
        gl = lse[b * nodes: (b + 1) * nodes].double().view(nodes, H, G).movedim(1, 0).reshape(H, nodes * G)
        assert ((gl - wl).abs() <= ds + (n + nodes + 16) * 2.0 ** -24 + 2.0 ** -22 * wl.abs()).all(), b


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes,G", [(1, 8), (2, 8), (3, 8), (5, 8), (8, 8), (16, 8), (24, 8), (256, 2)])
def test_int4_attention_weights_keep_their_bits(nodes, G, D):
    """V of 7 and -7 in turn: outputs are differences of weights, so what a weight loses shows as it is. A score has one product that is
    not zero. Bounds: that product and the softmax's scale and shift, exp2 (4 * 2^-24 of a score, 2^-21); sums of weights; weights to two
    bf16 terms (2^-16); the output, 2^-8 of it."""
    rng = np.random.default_rng(nodes + D)
    H, page, lens = 2, 16, [1, 2, 3, 10, 60, 300, 0, 1]
    B, need = len(lens), -(-(max(lens) + nodes) // page)
    kv = ace.AceKvCache(H, D, page, B * need, 1, "bf16", "int4")
    table = rng.permutation(B * need).reshape(B, need).astype(np.int32)
    q = np.zeros((B, nodes, H * G, D))
    q[..., 5] = rng.choice([-1, 1], (B, nodes, H * G)) * rng.integers(32, 256, (B, nodes, H * G)) / 128
    k, v = np.zeros((B, max(lens) + nodes, H, D)), np.zeros((B, max(lens) + nodes, H, D))
    k[..., 5], k[..., 7] = rng.integers(-7, 8, k.shape[:-1]) / 8, 7 / 8
    v[:] = 7 * (1 - 2 * (np.arange(v.shape[1]) % 2))[None, :, None, None]
    for b, n in enumerate(lens):
        pos = np.arange(n + nodes)
        slots = torch.from_numpy(table[b, pos // page].astype(np.int64) * page + pos % page).cuda()
        kv.write(0, *(torch.from_numpy(x[b, : n + nodes]).bfloat16().cuda() for x in (k, v)), slots)
    qt = torch.from_numpy(q).bfloat16().cuda().view(B * nodes, H * G, D)
    out, scale = torch.empty_like(qt), 0.7
    kv.attend(0, qt, _int(table), _int(lens), _int(range(0, B * nodes + 1, nodes)), out, None, nodes, scale)
    kv.sync()
    got = out.double().cpu().numpy().reshape(B, nodes, H * G, D)
    for b, n in enumerate(lens):
        kk = np.repeat(k[b, : n + nodes, :, 5], G, 1)
        s = q[b, :, :, 5][:, None, :] * kk[None] * scale                   # [node, position, head]
        s[np.arange(n + nodes)[None, :] > n + np.arange(nodes)[:, None]] = -np.inf
        p = np.exp(s - s.max(1, keepdims=True))
        want = np.einsum("nlh,l->nh", p, v[b, : n + nodes, 0, 0]) / p.sum(1)
        ds = 4 * 2.0 ** -24 * np.abs(np.where(np.isfinite(s), s, 0)).max() + 2.0 ** -21
        tol = 7 * (2 * ds + (n + nodes + 16) * 2.0 ** -24 + 2.0 ** -16) + 2.0 ** -8 * np.abs(want)
        assert (np.abs(got[b] - want[..., None]) <= tol[..., None]).all(), (b, (np.abs(got[b] - want[..., None]) / tol[..., None]).max())


def test_copies_beside_entries_that_do_nothing():
    """Entries with their page as their own source, or outside the pool, are no others to a copy; two that differ for one page are."""
    kv = ace.AceKvCache(2, 64, 16, 8, 2, "bf16", "int4")
    pools = [p.view(torch.uint8) for p in (kv.k_pool, kv.v_pool, kv.k_scale, kv.v_scale)]
    for i, p in enumerate(pools):
        p.copy_(torch.randint(0, 256, tuple(p.shape), generator=torch.Generator().manual_seed(i), dtype=torch.uint8))
    before = [p.clone() for p in pools]
    kv.copy_pages(_int([1, 2, 0, 0]), _int([1, 1, 3, 4]))           # 2 -> 1 beside 1 -> 1; one source twice
    kv.sync()
    kv.copy_pages(_int([9, 7, 6, 5]), _int([5, 5, 7, -1]))          # outside; 7 -> 5 and 6 -> 7: page 7 is a source
    with pytest.raises(ace.AceError) as err:
        kv.sync()
    assert err.value.status == 1
    for p, old in zip(pools, before):
        want = old.clone()
        for s, d in ((2, 1), (0, 3), (0, 4), (7, 5)):
            want[:, d] = old[:, s]
        assert torch.equal(p, want)
