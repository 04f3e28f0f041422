"""The speculative decode step's operators where their number formats end: small weights, values of very different size,
temperatures near zero, pages that do not exist."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import decode_oracle as R
from paper_2609_05228_gb300 import ace

from test_gpu_decode_ops import DT, Step, _check_verify, _rows, _run_verify, _verify_case

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------- attention


@pytest.mark.parametrize("fmt", ["fp8", "plain"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [5, 8, 16, 24, 32, 40, 128])
@pytest.mark.parametrize("e", [14, 16, 18, 20, 22])
def test_attention_sink_of_no_value_beside_small_weights(fmt, D, rows, e):
    """A first key takes nearly all of the weight and has V = 0; 8191 keys of 2^-e of it (up to 2^(7/8) more) make the output.
    As many requests as two an SM, so that a CTA meets the sink and all that follows; they share their pages.

    Relative bounds: the weight's rounding (fp8: 2^-12, in fp16's subnormals 2^-25 of a weight times 2^3 or more; plain: 2^-9),
    the sums of L positive terms, the weight's own (exp2 and a score's rounding of up to 22 units), the output's."""
    L, B, page = 8192, 304, 64
    rng = np.random.default_rng(e)
    x = rng.integers(0, 8, L) / 8.0
    x[0] = e
    k = torch.zeros(L, 1, D)
    k[:, 0, 0] = torch.from_numpy(x)
    vd = 1 + rng.integers(0, 8, (L, D)) / 8.0
    vd[0] = 0
    kv = ace.AceKvCache(1, D, page, L // page, 1, "bf16", fmt)
    kv.write(0, k.bfloat16().cuda(), torch.from_numpy(vd)[:, None].bfloat16().cuda(), torch.arange(L, device="cuda"))
    q = torch.zeros(B, rows, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    out = torch.empty_like(q)
    table = torch.arange(L // page, dtype=torch.int32, device="cuda").repeat(B, 1)
    lens = torch.full((B,), L - 1, dtype=torch.int32, device="cuda")
    kv.attend(0, q, table, lens, torch.arange(B + 1, dtype=torch.int32, device="cuda"), out, scale=float(np.log(2.0)))
    kv.sync()
    p = 2.0 ** (x - e)
    want = (p @ vd) / p.sum()
    rel = (2.0 ** -12 + 2.0 ** (e - 28) if fmt == "fp8" else 2.0 ** -9) + (L + 16) * 2.0 ** -24 + 2 * 22 * 2.0 ** -22 + 2.0 ** -8
    err = np.abs(out.double().cpu().numpy() - want) / want
    assert err.max() <= rel, (err.max(), rel)


@pytest.mark.parametrize("fmt,dtype,D", [("plain", "f32", 64), ("fp8", "f32", 40), ("plain", "bf16", 80), ("fp8", "bf16", 80), ("plain", "bf16", 128),
                                         ("fp8", "bf16", 128)])
@pytest.mark.parametrize("nodes", [3, 40])
def test_attention_nan_of_no_weight_reaches_rows_that_see_it(fmt, dtype, D, nodes):
    """A drafted V of NaN whose weight is below fp32's least is NaN in the rows that see it, as in the prefix, and in no other."""
    length, H, G, page = 40, 2, 2, 16
    dt = DT[dtype]
    total = length + nodes
    kv = ace.AceKvCache(H, D, page, 8, 1, dtype, fmt)
    k, v = torch.zeros(total, H, D, dtype=dt, device="cuda"), torch.ones(total, H, D, dtype=dt, device="cuda")
    k[length + 1, :, 0] = -448.0                    # scores of -13440
    v[length + 1, :, 2] = float("nan")
    kv.write(0, k, v, torch.arange(total, device="cuda"))
    q = torch.zeros(nodes, H * G, D, dtype=dt, device="cuda")
    q[..., 0] = 30.0
    out = torch.empty_like(q)
    kv.attend(0, q, torch.arange(8, dtype=torch.int32, device="cuda")[None], torch.tensor([length], dtype=torch.int32, device="cuda"),
              torch.tensor([0, nodes], dtype=torch.int32, device="cuda"), out, None, nodes, 1.0)
    kv.sync()
    want = torch.ones_like(out)
    want[1:, :, 2] = float("nan")
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert (torch.nan_to_num(out, 1.0).float() - 1).abs().max() <= 2.0 ** -8


def _check_by_row(s, out, ls):
    """The bounds of Step.check with each row's own positions: a value that a row does not see has no part in its bound. (L
    2^-25: weights down to fp16's least, 2^-24 of a factor of one or more for the largest.)"""
    out, scale = out.double().cpu().numpy(), s.D ** -0.5
    w = 0.0 if s.dtype == "f32" else 2.0 ** -9 if s.fmt == "plain" else 2.0 ** -12
    for b, n in enumerate(s.sizes):
        if not n:
            continue
        G = s.qd.shape[1] // s.k[b].shape[1]
        L = s.lens[b] + n
        for i in range(n):
            at = np.concatenate([np.arange(s.lens[b]), s.lens[b] + np.nonzero(s.sees[b][i])[0]])
            row = s.off[b] + i
            if not len(at):
                assert (out[row] == 0).all() and torch.isneginf(ls[row]).all()
                continue
            q = s.qd[row]
            k, v = np.repeat(s.k[b][at], G, 1), np.repeat(s.v[b][at], G, 1)
            x = np.einsum("hd,lhd->hl", q, k) * scale
            top = x.max(1)
            p = np.exp(x - top[:, None])
            want = np.einsum("hl,lhd->hd", p, v) / p.sum(1)[:, None]
            lse = top + np.log(p.sum(1))
            ds = (s.D + 8) * 2.0 ** -24 * np.einsum("hd,lhd->hl", np.abs(q), np.abs(k)).max(1) * scale + 2.0 ** -20
            tol = (2 * ds + (L + 16) * 2.0 ** -24 + L * 2.0 ** -25 + w) * np.abs(v).max((0, 2))
            o_tol = tol[:, None] + (0 if s.dtype == "f32" else 2.0 ** -8) * np.abs(want)
            err = np.abs(out[row] - want)
            assert (err <= o_tol).all(), (b, i, (err / o_tol).max())
            g = ls[row].double().cpu().numpy()
            assert (np.abs(g - lse) <= ds + (L + 16) * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse)).all(), (b, i)


def _scale_value(s, b, node, factor):
    """The V row of a node is `factor` times a new random one."""
    v, _ = _rows(s.rng, (1,) + s.v[b].shape[1:], s.dtype, factor)
    k = torch.from_numpy(s.k[b][s.lens[b] + node][None]).to(v.dtype).cuda()       # (exact: bf16 and fp32 hold a code's value)
    pos = s.lens[b] + node
    slot = int(s.table[b, pos // s.page]) * s.page + pos % s.page
    s.kv.write(s.layer, k, v, torch.tensor([slot], device="cuda"))
    vd = v.double().cpu().numpy()
    s.v[b][pos] = (R.quantise_rows(vd)[2] if s.fmt == "fp8" else vd)[0]


@pytest.mark.parametrize("fmt,dtype,D", [("fp8", "bf16", 128), ("fp8", "bf16", 64), ("plain", "bf16", 128), ("fp8", "f32", 40)])
@pytest.mark.parametrize("Hq,H,n", [(2, 1, 3), (4, 2, 4), (8, 2, 4), (4, 2, 16), (8, 2, 16), (4, 2, 60), (8, 2, 60), (3, 3, 200)])
@pytest.mark.parametrize("power", [3, 7, 12, 20, 60, 110])
@pytest.mark.parametrize("length", [0, 5, 300])
def test_attention_values_of_any_size_that_others_see(fmt, dtype, D, Hq, H, n, power, length):
    """A drafted node whose finite V is 2^power times the others' is nothing to the nodes that do not see it, and what it is to
    those that do: the last node of a chain, a node that none sees, one that two of three see, one before an empty prefix."""
    s = Step([length, 140, 30], [n, n, max(1, n // 2)], Hq, H, D, 16, fmt, dtype, seed=n + power)
    _scale_value(s, 0, n - 1, 2.0 ** power)                     # seen by itself alone
    _scale_value(s, 1, n // 2, 2.0 ** power)
    s.sees[1][:, n // 2] = False                                # by none
    _scale_value(s, 2, 0, 2.0 ** power)
    s.sees[2][::3, 0] = False                                   # node 0 is not seen by every third, not by itself
    out, ls = s.run()
    _check_by_row(s, out, ls)


@pytest.mark.parametrize("fmt,D", [("fp8", 128), ("fp8", 64)])
@pytest.mark.parametrize("Hq,H,n", [(4, 2, 4), (8, 2, 8), (8, 2, 16), (8, 2, 60), (2, 2, 250)])
def test_attention_values_of_many_sizes_in_trees(fmt, D, Hq, H, n):
    """Every node's V of another size, any masks, rows that see nothing, lengths that are cut over many CTAs."""
    s = Step([0, 9000, 127, 128], [n, n, n, max(1, n // 3)], Hq, H, D, 32, fmt, "bf16", seed=n)
    s.random_masks(0.3, empty=(1,))
    for b, size in enumerate(s.sizes):
        for i in range(0, size, 1 + size // 40):
            _scale_value(s, b, i, 2.0 ** float(s.rng.integers(-60, 61)))
    first = s.run()
    _check_by_row(s, *first)
    for q in (s.q, s.q.transpose(0, 1).contiguous().transpose(0, 1)):
        again = s.run(q=q)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("fmt,dtype,D", [("fp8", "bf16", 128), ("plain", "bf16", 128), ("fp8", "bf16", 64), ("plain", "bf16", 64),
                                         ("plain", "f32", 40), ("fp8", "bf16", 80)])
@pytest.mark.parametrize("Hq,H,n", [(4, 2, 1), (8, 2, 8), (4, 2, 30), (6, 2, 40), (4, 2, 100)])
@pytest.mark.parametrize("page,length,gone", [(16, 700, (0, 11, 12)), (16, 700, (42, 43)), (64, 5000, (3, 40)), (128, 900, (2,)), (256, 900, (0, 3)), (16, 20, (0, 1))])
def test_attention_has_zeros_for_pages_that_do_not_exist(fmt, dtype, D, Hq, H, n, page, length, gone):
    """Positions whose table entry names no page of the pool have K and V of zeros, in the prefix, among the nodes, a whole tile's;
    the other requests' results keep their bits, and the error is reported."""
    s = Step([length, 333], [n, n], Hq, H, D, page, fmt, dtype, seed=page + n)
    s.random_masks(0.6)
    good, good_ls = s.run()
    for i, g in enumerate(gone):
        s.table[0, g] = (-1, 1 << 20, -(1 << 31))[i % 3]
    out = torch.full_like(good, 7.0)
    ls = torch.full_like(good_ls, 7.0)
    args = [torch.from_numpy(np.asarray(a, np.int32)).cuda() for a in (s.table, s.lens, s.off)]
    s.kv.attend(0, s.q, *args, out, s.mask(), s.n_max, None, ls)
    with pytest.raises(ace.AceError) as err:
        s.kv.sync()
    assert err.value.status == 1
    assert torch.equal(out[n:], good[n:]) and torch.equal(ls[n:], good_ls[n:])
    pos = np.arange(length + n)
    s.k[0][np.isin(pos // page, gone)] = 0
    s.v[0][np.isin(pos // page, gone)] = 0
    _check_by_row(s, out, ls)


# ----------------------------------------------------------------------- verification


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("sizes,V", [([6, 1, 4, 8, 5], 9000), ([12, 9, 3], 1500), ([7] * 40, 700)])
@pytest.mark.parametrize("temp", [1e-3, 1e-4, 1e-5, 1e-6, 1e-7, 1e-8, 1e-20, 1e-30, 1e-37, 1e-40, 1e-45])
def test_verify_temperatures_near_zero(dtype, draft, sizes, V, temp):
    """The softmax of any positive temperature, down to fp32's least, for trees with and without a node a CTA."""
    rng = np.random.default_rng(V + int(-np.log10(temp)))
    c = _verify_case(rng, sizes, V, dtype, draft, temps=np.full(len(sizes), temp), sharp=6.0)
    # half of the nodes draft the likely token, or the second
    z = c["logits"].double().cpu().numpy()
    for b, ps in enumerate(c["parents"]):
        for i in range(1, len(ps)):
            if rng.random() < 0.5:
                c["tokens"][c["off"][b] + i] = np.argsort(-z[c["off"][b] + ps[i]], kind="stable")[rng.integers(0, 2)]
    n_max = max(sizes)
    _check_verify(c, _run_verify(c, n_max), n_max)


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("shift", [1e6, -3e6, 1e7, 1e8, -1e9, 1e30])
def test_verify_logits_far_from_zero(draft, shift):
    """Logits that share a large offset: their differences alone count."""
    rng = np.random.default_rng(int(abs(shift) % 1000003))
    c = _verify_case(rng, [6, 4, 8, 5] * 8, 3000, "f32", draft, temps=np.ones(32))
    c["logits"] += shift
    _check_verify(c, _run_verify(c, 8), 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("V", [20000, 20003])
@pytest.mark.parametrize("n_max", [8, 9])
def test_verify_trees_of_a_node_a_cta_and_one_more(dtype, draft, V, n_max):
    """A few requests whose largest tree has as many nodes as a cluster CTAs (all rows' statistics at once), or one more: absent
    requests, mixed sizes and temperatures; a NaN or a row of -inf where no walk comes is nothing to the others."""
    rng = np.random.default_rng(V + n_max)
    sizes = [2, n_max, 1, 0, 5, n_max, 7, 8]
    c = _verify_case(rng, sizes, V, dtype, draft, temps=[1.0, 0.8, 1.0, 1.0, 0.0, 1.2, 0.0, 1.0])
    c["parents"][7] = [-1, 0, 1, 2, 3, 4, 0, 0]
    o = c["off"][7]
    c["tokens"][o + 1] = -1                         # never accepted, so nodes 2 to 5 are not visited
    c["logits"][o + 2, 11] = float("nan")
    c["logits"][o + 4] = float("-inf")
    c["logits"][c["off"][0], 17] = float("nan")     # a root: the walk ends there
    _check_verify(c, _run_verify(c, n_max), n_max)


# ----------------------------------------------------------------------- masks


def test_tree_mask_leaves_out_offsets_outside_its_rows():
    """Offsets below zero, past the rows, decreasing, or of too many nodes: no row is written for them."""
    for off in ([0, 3, 9], [-2, 3, 5], [0, 3, 1 << 30], [-(1 << 31), 3, 5], [0, 3, -(1 << 31)], [0, 3, 2], [6, 3, 5]):
        mask = torch.full((64, 1), -1, dtype=torch.int64, device="cuda")
        depth = torch.full((64,), -1, dtype=torch.int32, device="cuda")
        parents = torch.full((64,), -1, dtype=torch.int32, device="cuda")
        parents[1:] = torch.arange(63, device="cuda")
        rows = slice(16, 22)                        # six rows of the 64
        ace.ace_tree_mask(parents[:6], torch.tensor(off, dtype=torch.int32, device="cuda"), 2, 4, mask[rows], depth[rows])
        torch.cuda.synchronize()
        want_mask, want_depth = np.full(64, -1), np.full(64, -1)
        for o0, o1 in zip(off, off[1:]):
            if 0 <= o0 < o1 <= 6 and o1 - o0 <= 4:
                ps = [int(p) for p in parents[o0:o1].tolist()]
                sees = R.ancestors(ps)
                want_mask[16 + o0: 16 + o1] = R.mask_words(sees, 1).view(np.int64)[:, 0]
                want_depth[16 + o0: 16 + o1] = sees.sum(1) - 1
        assert (mask[:, 0].cpu().numpy() == want_mask).all() and (depth.cpu().numpy() == want_depth).all(), off


# ----------------------------------------------------------------------- streams


def test_calls_follow_the_current_stream():
    """A step inside `with torch.cuda.stream(...)`, behind a long kernel there that makes its inputs, and captured in a graph."""
    side = torch.cuda.Stream()
    s = Step([700, 20], [6, 3], 8, 2, 128, 64, "fp8", "bf16", seed=12)
    want, _ = s.run(chain=True)
    args = [torch.from_numpy(np.asarray(a, np.int32)).cuda() for a in (s.table, s.lens, s.off)]
    q, out = torch.zeros_like(s.q), torch.empty_like(want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        q.copy_(s.q)
        s.kv.attend(0, q, *args, out, None, s.n_max)
        got = out.clone()
    s.kv.sync()
    side.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    out.zero_()
    with torch.cuda.graph(g):
        s.kv.attend(0, q, *args, out, None, s.n_max)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_calls_refuse_another_current_device():
    """A cache belongs to the device that was current at its creation: there is one here, so the handle's note of it is changed."""
    s = Step([30], [2], 4, 2, 64, 16, "fp8", "bf16")
    good, _ = s.run(chain=True)
    device = ctypes.c_int.from_address(s.kv.handle + ctypes.sizeof(ace.ace_kv_desc))
    assert device.value == torch.cuda.current_device()
    i = lambda *a: torch.zeros(*a, dtype=torch.int32, device="cuda")    # noqa: E731
    rows, slots = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.full((1,), -1, dtype=torch.int64, device="cuda")
    calls = [lambda: s.kv.write(0, rows, rows, slots), lambda: s.kv.read(0, slots, rows, rows),
             lambda: s.kv.keep(i(1, 3), i(1), i(1, 2), i(1)), lambda: s.run(chain=True)]
    device.value += 1
    try:
        for call in calls:
            with pytest.raises(ace.AceError, match="another device") as err:
                call()
            assert err.value.status == 1
    finally:
        device.value -= 1
    for call in calls:
        call()
    again, _ = s.run(chain=True)
    assert torch.equal(again, good)
