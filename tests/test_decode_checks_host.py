"""What the speculative decode step's calls refuse before any device call: memory that its kernels could not read."""
import ctypes
import importlib.util
import os

import pytest
import torch

from paper_2609_05228_gb300 import ace, build

INVALID = 1


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ace.LIBPATH):
        build.build()
    ace._lib = None
    return ace.lib()


@pytest.mark.parametrize("head_dim,dtype", [(64, ace.ACE_BF16), (128, ace.ACE_BF16), (80, ace.ACE_F32)])
@pytest.mark.parametrize("ks,vs", [(17, 16), (16, 33), (24, 16), (16, 20), (18, 18)])
def test_create_refuses_scales_that_are_not_aligned(L, head_dim, dtype, ks, vs):
    out = ctypes.c_void_p(7)
    d = ace.ace_kv_desc(1, 4, 16, 2, head_dim, dtype, ace.ACE_KV_FP8)
    assert L.ace_kv_create(ctypes.byref(d), 16, 16, ks, vs, None, ctypes.byref(out)) == INVALID
    assert out.value is None and b"scales" in L.ace_last_error_message()


class Calls:
    """A library that notes its calls and launches nothing."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            return 0
        return call


@pytest.fixture
def calls(monkeypatch):
    """The binding over a library that does nothing; CPU tensors count as the GPU's."""
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
    return fake.made


def _verify_args(T=4, B=2, V=16):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)       # noqa: E731
    return dict(logits=torch.zeros(T, V), tokens=i(T), parents=i(T), node_offsets=i(B + 1), max_nodes=4, uniforms=torch.zeros(T),
                noise=torch.ones(B, V), path=i(B, 4), n_keep=i(B), next_token=i(B), draft_probs=torch.zeros(T, V))


@pytest.mark.parametrize("name", ["logits", "noise", "draft_probs"])
def test_verify_refuses_rows_that_overlap(calls, name):
    """Broadcast rows have a stride of 0, windows into one buffer a small one: neither is a row every `vocab` elements."""
    a = _verify_args()
    rows, V = a[name].shape
    for t in (torch.zeros(1, V).expand(rows, V), torch.zeros(2 * V).as_strided((rows, V), (3, 1))):
        with pytest.raises(ValueError, match=name):
            ace.ace_verify_tree(**dict(a, **{name: t}))
    assert calls == []


def test_verify_passes_on_the_strides_of_rows(calls):
    """Padded rows, and single rows, whose stride says nothing."""
    a = _verify_args()
    a["logits"] = torch.zeros(4, 24)[:, :16]
    a["noise"] = torch.zeros(2, 40)[:, :16]
    ace.ace_verify_tree(**a)
    one = _verify_args(1, 1)
    one["logits"], one["noise"] = torch.zeros(16).expand(1, 16), torch.zeros(32).as_strided((1, 16), (0, 1))
    ace.ace_verify_tree(**one)
    (n0, c0), (n1, c1) = calls
    assert n0 == n1 == "ace_verify_tree"
    assert (c0[2], c0[11], c0[15]) == (24, 16, 40) and (c1[2], c1[11], c1[15]) == (16, 16, 16)


def _mask_args(T=5, B=2, n=70, depth=True):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)       # noqa: E731
    return dict(parents=i(T), node_offsets=i(B + 1), B=B, max_nodes=n, mask=torch.zeros(T, -(-n // 64), dtype=torch.int64),
                depth=i(T) if depth else None)


@pytest.mark.parametrize("name,t", [
    ("mask", torch.zeros(5, 2, dtype=torch.int32)), ("mask", torch.zeros(5, 1, dtype=torch.int64)),
    ("mask", torch.zeros(4, 2, dtype=torch.int64)), ("mask", torch.zeros(2, 5, dtype=torch.int64).T),
    ("parents", torch.zeros(5, dtype=torch.int64)), ("parents", torch.zeros(10, dtype=torch.int32)[::2]),
    ("node_offsets", torch.zeros(2, dtype=torch.int32)), ("node_offsets", torch.zeros(3)),
    ("depth", torch.zeros(4, dtype=torch.int32)), ("depth", torch.zeros(5))])
def test_tree_mask_refuses_tensors_that_it_would_overrun(calls, name, t):
    with pytest.raises(ValueError, match=name):
        ace.ace_tree_mask(**dict(_mask_args(), **{name: t}))
    assert calls == []


def test_tree_mask_takes_its_own_layouts(calls):
    ace.ace_tree_mask(**_mask_args())
    ace.ace_tree_mask(**_mask_args(depth=False))
    ace.ace_tree_mask(**_mask_args(0, 0, 1))
    assert len(calls) == 3


def test_tree_mask_refuses_memory_of_the_host():
    with pytest.raises(ValueError, match="on a GPU"):
        ace.ace_tree_mask(**_mask_args())


def test_tree_mask_tells_its_rows(calls):
    ace.ace_tree_mask(**_mask_args())
    (name, args), = calls
    assert name == "ace_tree_mask_rows" and args[2:5] == (2, 5, 70)


def test_tree_mask_rows_refuses(L):
    assert L.ace_tree_mask_rows(16, 16, 1, -1, 4, 16, None, None) == INVALID
    assert L.ace_tree_mask_rows(16, 16, -1, 4, 4, 16, None, None) == INVALID
    for n in (0, 257):
        assert L.ace_tree_mask_rows(16, 16, 1, 4, n, 16, None, None) == INVALID
    assert L.ace_tree_mask_rows(None, 16, 1, 4, 4, 16, None, None) == INVALID
    assert L.ace_tree_mask_rows(None, None, 2, 0, 4, None, None, None) == 0


def _cache(calls, layers=2):
    """A cache object over CPU tensors, without a handle's memory."""
    kv = ace.AceKvCache.__new__(ace.AceKvCache)
    kv.handle, kv.layers, kv.n_pages, kv.page_size, kv.n_kv_heads, kv.head_dim = 7, layers, 4, 16, 2, 64
    kv.torch_dtype, kv._dt = torch.bfloat16, "bfloat16"
    return kv


def test_calls_run_on_the_current_stream(calls, monkeypatch):
    """Without a stream, calls on torch tensors are ordered with what made the tensors: torch's current stream."""
    seen = []
    monkeypatch.setattr(ace, "_raw_stream", lambda device: seen.append(device) or 77, raising=False)
    kv = _cache(calls)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)       # noqa: E731
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)    # noqa: E731
    slots = torch.zeros(3, dtype=torch.int64)
    runs = [lambda **s: kv.write(0, b(3, 2, 64), b(3, 2, 64), slots, **s), lambda **s: kv.read(0, slots, b(3, 2, 64), b(3, 2, 64), **s),
            lambda **s: kv.keep(i(2, 4), i(2), i(2, 8), i(2), i(2), **s),
            lambda **s: kv.attend(0, b(3, 4, 64), i(2, 4), i(2), i(3), b(3, 4, 64), **s),
            lambda **s: ace.ace_tree_mask(**_mask_args(), **s), lambda **s: ace.ace_verify_tree(**_verify_args(), **s)]
    for run in runs:
        run()
        assert calls[-1][1][-1] == 77, calls[-1]
        run(stream=5)
        assert calls[-1][1][-1] == 5, calls[-1]
        run(stream=0)                               # the legacy default stream, if that is what is wanted
        assert calls[-1][1][-1] == 0
    assert len(seen) == len(runs) and all(d == -1 for d in seen)
    kv.handle = None


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decode.py")
    spec = importlib.util.spec_from_file_location("speculative_decode", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("count,drafted,used", [(64, True, 0), (17, True, 0), (59, False, 6)])
def test_example_refuses_more_tokens_than_its_pages_hold(example, count, drafted, used):
    """The request that accepts most runs ahead of the one that ends the loop; its rows have to have pages."""
    class Full:
        pages, lens = torch.zeros(4, 4, dtype=torch.int32), torch.tensor([0, used, 0, 0], dtype=torch.int32)
    assert Full.pages.shape[1] * example.PAGE == 64
    with pytest.raises(ValueError, match="positions"):
        example.generate(Full(), torch.zeros(4, dtype=torch.int32), count, 0.8, drafted)


def test_example_counts_the_positions_of_the_luckiest_request(example):
    """Every step one token for the slowest request and all that a path can give for the fastest; a tree's rows in each step."""
    tree = example.TREE
    depth = max(len(_path(tree, i)) for i in range(len(tree)))
    for count in (1, 2, 15, 64):
        rows = slow = fast = 0
        while slow < count:
            rows = max(rows, fast + len(tree))
            slow, fast = slow + 1, fast + depth
        assert example.positions(count) == max(rows, fast)
        assert example.positions(count, False) == count


def _path(parents, i):
    return [] if i < 0 else _path(parents, parents[i]) + [i]
