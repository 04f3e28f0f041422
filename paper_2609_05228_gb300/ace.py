"""ctypes binding of libace.so (include/ace.h). Argument marshalling only:
every step of the layer runs in the library's CUDA kernels.

Functions keep the C names. Device pointers may be given as ints or as torch
tensors (their data_ptr()); host outputs are returned as numpy arrays.
Streams may be None (default stream), an int handle or a torch.cuda.Stream.
The library is loaded on first use; a missing library raises AceError.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_LIBDIR = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_lib")
# ACE_LIB_VARIANT=debug loads libace_debug.so (index guards and canary words)
LIBNAME = "libace_debug.so" if os.environ.get("ACE_LIB_VARIANT") == "debug" else "libace.so"
LIBPATH = os.path.join(_LIBDIR, LIBNAME)

ACE_BF16, ACE_F32 = 0, 1
ACE_SKIP_THRESHOLD, ACE_SKIP_RATIO = 0, 1
ACE_KV_PLAIN, ACE_KV_FP8 = 0, 1
# Skip rules (ace_fusion): index = enum value. "max" is ACE.
FUSIONS = ("max", "min", "mean", "gsp", "rcr", "score")
ACE_FUSION_MAX, ACE_FUSION_MIN, ACE_FUSION_MEAN, ACE_FUSION_GSP, ACE_FUSION_RCR, ACE_FUSION_SCORE = range(6)
STATUS = {0: "ACE_OK", 1: "ACE_ERR_INVALID_ARG", 2: "ACE_ERR_UNSUPPORTED", 3: "ACE_ERR_OOM",
          4: "ACE_ERR_CUDA", 5: "ACE_ERR_TIMEOUT", 6: "ACE_ERR_NUMERIC", 7: "ACE_ERR_STATE"}


class AceError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class ace_layer_desc(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int), ("n_experts", ctypes.c_int), ("top_k", ctypes.c_int),
                ("ffn", ctypes.c_int), ("max_tokens", ctypes.c_int), ("dtype", ctypes.c_int),
                ("eps", ctypes.c_float), ("rms_eps", ctypes.c_float), ("router_temp", ctypes.c_float),
                ("min_active", ctypes.c_int), ("has_router_bias", ctypes.c_int), ("add_residual", ctypes.c_int)]


class ace_skip_ctl(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int), ("value", ctypes.c_float), ("fusion", ctypes.c_int)]


class ace_kv_desc(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int), ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int),
                ("n_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("dtype", ctypes.c_int),
                ("format", ctypes.c_int)]


_lib = None
_P = ctypes.c_void_p
_I = ctypes.c_int
_LL = ctypes.c_longlong
_F = ctypes.c_float
_S = ctypes.c_int  # ace_status


def lib() -> ctypes.CDLL:
    """Load libace.so (raises AceError if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIBPATH):
            raise AceError(4, f"{LIBNAME} not found at {LIBPATH}; build it with "
                              "`python -m paper_2609_05228_gb300.build`")
        L = ctypes.CDLL(LIBPATH)
        sig = {
            "ace_layer_create": (_S, [ctypes.POINTER(ace_layer_desc), _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                      ctypes.POINTER(_P)]),
            "ace_layer_destroy": (None, [_P]),
            "ace_moe_forward": (_S, [_P, _P, _P, _I, ace_skip_ctl, _P]),
            "ace_moe_forward_host": (_S, [_P, _P, _P, _I, ace_skip_ctl, _P]),
            "ace_route_logits": (_S, [_P, _P, _I, ace_skip_ctl, _P]),
            "ace_last_skip_mask": (_S, [_P, _P, _P, _P, _P, _P]),
            "ace_last_router_logits": (_S, [_P, _P]),
            "ace_last_permutation": (_S, [_P, _P, _P]),
            "ace_layer_sync": (_S, [_P]),
            "ace_debug_exp32": (_S, [_P, _P, _I, _P]),
            "ace_debug_set_wait_budget": (_S, [_P, ctypes.c_longlong]),
            "ace_debug_checks_enabled": (_I, []),
            "ace_debug_poke_canary": (_S, [_P, _I]),
            "ace_layer_get_desc": (_S, [_P, ctypes.POINTER(ace_layer_desc)]),
            "ace_layer_set_profiling": (_S, [_P, _I]),
            "ace_last_stage_times": (_S, [_P, _P, _I, _P]),
            "ace_last_launch_count": (_S, [_P, _P]),
            "ace_route_decide_noalloc": (_S, [_P, _I, _I, _I, _P, _P, ctypes.c_float, _I, ace_skip_ctl, _P, _P, _P,
                                              _P, _P]),
            "ace_stack_create": (_S, [ctypes.POINTER(_P), _I, ctypes.POINTER(_P)]),
            "ace_stack_forward": (_S, [_P, _P, _P, _I, ace_skip_ctl, _P]),
            "ace_stack_destroy": (None, [_P]),
            "ace_stack_forward_host": (_S, [_P, _P, _P, _I, ace_skip_ctl, _P]),
            "ace_offline_tables_device": (_S, [_I, _I, _I, _P, _P, _P, _P, _P, ctypes.c_double, _I, ctypes.c_size_t,
                                               _P, _P, _P]),
            "ace_kv_create": (_S, [ctypes.POINTER(ace_kv_desc), _P, _P, _P, _P, _P, ctypes.POINTER(_P)]),
            "ace_kv_destroy": (None, [_P]),
            "ace_kv_sync": (_S, [_P]),
            "ace_kv_write": (_S, [_P, _I, _P, _LL, _LL, _P, _LL, _LL, _P, _I, _P]),
            "ace_kv_read": (_S, [_P, _I, _P, _I, _P, _P, _P]),
            "ace_kv_keep": (_S, [_P, _P, _I, _P, _P, _I, _P, _I, _P, _P]),
            "ace_tree_mask": (_S, [_P, _P, _I, _I, _P, _P, _P]),
            "ace_tree_mask_rows": (_S, [_P, _P, _I, _I, _I, _P, _P, _P]),
            "ace_tree_attention": (_S, [_P, _I, _P, _LL, _LL, _I, _P, _I, _P, _P, _P, _I, _I, _I, _F, _P, _P, _P]),
            "ace_verify_tree": (_S, [_P, _I, _LL, _I, _P, _P, _P, _I, _I, _I, _P, _LL, _P, _P, _P, _LL, _P, _P, _P, _P]),
            "ace_status_string": (ctypes.c_char_p, [_S]),
            "ace_last_error_message": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _ptr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    raise TypeError(f"cannot take a pointer of {type(x)}")


def _stream(s) -> int | None:
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(st: int) -> None:
    if st != 0:
        raise AceError(st, lib().ace_last_error_message().decode())


def _fusion(fusion) -> int:
    if isinstance(fusion, str):
        if fusion not in FUSIONS:
            raise ValueError(f"unknown fusion {fusion!r}; one of {FUSIONS}")
        return FUSIONS.index(fusion)
    return int(fusion)


def _ctl(mode, value, fusion=ACE_FUSION_MAX) -> ace_skip_ctl:
    if isinstance(mode, str):
        mode = ACE_SKIP_RATIO if mode == "ratio" else ACE_SKIP_THRESHOLD
    return ace_skip_ctl(int(mode), float(value), _fusion(fusion))


def ace_layer_create(desc: ace_layer_desc, router_w, router_b, w_gate, w_up, w_down, rms_gamma,
                     a_gsp: np.ndarray, a_rcr: np.ndarray, stream=None) -> int:
    a_gsp = np.ascontiguousarray(a_gsp, dtype=np.float32)
    a_rcr = np.ascontiguousarray(a_rcr, dtype=np.float32)
    out = _P()
    _check(lib().ace_layer_create(ctypes.byref(desc), _ptr(router_w), _ptr(router_b), _ptr(w_gate),
                                  _ptr(w_up), _ptr(w_down), _ptr(rms_gamma), a_gsp.ctypes.data,
                                  a_rcr.ctypes.data, _stream(stream), ctypes.byref(out)))
    return out.value


def ace_layer_destroy(layer: int) -> None:
    if layer:
        lib().ace_layer_destroy(layer)


def ace_moe_forward(layer: int, x, out, T: int, mode, value: float, stream=None, fusion=ACE_FUSION_MAX) -> None:
    _check(lib().ace_moe_forward(layer, _ptr(x), _ptr(out), int(T), _ctl(mode, value, fusion), _stream(stream)))


def ace_moe_forward_host(layer: int, x_host, out_host, T: int, mode, value: float, stream=None, fusion=ACE_FUSION_MAX) -> None:
    _check(lib().ace_moe_forward_host(layer, _ptr(x_host), _ptr(out_host), int(T), _ctl(mode, value, fusion),
                                      _stream(stream)))


def ace_route_logits(layer: int, logits, T: int, mode, value: float, stream=None, fusion=ACE_FUSION_MAX) -> None:
    _check(lib().ace_route_logits(layer, _ptr(logits), int(T), _ctl(mode, value, fusion), _stream(stream)))


def ace_stack_create(layers) -> int:
    """A stack over layer handles (ints); the layers must outlive it."""
    arr = (_P * len(layers))(*[int(h) for h in layers])
    out = _P()
    _check(lib().ace_stack_create(arr, len(layers), ctypes.byref(out)))
    return out.value


def ace_stack_forward(stack: int, x, out, T: int, mode, value: float, stream=None, fusion=ACE_FUSION_MAX) -> None:
    _check(lib().ace_stack_forward(stack, _ptr(x), _ptr(out), int(T), _ctl(mode, value, fusion), _stream(stream)))


def ace_stack_forward_host(stack: int, x_host, out_host, T: int, mode, value: float, stream=None,
                           fusion=ACE_FUSION_MAX) -> None:
    _check(lib().ace_stack_forward_host(stack, _ptr(x_host), _ptr(out_host), int(T), _ctl(mode, value, fusion),
                                        _stream(stream)))


def ace_stack_destroy(stack: int) -> None:
    if stack:
        lib().ace_stack_destroy(stack)


def ace_last_skip_mask(layer: int, T: int, k: int):
    """Returns (skip uint8 [T,k], ids int32 [T,k], gates_hat float32 [T,k], tau, R)."""
    skip = np.zeros((T, k), np.uint8)
    ids = np.zeros((T, k), np.int32)
    gh = np.zeros((T, k), np.float32)
    tau = np.zeros(1, np.float32)
    r = np.zeros(1, np.int32)
    _check(lib().ace_last_skip_mask(layer, skip.ctypes.data, ids.ctypes.data, gh.ctypes.data,
                                    tau.ctypes.data, r.ctypes.data))
    return skip, ids, gh, tau[0], int(r[0])


def ace_last_router_logits(layer: int, T: int, N: int) -> np.ndarray:
    z = np.zeros((T, N), np.float32)
    _check(lib().ace_last_router_logits(layer, z.ctypes.data))
    return z


def ace_last_permutation(layer: int, N: int, R: int):
    off = np.zeros(N + 1, np.int32)
    perm = np.zeros(max(R, 1), np.int32)
    _check(lib().ace_last_permutation(layer, off.ctypes.data, perm.ctypes.data))
    return off, perm[:R]


def ace_layer_sync(layer: int) -> None:
    _check(lib().ace_layer_sync(layer))


def ace_debug_set_wait_budget(layer: int, cycles: int) -> None:
    _check(lib().ace_debug_set_wait_budget(layer, int(cycles)))


def ace_debug_checks_enabled() -> bool:
    return bool(lib().ace_debug_checks_enabled())


def ace_debug_poke_canary(layer: int, index: int) -> None:
    _check(lib().ace_debug_poke_canary(layer, int(index)))


def ace_debug_exp32(x, y, n: int, stream=None) -> None:
    _check(lib().ace_debug_exp32(_ptr(x), _ptr(y), int(n), _stream(stream)))


STAGES = ["rmsnorm", "router", "route", "gather", "gate_up", "down", "combine"]


def ace_layer_set_profiling(layer: int, enable: bool) -> None:
    _check(lib().ace_layer_set_profiling(layer, int(bool(enable))))


def ace_last_stage_times(layer: int) -> dict:
    ms = np.zeros(16, np.float32)
    n = np.zeros(1, np.int32)
    _check(lib().ace_last_stage_times(layer, ms.ctypes.data, 16, n.ctypes.data))
    return {STAGES[i] if i < len(STAGES) else f"stage{i}": float(ms[i]) for i in range(int(n[0]))}


def ace_route_decide_noalloc(logits, T: int, n_experts: int, top_k: int, a_gsp, a_rcr, eps: float,
                             min_active: int, mode, value: float, ids, skip, gates_hat, tau, stream=None,
                             fusion=ACE_FUSION_MAX) -> None:
    """Routing decision without a layer or any device allocation (all pointers are device buffers)."""
    _check(lib().ace_route_decide_noalloc(_ptr(logits), int(T), int(n_experts), int(top_k), _ptr(a_gsp), _ptr(a_rcr),
                                          float(eps), int(min_active), _ctl(mode, value, fusion), _ptr(ids), _ptr(skip),
                                          _ptr(gates_hat), _ptr(tau), _stream(stream)))


def ace_offline_tables_device(d: int, N: int, m: int, gamma, router_w, w_gate, w_up, w_down, eps: float = 1e-6,
                              rcr_apply_gamma: bool = False, tile_budget: int = 0, stream=None):
    """(A^GSP, A^RCR) float32 [N] computed on the GPU from bf16 device weights."""
    gsp = np.empty(N, np.float32)
    rcr = np.empty(N, np.float32)
    _check(lib().ace_offline_tables_device(int(d), int(N), int(m), _ptr(gamma), _ptr(router_w), _ptr(w_gate),
                                           _ptr(w_up), _ptr(w_down), float(eps), int(bool(rcr_apply_gamma)),
                                           int(tile_budget), gsp.ctypes.data, rcr.ctypes.data, _stream(stream)))
    return gsp, rcr


def ace_last_launch_count(layer: int) -> int:
    n = np.zeros(1, np.int32)
    _check(lib().ace_last_launch_count(layer, n.ctypes.data))
    return int(n[0])


def ace_layer_get_desc(layer: int) -> ace_layer_desc:
    d = ace_layer_desc()
    _check(lib().ace_layer_get_desc(layer, ctypes.byref(d)))
    return d


# --------------------------------------------------------------------------
# Speculative decode step: the cache, attention for trees of drafted tokens, verification
# --------------------------------------------------------------------------

def ace_kv_create(desc: ace_kv_desc, k_pool, v_pool, k_scale=None, v_scale=None, stream=None) -> int:
    out = _P()
    _check(lib().ace_kv_create(ctypes.byref(desc), _ptr(k_pool), _ptr(v_pool), _ptr(k_scale), _ptr(v_scale),
                               _stream(stream), ctypes.byref(out)))
    return out.value


def ace_kv_destroy(kv: int) -> None:
    if kv:
        lib().ace_kv_destroy(kv)


def ace_kv_sync(kv: int) -> None:
    _check(lib().ace_kv_sync(kv))


def ace_kv_write(kv: int, layer: int, k, k_token_stride: int, k_head_stride: int, v, v_token_stride: int,
                 v_head_stride: int, slots, T: int, stream=None) -> None:
    _check(lib().ace_kv_write(kv, layer, _ptr(k), k_token_stride, k_head_stride, _ptr(v), v_token_stride, v_head_stride,
                              _ptr(slots), T, _stream(stream)))


def ace_kv_read(kv: int, layer: int, slots, T: int, k_out, v_out, stream=None) -> None:
    _check(lib().ace_kv_read(kv, layer, _ptr(slots), T, _ptr(k_out), _ptr(v_out), _stream(stream)))


def ace_kv_keep(kv: int, page_table, max_pages: int, lens, path, max_nodes: int, n_keep, B: int, new_lens=None,
                stream=None) -> None:
    _check(lib().ace_kv_keep(kv, _ptr(page_table), max_pages, _ptr(lens), _ptr(path), max_nodes, _ptr(n_keep), B,
                             _ptr(new_lens), _stream(stream)))


def ace_tree_mask(parents, node_offsets, B: int, max_nodes: int, mask, depth=None, stream=None) -> None:
    """Ancestor masks [T, ceil(max_nodes / 64)] (int64 words) and depths [T] of trees given by parents [T] (torch tensors).
    Requests whose offsets are not within 0 .. T are left out. Runs on torch's current stream unless one is given."""
    T = parents.shape[0]
    for name, t in (("parents", parents), ("depth", depth)):
        if t is not None:
            _want(name, t, "int32", (T,))
    _want("node_offsets", node_offsets, "int32", (B + 1,))
    _want("mask", mask, "int64", (T, (max_nodes + 63) // 64))
    _check(lib().ace_tree_mask_rows(_ptr(parents), _ptr(node_offsets), B, T, max_nodes, _ptr(mask), _ptr(depth),
                                    _stream_for(parents, stream)))


def ace_tree_attention(kv: int, layer: int, q, q_token_stride: int, q_head_stride: int, n_heads: int, page_table,
                       max_pages: int, lens, node_offsets, mask, B: int, T: int, max_nodes: int, scale: float, out,
                       lse=None, stream=None) -> None:
    _check(lib().ace_tree_attention(kv, layer, _ptr(q), q_token_stride, q_head_stride, n_heads, _ptr(page_table), max_pages,
                                    _ptr(lens), _ptr(node_offsets), _ptr(mask), B, T, max_nodes, scale, _ptr(out),
                                    _ptr(lse), _stream(stream)))


_dtypes = None


def _dtype(name: str):
    """torch's dtype of that name (torch is imported at the first use)."""
    global _dtypes
    if _dtypes is None:
        import torch

        _dtypes = {n: getattr(torch, n) for n in ("bfloat16", "float32", "int32", "int64", "uint8", "float8_e4m3fn")}
    return _dtypes[name]


_current_stream = None


def _raw_stream(device: int) -> int:
    """torch's current stream on a device, as a pointer (torch is imported at the first use)."""
    global _current_stream
    if _current_stream is None:
        import torch

        _current_stream = torch._C._cuda_getCurrentRawStream
    return _current_stream(device)


def _stream_for(t, stream) -> int:
    """The stream of a call on torch tensors such as t: the one given, or torch's current one, which made them."""
    return _raw_stream(t.get_device()) if stream is None else _stream(stream)


def _want(name: str, t, dtype: str, shape=None, contiguous: bool = True):
    """Checks a torch tensor argument: its type, shape (None: any size) and layout."""
    if t.dtype is _dtype(dtype) and (shape is None or t.shape == shape) and (not contiguous or t.is_contiguous()) and t.is_cuda:
        return
    if t.dtype is not _dtype(dtype):
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if shape is not None and (t.dim() != len(shape) or any(w is not None and w != g for w, g in zip(shape, t.shape))):
        raise ValueError(f"{name} must have shape {shape}, not {tuple(t.shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU")


def _row_stride(name: str, t, V: int) -> int:
    """Elements from one row of t [rows, V] to the next. A single row's stride says nothing and counts as V."""
    rows, stride = t.shape[0], t.stride(0)
    if rows and V > 1 and t.stride(1) != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    if rows > 1 and stride < V:
        raise ValueError(f"the rows of {name} must not overlap (a broadcast tensor has to be laid out)")
    return max(V, stride)


def ace_verify_tree(logits, tokens, parents, node_offsets, max_nodes: int, uniforms, noise, path, n_keep, next_token,
                    draft_probs=None, temperature=None, stream=None) -> None:
    """Verification of drafted tokens (torch tensors; layouts in include/ace.h): fills path [B, max_nodes],
    n_keep [B] and next_token [B] (int32). logits and draft_probs [T, vocab] and noise [B, vocab] may have padded rows. Runs on
    torch's current stream unless one is given."""
    T, V = logits.shape
    B = node_offsets.shape[0] - 1
    dt = ACE_BF16 if logits.dtype is _dtype("bfloat16") else ACE_F32
    if dt == ACE_F32 and logits.dtype is not _dtype("float32"):
        raise ValueError(f"logits must be bfloat16 or float32, not {logits.dtype}")
    _want("logits", logits, "bfloat16" if dt == ACE_BF16 else "float32", (T, V), False)
    _want("noise", noise, "float32", (B, V), False)
    _want("uniforms", uniforms, "float32", (T,))
    if draft_probs is not None:
        _want("draft_probs", draft_probs, "float32", (T, V), False)
    if temperature is not None:
        _want("temperature", temperature, "float32", (B,))
    for name, t, shape in (("tokens", tokens, (T,)), ("parents", parents, (T,)), ("node_offsets", node_offsets, (B + 1,)),
                           ("path", path, (B, max_nodes)), ("n_keep", n_keep, (B,)), ("next_token", next_token, (B,))):
        _want(name, t, "int32", shape)
    logits_stride, noise_stride = _row_stride("logits", logits, V), _row_stride("noise", noise, V)
    draft_stride = _row_stride("draft_probs", draft_probs, V) if draft_probs is not None else V
    _check(lib().ace_verify_tree(logits.data_ptr(), dt, logits_stride, V, tokens.data_ptr(), parents.data_ptr(),
                                 node_offsets.data_ptr(), B, T, max_nodes, _ptr(draft_probs), draft_stride,
                                 _ptr(temperature), uniforms.data_ptr(), noise.data_ptr(), noise_stride, path.data_ptr(),
                                 n_keep.data_ptr(), next_token.data_ptr(), _stream_for(logits, stream)))


class AceKvCache:
    """A paged key/value cache of a model's layers and its ace_kv handle. The pools are torch tensors:
    those given, or new ones (zeros). fmt "plain" keeps rows in dtype, "fp8" e4m3 codes and a scale
    byte per (token, head). Slots are page * page_size + row. Calls run on torch's current stream unless one is given."""

    def __init__(self, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, layers: int = 1, dtype: str = "bf16",
                 fmt: str = "fp8", k_pool=None, v_pool=None, k_scale=None, v_scale=None, device: int = 0):
        import torch

        if dtype not in ("bf16", "f32") or fmt not in ("plain", "fp8"):
            raise ValueError("dtype must be 'bf16' or 'f32' and fmt 'plain' or 'fp8'")
        self.handle = None
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self._dt = "bfloat16" if dtype == "bf16" else "float32"
        self.layers, self.n_pages, self.page_size = int(layers), int(n_pages), int(page_size)
        self.n_kv_heads, self.head_dim = int(n_kv_heads), int(head_dim)
        rows = (self.layers, self.n_pages, self.n_kv_heads, self.page_size)
        dev = torch.device("cuda", device)
        pool_dt = torch.float8_e4m3fn if fmt == "fp8" else self.torch_dtype

        def own(t, shape, dt, name):
            if t is None:
                return torch.zeros(shape, dtype=dt, device=dev)
            _want(name, t, str(dt)[6:], shape)
            return t

        self.k_pool = own(k_pool, rows + (self.head_dim,), pool_dt, "k_pool")
        self.v_pool = own(v_pool, rows + (self.head_dim,), pool_dt, "v_pool")
        self.k_scale = self.v_scale = None
        if fmt == "fp8":
            self.k_scale = own(k_scale, rows, torch.uint8, "k_scale")
            self.v_scale = own(v_scale, rows, torch.uint8, "v_scale")
        self.desc = ace_kv_desc(self.layers, self.n_pages, self.page_size, self.n_kv_heads, self.head_dim,
                                ACE_BF16 if dtype == "bf16" else ACE_F32, ACE_KV_FP8 if fmt == "fp8" else ACE_KV_PLAIN)
        with torch.cuda.device(self.k_pool.device):
            self.handle = ace_kv_create(self.desc, self.k_pool, self.v_pool, self.k_scale, self.v_scale,
                                        _stream_for(self.k_pool, None))

    def _rows(self, name, t, heads):
        """(token stride, head stride) of rows [T, heads, head_dim] of any strides but the last."""
        _want(name, t, self._dt, (t.shape[0], heads, self.head_dim), False)
        if t.numel() and t.stride(2) != 1:
            raise ValueError(f"the last axis of {name} must be contiguous")
        return t.stride(0), t.stride(1)

    def write(self, layer: int, k, v, slots, stream=None) -> None:
        """k, v [T, n_kv_heads, head_dim] (any strides but the last) to `slots` [T] int64 of a layer."""
        T = k.shape[0]
        ks, vs = self._rows("k", k, self.n_kv_heads), self._rows("v", v, self.n_kv_heads)
        if v.shape[0] != T:
            raise ValueError("k and v must have the same tokens")
        _want("slots", slots, "int64", (T,))
        ace_kv_write(self.handle, layer, k, *ks, v, *vs, slots, T, _stream_for(k, stream))

    def read(self, layer, slots, k_out, v_out, stream=None) -> None:
        """The rows at `slots` [T] to k_out, v_out [T, n_kv_heads, head_dim]; layer None: of all layers,
        [layers, T, n_kv_heads, head_dim]."""
        T = slots.shape[0]
        shape = (T, self.n_kv_heads, self.head_dim)
        if layer is None:
            layer, shape = -1, (self.layers,) + shape
        _want("slots", slots, "int64", (T,))
        for name, t in (("k_out", k_out), ("v_out", v_out)):
            _want(name, t, self._dt, shape)
        ace_kv_read(self.handle, layer, slots, T, k_out, v_out, _stream_for(slots, stream))

    def keep(self, page_table, lens, path, n_keep, new_lens=None, stream=None) -> None:
        """The rows of nodes path[b, :n_keep[b]] move to positions lens[b] + 0, 1, .. in every layer."""
        B, max_pages = page_table.shape
        max_nodes = path.shape[1]
        _want("page_table", page_table, "int32")
        _want("path", path, "int32", (B, max_nodes))
        for name, t in (("lens", lens), ("n_keep", n_keep)) + ((("new_lens", new_lens),) if new_lens is not None else ()):
            _want(name, t, "int32", (B,))
        ace_kv_keep(self.handle, page_table, max_pages, lens, path, max_nodes, n_keep, B, new_lens, _stream_for(lens, stream))

    def attend(self, layer: int, q, page_table, lens, node_offsets, out, mask=None, max_nodes: int = 1, scale=None,
               lse=None, stream=None) -> None:
        """q [T, n_heads, head_dim] (any strides but the last) attends to the cached prefixes and, by
        `mask` (int64 words, None: a chain), to the trees' nodes; out like q, contiguous; scale None: 1 / sqrt(head_dim)."""
        T, heads = q.shape[0], q.shape[1]
        qs = self._rows("q", q, heads)
        B, max_pages = page_table.shape
        _want("page_table", page_table, "int32")
        _want("lens", lens, "int32", (B,))
        _want("node_offsets", node_offsets, "int32", (B + 1,))
        _want("out", out, self._dt, q.shape)
        if mask is not None:
            _want("mask", mask, "int64", (T, (max_nodes + 63) // 64))
        if lse is not None:
            _want("lse", lse, "float32", (T, heads))
        ace_tree_attention(self.handle, layer, q, *qs, heads, page_table, max_pages, lens, node_offsets, mask, B, T,
                           max_nodes, self.head_dim ** -0.5 if scale is None else scale, out, lse, _stream_for(q, stream))

    def sync(self) -> None:
        """Waits for the last call and raises AceError for what its kernels found."""
        ace_kv_sync(self.handle)

    def close(self) -> None:
        if getattr(self, "handle", None):
            ace_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# --------------------------------------------------------------------------
# Convenience: a layer built from host arrays (synth.LayerWeights-like), with
# torch used only to hold the device copies during creation.
# --------------------------------------------------------------------------

class AceLayer:
    """Owns one ace_layer. `w` holds nn.Linear-shaped host arrays (bf16 as
    uint16 bits or float32); a_gsp / a_rcr are the offline tables."""

    def __init__(self, w, a_gsp, a_rcr, max_tokens: int, device: int = 0, residual: bool = False):
        import torch

        spec = w.spec
        bf = spec.dtype == "bf16"
        tdt = torch.bfloat16 if bf else torch.float32
        dev = torch.device("cuda", device)

        def up(a):
            a = np.ascontiguousarray(a)
            if a.dtype == np.uint16:
                return torch.from_numpy(a.view(np.int16)).view(torch.bfloat16).to(dev)
            return torch.from_numpy(a.astype(np.float32, copy=False)).to(dev)

        has_bias = bool(np.any(w.router_b != 0))
        self.desc = ace_layer_desc(spec.hidden, spec.n_experts, spec.top_k, spec.ffn, int(max_tokens),
                                   ACE_BF16 if bf else ACE_F32, spec.eps, spec.rms_eps, spec.router_temp,
                                   spec.min_active, int(has_bias), int(residual))
        tensors = [up(w.router_w), torch.from_numpy(np.ascontiguousarray(w.router_b, np.float32)).to(dev),
                   up(w.w_gate), up(w.w_up), up(w.w_down), up(w.gamma)]
        torch.cuda.synchronize(dev)
        self.handle = ace_layer_create(self.desc, *tensors, a_gsp, a_rcr)
        del tensors
        self.spec = spec
        self.torch_dtype = tdt

    def forward(self, x, out, T: int, mode="threshold", value: float = 0.0, stream=None,
                fusion=ACE_FUSION_MAX) -> None:
        ace_moe_forward(self.handle, x, out, T, mode, value, stream, fusion)

    def close(self) -> None:
        if getattr(self, "handle", None):
            ace_layer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
