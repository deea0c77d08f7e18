"""Thin binding over the C-ABI CUDA library (``libqp.so``): argument marshalling only.

Every function has the name and the meaning of the C entry point it forwards to
(see ``include/qp.h``).  torch is used for device memory, pointers and the current
stream; no step of the path runs in Python or on the CPU.  Loading fails loudly
when the library has not been built.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# QP_LIBRARY selects another build of the same library (the range-checked debug build libqp_checked.so)
LIB_PATH = os.environ.get("QP_LIBRARY") or os.path.join(_HERE, "libqp.so")

QP_OK = 0
QP_MAX_LAYERS = 128
QP_MAX_DRAFTS = 64
QP_MAX_SEQS = 2048
STATUS_NAMES = {0: "QP_OK", 1: "QP_ERR_INVALID_ARG", 2: "QP_ERR_UNSUPPORTED", 3: "QP_ERR_BUDGET",
                4: "QP_ERR_WORKSPACE", 5: "QP_ERR_ALIGNMENT", 6: "QP_ERR_CUDA"}

EXPORTS = ["qp_status_string", "qp_n_keep", "qp_cache_layout", "qp_compress_workspace_bytes",
           "qp_decode_workspace_bytes", "qp_window_scores", "qp_select_topk", "qp_gather_quantize",
           "qp_compress_layer", "qp_decode_attn", "qp_decode_attn_layers", "qp_decode_attn_static",
           "qp_cache_layout_cap", "qp_append_kv", "qp_append_kv_layers", "qp_decode_attn_tail",
           "qp_decode_attn_tail_layers", "qp_compress_layers", "qp_decode_overlap", "qp_gather_quantize_ex",
           "qp_decode_attn_ex", "qp_decode_attn_layers_ex", "qp_head_budgets", "qp_head_budgets_workspace_bytes", "qp_debug_check",
           "qp_prompt_weights", "qp_prompt_weights_workspace_bytes", "qp_heavy_select", "qp_decode_attn_weights",
           "qp_decode_weights_workspace_bytes", "qp_evict_kv", "qp_decode_attn_tree", "qp_decode_tree_workspace_bytes", "qp_debug_give_up",
           "qp_rope_init", "qp_rope_freqs", "qp_rotary", "qp_paged_layout", "qp_paged_append", "qp_paged_attn",
           "qp_paged_attn_workspace_bytes"]


class QpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({status_string(status)})")


class qp_cache(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("bits", ctypes.c_int32), ("group", ctypes.c_int32),
                ("n_keep", ctypes.c_int32), ("n_cap", ctypes.c_int32),
                ("k_codes_bytes", ctypes.c_size_t), ("v_codes_bytes", ctypes.c_size_t),
                ("k_meta_bytes", ctypes.c_size_t), ("v_meta_bytes", ctypes.c_size_t),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("k_zero", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("v_zero", ctypes.c_void_p)]


class qp_side(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_int32), ("reserved_", ctypes.c_int32), ("idx", ctypes.c_void_p),
                ("val", ctypes.c_void_p), ("cnt", ctypes.c_void_p), ("tile_ptr", ctypes.c_void_p)]


class qp_strategy(ctypes.Structure):
    _fields_ = [("k_axis", ctypes.c_int32), ("outlier_threshold", ctypes.c_float),
                ("k_side", qp_side), ("v_side", qp_side)]


class qp_tail(ctypes.Structure):
    _fields_ = [("n_tail", ctypes.c_int32), ("reserved_", ctypes.c_int32),
                ("k_tail", ctypes.c_void_p), ("v_tail", ctypes.c_void_p)]


class qp_rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("factor", ctypes.c_float),
                ("reserved_", ctypes.c_int32), ("turn", ctypes.c_uint64 * 64)]


class qp_paged(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("format", ctypes.c_int32), ("page", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("codes_bytes", ctypes.c_size_t), ("scale_bytes", ctypes.c_size_t), ("tail_bytes", ctypes.c_size_t),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("k_tail", ctypes.c_void_p), ("v_tail", ctypes.c_void_p)]


class qp_step(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("max_new", ctypes.c_int32), ("start", ctypes.c_void_p),
                ("len", ctypes.c_void_p), ("pages", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded CUDA library.  Raises if it is missing: there is no fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2412_12706_b200.build` (needs nvcc, sm_100a)")
        L = ctypes.CDLL(LIB_PATH)
        i, i64, p, sz = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
        cp = ctypes.POINTER(qp_cache)
        L.qp_status_string.restype = ctypes.c_char_p
        L.qp_status_string.argtypes = [i]
        L.qp_n_keep.restype = i
        L.qp_n_keep.argtypes = [i64, i, i, i, i, ctypes.POINTER(ctypes.c_int32)]
        L.qp_cache_layout.restype = i
        L.qp_cache_layout.argtypes = [i, i, i, i, i, i, i, cp]
        L.qp_compress_workspace_bytes.restype = sz
        L.qp_compress_workspace_bytes.argtypes = [i, i, i, i, i, i]
        L.qp_decode_workspace_bytes.restype = sz
        L.qp_decode_workspace_bytes.argtypes = [cp]
        L.qp_window_scores.restype = i
        L.qp_window_scores.argtypes = [p, p, i, i, i, i, i, i, i, p, p, sz, p]
        L.qp_select_topk.restype = i
        L.qp_select_topk.argtypes = [p, i, i, i, i, i, p, p]
        L.qp_gather_quantize.restype = i
        L.qp_gather_quantize.argtypes = [p, p, p, i, cp, p]
        L.qp_compress_layer.restype = i
        L.qp_compress_layer.argtypes = [p, p, p, i, i, i, i, i, i, i64, i, i, i, cp, p, p, sz, p]
        L.qp_decode_attn.restype = i
        L.qp_decode_attn.argtypes = [p, cp, p, p, sz, p]
        L.qp_decode_attn_layers.restype = i
        L.qp_decode_attn_layers.argtypes = [i, ctypes.POINTER(p), cp, ctypes.POINTER(p), p, sz, p]
        L.qp_decode_attn_static.restype = i
        L.qp_decode_attn_static.argtypes = [p, cp, p, p]
        tp = ctypes.POINTER(qp_tail)
        L.qp_compress_layers.restype = i
        L.qp_compress_layers.argtypes = [i, ctypes.POINTER(p), ctypes.POINTER(p), ctypes.POINTER(p), i, i, i, i, i, i,
                                         ctypes.POINTER(i64), i, i, i, cp, ctypes.POINTER(p), p, sz, p]
        L.qp_cache_layout_cap.restype = i
        L.qp_cache_layout_cap.argtypes = [i, i, i, i, i, i, i, i, cp]
        L.qp_append_kv.restype = i
        L.qp_append_kv.argtypes = [p, p, cp, tp, p]
        L.qp_append_kv_layers.restype = i
        L.qp_append_kv_layers.argtypes = [i, ctypes.POINTER(p), ctypes.POINTER(p), cp, tp, p]
        L.qp_decode_attn_tail.restype = i
        L.qp_decode_attn_tail.argtypes = [p, cp, tp, p, p, sz, p]
        L.qp_decode_attn_tail_layers.restype = i
        L.qp_decode_attn_tail_layers.argtypes = [i, ctypes.POINTER(p), cp, tp, ctypes.POINTER(p), p, sz, p]
        sp = ctypes.POINTER(qp_strategy)
        L.qp_gather_quantize_ex.restype = i
        L.qp_gather_quantize_ex.argtypes = [p, p, p, i, cp, sp, p]
        L.qp_decode_attn_ex.restype = i
        L.qp_decode_attn_ex.argtypes = [p, cp, sp, p, p, sz, p]
        L.qp_decode_attn_layers_ex.restype = i
        L.qp_decode_attn_layers_ex.argtypes = [i, ctypes.POINTER(p), cp, sp, ctypes.POINTER(p), p, sz, p]
        L.qp_head_budgets_workspace_bytes.restype = sz
        L.qp_head_budgets_workspace_bytes.argtypes = [i, i, i, i, i]
        L.qp_head_budgets.restype = i
        L.qp_head_budgets.argtypes = [p, i, i, i, i, i, i, p, p, sz, p]
        L.qp_debug_check.restype = i
        L.qp_debug_check.argtypes = [ctypes.POINTER(ctypes.c_uint32)]
        L.qp_debug_give_up.restype = i
        L.qp_debug_give_up.argtypes = [i]
        L.qp_decode_overlap.restype = i
        L.qp_decode_overlap.argtypes = [p, i]
        L.qp_prompt_weights_workspace_bytes.restype = sz
        L.qp_prompt_weights_workspace_bytes.argtypes = [i] * 7
        L.qp_prompt_weights.restype = i
        L.qp_prompt_weights.argtypes = [p, p] + [i] * 8 + [p, p, sz, p]
        L.qp_heavy_select.restype = i
        L.qp_heavy_select.argtypes = [p] + [i] * 6 + [p, p, p, p]
        L.qp_decode_weights_workspace_bytes.restype = sz
        L.qp_decode_weights_workspace_bytes.argtypes = [cp]
        L.qp_decode_attn_weights.restype = i
        L.qp_decode_attn_weights.argtypes = [p, cp, sp, p, p, p, sz, p]
        L.qp_evict_kv.restype = i
        L.qp_evict_kv.argtypes = [p, p, cp, sp, p, p, i, i, p, p]
        L.qp_decode_tree_workspace_bytes.restype = sz
        L.qp_decode_tree_workspace_bytes.argtypes = [cp, i]
        L.qp_decode_attn_tree.restype = i
        L.qp_decode_attn_tree.argtypes = [p, i, cp, sp, tp, p, p, p, p, p, sz, p]
        rp, pp, st, dp = ctypes.POINTER(qp_rope), ctypes.POINTER(qp_paged), ctypes.POINTER(qp_step), ctypes.c_double
        L.qp_rope_init.restype = i
        L.qp_rope_init.argtypes = [i, i, dp, i, dp, i, rp]
        L.qp_rope_freqs.restype = i
        L.qp_rope_freqs.argtypes = [i, i, ctypes.POINTER(dp), ctypes.c_float, rp]
        L.qp_rotary.restype = i
        L.qp_rotary.argtypes = [p, ctypes.POINTER(i64), p, ctypes.POINTER(i64), i, i, i, i, p, i64, rp, i, p]
        L.qp_paged_layout.restype = i
        L.qp_paged_layout.argtypes = [i] * 8 + [pp]
        L.qp_paged_append.restype = i
        L.qp_paged_append.argtypes = [p, i64, p, i64, pp, st, rp, p, p, i64, p, p]
        L.qp_paged_attn_workspace_bytes.restype = sz
        L.qp_paged_attn_workspace_bytes.argtypes = [pp, i, i]
        L.qp_paged_attn.restype = i
        L.qp_paged_attn.argtypes = [p, i64, pp, st, p, p, sz, p]
        _lib = L
    return _lib


def _check(status: int, where: str) -> None:
    if status != QP_OK:
        raise QpError(status, where)


# the handle of torch's current stream without building a Stream object (3 us, as much as a launch)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def status_string(status: int) -> str:
    return lib().qp_status_string(status).decode()


def n_keep(budget_bits: int, bits: int, group: int, L: int, w: int) -> int:
    out = ctypes.c_int32(0)
    _check(lib().qp_n_keep(budget_bits, bits, group, L, w, ctypes.byref(out)), "qp_n_keep")
    return out.value


def cache_layout(batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, bits: int, group: int,
                 n_keep_: int) -> qp_cache:
    c = qp_cache()
    _check(lib().qp_cache_layout(batch, n_q_heads, n_kv_heads, head_dim, bits, group, n_keep_,
                                 ctypes.byref(c)), "qp_cache_layout")
    return c


def cache_layout_cap(batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, bits: int, group: int,
                     n_keep_: int, n_cap: int) -> qp_cache:
    c = qp_cache()
    _check(lib().qp_cache_layout_cap(batch, n_q_heads, n_kv_heads, head_dim, bits, group, n_keep_, n_cap,
                                     ctypes.byref(c)), "qp_cache_layout_cap")
    return c


def compress_workspace_bytes(batch, n_q_heads, n_kv_heads, head_dim, L, w) -> int:
    return int(lib().qp_compress_workspace_bytes(batch, n_q_heads, n_kv_heads, head_dim, L, w))


def decode_workspace_bytes(cache: "Cache | qp_cache") -> int:
    c = cache.desc if isinstance(cache, Cache) else cache
    return int(lib().qp_decode_workspace_bytes(ctypes.byref(c)))


@dataclass
class Cache:
    """Device buffers of one layer's packed cache plus the C descriptor that points at them."""
    desc: qp_cache
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scale: torch.Tensor | None
    k_zero: torch.Tensor | None
    v_scale: torch.Tensor | None
    v_zero: torch.Tensor | None

    @property
    def nbytes(self) -> int:
        d = self.desc
        return d.k_codes_bytes + d.v_codes_bytes + 2 * d.k_meta_bytes + 2 * d.v_meta_bytes


def alloc_cache(batch, n_q_heads, n_kv_heads, head_dim, bits, group, n_keep_, device="cuda",
                n_cap: int = 0) -> Cache:
    """Allocates the buffers of ``qp_cache_layout`` (``qp_cache_layout_cap`` when ``n_cap`` leaves room
    for appended tokens) with torch and fills in the pointers."""
    d = cache_layout_cap(batch, n_q_heads, n_kv_heads, head_dim, bits, group, n_keep_, n_cap)
    n, D, g = (n_cap or n_keep_), head_dim, group
    if bits == 16:
        kc = torch.empty((batch, n_kv_heads, n, D), dtype=torch.bfloat16, device=device)
        vc = torch.empty_like(kc)
        ks = kz = vs = vz = None
    else:
        wpg = g * bits // 32
        kc = torch.empty((batch, n_kv_heads, n // g, D, wpg), dtype=torch.int32, device=device)
        vc = torch.empty((batch, n_kv_heads, n, D // g, wpg), dtype=torch.int32, device=device)
        ks = torch.empty((batch, n_kv_heads, n // g, D), dtype=torch.float16, device=device)
        kz = torch.empty_like(ks)
        vs = torch.empty((batch, n_kv_heads, n, D // g), dtype=torch.float16, device=device)
        vz = torch.empty_like(vs)
    assert kc.numel() * kc.element_size() == d.k_codes_bytes and vc.numel() * vc.element_size() == d.v_codes_bytes
    d.k_codes, d.v_codes = _ptr(kc), _ptr(vc)
    d.k_scale, d.k_zero, d.v_scale, d.v_zero = _ptr(ks), _ptr(kz), _ptr(vs), _ptr(vz)
    return Cache(d, kc, vc, ks, kz, vs, vz)


def _dims(K: torch.Tensor, Q_win: torch.Tensor):
    Bt, Hkv, L, D = K.shape
    _, Hq, w, _ = Q_win.shape
    return Bt, Hq, Hkv, D, L, w


def _dev_bf16(t: torch.Tensor) -> None:
    assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous()


def window_scores(Q_win: torch.Tensor, K: torch.Tensor, pool: int = 7, workspace: torch.Tensor | None = None,
                  scores: torch.Tensor | None = None) -> torch.Tensor:
    _dev_bf16(Q_win); _dev_bf16(K)
    Bt, Hq, Hkv, D, L, w = _dims(K, Q_win)
    if scores is None:
        scores = torch.empty((Bt, Hkv, L - w), dtype=torch.float32, device=K.device)
    if workspace is None:
        workspace = torch.empty(max(16, compress_workspace_bytes(Bt, Hq, Hkv, D, L, w)), dtype=torch.uint8,
                                device=K.device)
    _check(lib().qp_window_scores(_ptr(Q_win), _ptr(K), Bt, Hq, Hkv, D, L, w, pool, _ptr(scores),
                                  _ptr(workspace), workspace.numel(), _stream()), "qp_window_scores")
    return scores


def select_topk(scores: torch.Tensor, L: int, w: int, n_keep_: int,
                kept_idx: torch.Tensor | None = None) -> torch.Tensor:
    assert scores.is_cuda and scores.dtype == torch.float32 and scores.is_contiguous()
    Bt, Hkv, P = scores.shape
    assert P == L - w
    if kept_idx is None:
        kept_idx = torch.empty((Bt, Hkv, n_keep_), dtype=torch.int32, device=scores.device)
    _check(lib().qp_select_topk(_ptr(scores), Bt, Hkv, L, w, n_keep_, _ptr(kept_idx), _stream()),
           "qp_select_topk")
    return kept_idx


def gather_quantize(K: torch.Tensor, V: torch.Tensor, kept_idx: torch.Tensor, cache: Cache) -> Cache:
    _dev_bf16(K); _dev_bf16(V)
    assert kept_idx.is_cuda and kept_idx.dtype == torch.int32 and kept_idx.is_contiguous()
    _check(lib().qp_gather_quantize(_ptr(K), _ptr(V), _ptr(kept_idx), K.shape[2], ctypes.byref(cache.desc),
                                    _stream()), "qp_gather_quantize")
    return cache


def compress_layer(K: torch.Tensor, V: torch.Tensor, Q_win: torch.Tensor, budget_bits: int, bits: int,
                   group: int = 32, pool: int = 7, cache: Cache | None = None,
                   kept_idx: torch.Tensor | None = None, workspace: torch.Tensor | None = None, n_cap: int = 0):
    """qp_compress_layer: returns (cache, kept_idx).  Buffers are allocated with torch when not given
    (with room for ``n_cap`` tokens per KV head when ``n_cap`` is given)."""
    _dev_bf16(K); _dev_bf16(V); _dev_bf16(Q_win)
    Bt, Hq, Hkv, D, L, w = _dims(K, Q_win)
    n = n_keep(budget_bits, bits, group, L, w)
    if cache is None:
        cache = alloc_cache(Bt, Hq, Hkv, D, bits, group, n, K.device, n_cap)
    if kept_idx is None:
        kept_idx = torch.empty((Bt, Hkv, n), dtype=torch.int32, device=K.device)
    if workspace is None:
        workspace = torch.empty(max(16, compress_workspace_bytes(Bt, Hq, Hkv, D, L, w)), dtype=torch.uint8,
                                device=K.device)
    _check(lib().qp_compress_layer(_ptr(K), _ptr(V), _ptr(Q_win), Bt, Hq, Hkv, D, L, w, budget_bits, bits,
                                   group, pool, ctypes.byref(cache.desc), _ptr(kept_idx), _ptr(workspace),
                                   workspace.numel(), _stream()), "qp_compress_layer")
    return cache, kept_idx


def compress_layers(Ks: list[torch.Tensor], Vs: list[torch.Tensor], Q_wins: list[torch.Tensor], budget_bits: list[int],
                    bits: int, group: int = 32, pool: int = 7, caches: list[Cache] | None = None,
                    kept_idx: list[torch.Tensor] | None = None, workspace: torch.Tensor | None = None):
    """qp_compress_layers: the prefill-side path of several layers of one shape, one launch per stage.
    Returns (caches, kept_idx); buffers are allocated with torch when not given."""
    nl = len(Ks)
    assert 1 <= nl <= QP_MAX_LAYERS and len(Vs) == nl and len(Q_wins) == nl and len(budget_bits) == nl
    for t in (*Ks, *Vs, *Q_wins):
        _dev_bf16(t)
    Bt, Hq, Hkv, D, L, w = _dims(Ks[0], Q_wins[0])
    ns = [n_keep(b, bits, group, L, w) for b in budget_bits]
    dev = Ks[0].device
    if caches is None:
        caches = [alloc_cache(Bt, Hq, Hkv, D, bits, group, n, dev) for n in ns]
    if kept_idx is None:
        kept_idx = [torch.empty((Bt, Hkv, n), dtype=torch.int32, device=dev) for n in ns]
    if workspace is None:
        workspace = torch.empty(max(16, compress_workspace_bytes(Bt * nl, Hq, Hkv, D, L, w)), dtype=torch.uint8, device=dev)
    arr = lambda ts: (ctypes.c_void_p * nl)(*[t.data_ptr() for t in ts])
    _check(lib().qp_compress_layers(nl, arr(Ks), arr(Vs), arr(Q_wins), Bt, Hq, Hkv, D, L, w,
                                    (ctypes.c_int64 * nl)(*budget_bits), bits, group, pool,
                                    (qp_cache * nl)(*[c.desc for c in caches]), arr(kept_idx), _ptr(workspace),
                                    workspace.numel(), _stream()), "qp_compress_layers")
    return caches, kept_idx


def new_decode_workspace(nbytes: int, device) -> torch.Tensor:
    """Scratch for the decode calls (contents irrelevant); reuse one per stream across calls."""
    return torch.empty(max(16, nbytes), dtype=torch.uint8, device=device)


def decode_attn(q: torch.Tensor, cache: Cache, out: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None) -> torch.Tensor:
    _dev_bf16(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_decode_workspace(decode_workspace_bytes(cache), q.device)
    _check(lib().qp_decode_attn(_ptr(q), ctypes.byref(cache.desc), _ptr(out), _ptr(workspace),
                                workspace.numel(), _stream()), "qp_decode_attn")
    return out


def decode_overlap(enable: bool) -> None:
    """qp_decode_overlap for torch's current stream: let consecutive decode calls on it overlap on the GPU
    (see include/qp.h for what the caller promises while it is on).  Off by default."""
    _check(lib().qp_decode_overlap(_stream(), 1 if enable else 0), "qp_decode_overlap")


class LayerBatch:
    """Marshalled host arrays for ``qp_decode_attn_layers`` (built once, reused every step)."""

    def __init__(self, qs: list[torch.Tensor], caches: list[Cache], outs: list[torch.Tensor],
                 workspace: torch.Tensor | None = None):
        n = len(caches)
        assert 1 <= n <= QP_MAX_LAYERS and len(qs) == n and len(outs) == n
        self.n = n
        self.keep = (qs, caches, outs)
        self.q_arr = (ctypes.c_void_p * n)(*[t.data_ptr() for t in qs])
        self.out_arr = (ctypes.c_void_p * n)(*[t.data_ptr() for t in outs])
        self.cache_arr = (qp_cache * n)(*[c.desc for c in caches])
        if workspace is None:
            workspace = new_decode_workspace(sum(decode_workspace_bytes(c) for c in caches), qs[0].device)
        self.workspace = workspace


def decode_attn_layers(batch: LayerBatch) -> None:
    _check(lib().qp_decode_attn_layers(batch.n, batch.q_arr, batch.cache_arr, batch.out_arr,
                                       _ptr(batch.workspace), batch.workspace.numel(), _stream()),
           "qp_decode_attn_layers")


@dataclass
class Tail:
    """Device buffers of one layer's unquantized tail plus the C descriptor (host state: n_tail)."""
    desc: qp_tail
    k_tail: torch.Tensor | None
    v_tail: torch.Tensor | None


def alloc_tail(cache: Cache, device=None) -> Tail:
    """bf16 [Bt,Hkv,group,D] buffers for the tokens that wait for a full group (none at 16 bit)."""
    d = cache.desc
    t = qp_tail()
    if d.bits == 16:
        return Tail(t, None, None)
    device = device or cache.k_codes.device
    kt = torch.zeros((d.batch, d.n_kv_heads, d.group, d.head_dim), dtype=torch.bfloat16, device=device)
    vt = torch.zeros_like(kt)
    t.k_tail, t.v_tail = _ptr(kt), _ptr(vt)
    return Tail(t, kt, vt)


def append_kv(k_new: torch.Tensor, v_new: torch.Tensor, cache: Cache, tail: Tail) -> None:
    """qp_append_kv: Eq. 2 for one layer; updates cache.desc.n_keep and tail.desc.n_tail."""
    _dev_bf16(k_new); _dev_bf16(v_new)
    _check(lib().qp_append_kv(_ptr(k_new), _ptr(v_new), ctypes.byref(cache.desc), ctypes.byref(tail.desc),
                              _stream()), "qp_append_kv")


def decode_attn_tail(q: torch.Tensor, cache: Cache, tail: Tail, out: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None) -> torch.Tensor:
    _dev_bf16(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_decode_workspace(decode_workspace_bytes(cache), q.device)
    _check(lib().qp_decode_attn_tail(_ptr(q), ctypes.byref(cache.desc), ctypes.byref(tail.desc), _ptr(out),
                                     _ptr(workspace), workspace.numel(), _stream()), "qp_decode_attn_tail")
    return out


class GenBatch:
    """Marshalled host arrays for a generation loop over many layers: ``qp_append_kv_layers`` followed by
    ``qp_decode_attn_tail_layers``.  The descriptor arrays are owned here and updated in place by the
    append call (the Cache / Tail objects passed in keep their initial descriptors)."""

    def __init__(self, qs, k_news, v_news, caches: list[Cache], tails: list[Tail], outs,
                 workspace: torch.Tensor | None = None):
        n = len(caches)
        assert 1 <= n <= QP_MAX_LAYERS and len(qs) == len(outs) == len(tails) == len(k_news) == len(v_news) == n
        self.n = n
        self.keep = (qs, k_news, v_news, caches, tails, outs)
        arr = lambda ts: (ctypes.c_void_p * n)(*[t.data_ptr() for t in ts])
        self.q_arr, self.out_arr, self.kn_arr, self.vn_arr = arr(qs), arr(outs), arr(k_news), arr(v_news)
        self.cache_arr = (qp_cache * n)(*[c.desc for c in caches])
        self.tail_arr = (qp_tail * n)(*[t.desc for t in tails])
        if workspace is None:
            workspace = new_decode_workspace(sum(decode_workspace_bytes(c) for c in caches), qs[0].device)
        self.workspace = workspace


def append_kv_layers(batch: GenBatch) -> None:
    _check(lib().qp_append_kv_layers(batch.n, batch.kn_arr, batch.vn_arr, batch.cache_arr, batch.tail_arr,
                                     _stream()), "qp_append_kv_layers")


def decode_attn_tail_layers(batch: GenBatch) -> None:
    _check(lib().qp_decode_attn_tail_layers(batch.n, batch.q_arr, batch.cache_arr, batch.tail_arr, batch.out_arr,
                                            _ptr(batch.workspace), batch.workspace.numel(), _stream()),
           "qp_decode_attn_tail_layers")


STATIC_SCRATCH_BYTES = 4 << 20


def decode_attn_static(q: torch.Tensor, cache: Cache, out: torch.Tensor | None = None) -> torch.Tensor:
    """qp_decode_attn_static: decode attention whose split partials live in the library's built-in
    scratch array, for hosts that cannot hand the library any temporary device memory.  Only
    ``out`` is allocated here (by torch) when the caller passes none; the C call allocates nothing.
    Raises QpError(QP_ERR_WORKSPACE) when the cache needs more than STATIC_SCRATCH_BYTES of scratch.
    Calls on one device share that array: do not let two of them overlap on the GPU."""
    _dev_bf16(q)
    if out is None:
        out = torch.empty_like(q)
    st = lib().qp_decode_attn_static(_ptr(q), ctypes.byref(cache.desc), _ptr(out), _stream())
    if st == 4:
        raise QpError(st, f"qp_decode_attn_static: this cache needs more than the built-in "
                          f"{STATIC_SCRATCH_BYTES} bytes of scratch; use qp_decode_attn with a workspace")
    _check(st, "qp_decode_attn_static")
    return out


@dataclass
class Strategy:
    """A quantization strategy of Sec. 5.3 (qp_strategy) with torch-owned side-list buffers."""
    desc: qp_strategy
    bufs: list


def make_strategy(cache: Cache, k_axis: int = 0, outlier_threshold: float | None = None, cap: int | None = None) -> Strategy:
    """Fills a qp_strategy; with filtering on, allocates the two side lists for `cache` (cap entries per
    (batch, KV head), default 4 % of the head's elements)."""
    d = cache.desc
    s = qp_strategy()
    s.k_axis = k_axis
    s.outlier_threshold = float(outlier_threshold) if outlier_threshold else 0.0
    bufs = []
    if outlier_threshold:
        n = d.n_cap or d.n_keep
        cap = cap or max(64, n * d.head_dim // 25)
        dev = cache.k_codes.device
        for side in (s.k_side, s.v_side):
            idx = torch.zeros((d.batch, d.n_kv_heads, cap), dtype=torch.int32, device=dev)
            val = torch.zeros((d.batch, d.n_kv_heads, cap), dtype=torch.bfloat16, device=dev)
            cnt = torch.zeros((d.batch, d.n_kv_heads), dtype=torch.int32, device=dev)
            tp = torch.zeros((d.batch, d.n_kv_heads, (n + 31) // 32 + 1), dtype=torch.int32, device=dev)
            side.cap, side.idx, side.val, side.cnt, side.tile_ptr = cap, _ptr(idx), _ptr(val), _ptr(cnt), _ptr(tp)
            bufs.append((idx, val, cnt, tp))
    return Strategy(s, bufs)


def gather_quantize_ex(K: torch.Tensor, V: torch.Tensor, kept_idx: torch.Tensor, cache: Cache, strategy: Strategy) -> Cache:
    _dev_bf16(K); _dev_bf16(V)
    assert kept_idx.is_cuda and kept_idx.dtype == torch.int32 and kept_idx.is_contiguous()
    _check(lib().qp_gather_quantize_ex(_ptr(K), _ptr(V), _ptr(kept_idx), K.shape[2], ctypes.byref(cache.desc),
                                       ctypes.byref(strategy.desc), _stream()), "qp_gather_quantize_ex")
    return cache


def decode_attn_ex(q: torch.Tensor, cache: Cache, strategy: Strategy, out: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None) -> torch.Tensor:
    _dev_bf16(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_decode_workspace(decode_workspace_bytes(cache), q.device)
    _check(lib().qp_decode_attn_ex(_ptr(q), ctypes.byref(cache.desc), ctypes.byref(strategy.desc), _ptr(out),
                                   _ptr(workspace), workspace.numel(), _stream()), "qp_decode_attn_ex")
    return out


def decode_attn_layers_ex(qs: list[torch.Tensor], caches: list[Cache], strategy: Strategy, outs: list[torch.Tensor],
                          workspace: torch.Tensor | None = None) -> None:
    n = len(caches)
    assert 1 <= n <= QP_MAX_LAYERS and len(qs) == n and len(outs) == n
    if workspace is None:
        workspace = new_decode_workspace(sum(decode_workspace_bytes(c) for c in caches), qs[0].device)
    arr = lambda ts: (ctypes.c_void_p * n)(*[t.data_ptr() for t in ts])
    _check(lib().qp_decode_attn_layers_ex(n, arr(qs), (qp_cache * n)(*[c.desc for c in caches]),
                                          ctypes.byref(strategy.desc), arr(outs), _ptr(workspace), workspace.numel(),
                                          _stream()), "qp_decode_attn_layers_ex")


def head_budgets(scores: torch.Tensor, L: int, w: int, n_mean: int, unit: int = 32) -> torch.Tensor:
    """qp_head_budgets: scores fp32 [Bt,Hkv,P] (device) -> tokens kept per KV head, int32 [Bt,Hkv] (device)."""
    assert scores.is_cuda and scores.dtype == torch.float32 and scores.is_contiguous()
    Bt, Hkv, P = scores.shape
    assert P == L - w
    out = torch.empty((Bt, Hkv), dtype=torch.int32, device=scores.device)
    ws = torch.empty(max(16, int(lib().qp_head_budgets_workspace_bytes(Bt, Hkv, L, w, n_mean))), dtype=torch.uint8,
                     device=scores.device)
    _check(lib().qp_head_budgets(_ptr(scores), Bt, Hkv, L, w, n_mean, unit, _ptr(out), _ptr(ws), ws.numel(), _stream()),
           "qp_head_budgets")
    return out


@dataclass
class HeadCaches:
    """One packed cache per (batch, KV head) of a layer pruned with head-level budgets (descriptors with
    batch = 1, n_kv_heads = 1, n_q_heads = G), in (batch, head) order, and the strategy they were written with."""
    caches: list
    kept: list
    n_heads: list            # tokens kept per (batch, KV head), host ints
    strategy: "Strategy | None"
    shape: tuple             # (Bt, Hq, Hkv, D)


def compress_layer_heads(K: torch.Tensor, V: torch.Tensor, Q_win: torch.Tensor, n_mean: int, bits: int, group: int = 32,
                         pool: int = 7, k_axis: int = 1, unit: int | None = None) -> HeadCaches:
    """The prefill-side path with head-level budgets: qp_window_scores -> qp_head_budgets -> (one copy of the
    Bt x Hkv counts to the host, to size the heads' caches) -> per head qp_select_topk and
    qp_gather_quantize(_ex).  k_axis = 1: keys per token, the arrangement the paper pairs with these methods;
    k_axis = 0: the main path's per-channel keys (unit must then be a multiple of the group)."""
    _dev_bf16(K); _dev_bf16(V); _dev_bf16(Q_win)
    Bt, Hq, Hkv, D, L, w = _dims(K, Q_win)
    G = Hq // Hkv
    unit = unit or group
    scores = window_scores(Q_win, K, pool)
    n_dev = head_budgets(scores, L, w, n_mean, unit)
    n_host = n_dev.cpu().view(-1).tolist()             # the one host round trip of this path
    caches, kepts = [], []
    strategy = None
    for i, n in enumerate(n_host):
        b, h = divmod(i, Hkv)
        c = alloc_cache(1, G, 1, D, bits, group, n, K.device)
        kept = torch.empty((1, 1, n), dtype=torch.int32, device=K.device)
        _check(lib().qp_select_topk(scores[b, h].data_ptr(), 1, 1, L, w, n, _ptr(kept), _stream()), "qp_select_topk")
        if bits == 16 or k_axis == 0:
            _check(lib().qp_gather_quantize(K[b, h].data_ptr(), V[b, h].data_ptr(), _ptr(kept), L, ctypes.byref(c.desc),
                                            _stream()), "qp_gather_quantize")
        else:
            strategy = strategy or make_strategy(c, 1, None)
            _check(lib().qp_gather_quantize_ex(K[b, h].data_ptr(), V[b, h].data_ptr(), _ptr(kept), L, ctypes.byref(c.desc),
                                               ctypes.byref(strategy.desc), _stream()), "qp_gather_quantize_ex")
        caches.append(c); kepts.append(kept)
    return HeadCaches(caches, kepts, n_host, strategy, (Bt, Hq, Hkv, D))


def decode_attn_heads(q: torch.Tensor, hc: HeadCaches, out: torch.Tensor | None = None) -> torch.Tensor:
    """Decode attention over the per-head caches of compress_layer_heads: q, out bf16 [Bt,Hq,D]; every head is one
    entry of a multi-cache call (qp_decode_attn_layers, or qp_decode_attn_layers_ex for per-token keys)."""
    _dev_bf16(q)
    Bt, Hq, Hkv, D = hc.shape
    G = Hq // Hkv
    if out is None:
        out = torch.empty_like(q)
    qv, ov = q.view(Bt * Hkv, 1, G, D), out.view(Bt * Hkv, 1, G, D)
    for lo in range(0, len(hc.caches), QP_MAX_LAYERS):
        hi = min(len(hc.caches), lo + QP_MAX_LAYERS)
        qs, outs = [qv[i] for i in range(lo, hi)], [ov[i] for i in range(lo, hi)]
        if hc.strategy is None:
            decode_attn_layers(LayerBatch(qs, hc.caches[lo:hi], outs))
        else:
            decode_attn_layers_ex(qs, hc.caches[lo:hi], hc.strategy, outs)
    return out


def prompt_weights_workspace_bytes(batch, n_q_heads, n_kv_heads, head_dim, L, q_start, n_q) -> int:
    return int(lib().qp_prompt_weights_workspace_bytes(batch, n_q_heads, n_kv_heads, head_dim, L, q_start, n_q))


def decode_weights_workspace_bytes(cache: "Cache | qp_cache") -> int:
    return int(lib().qp_decode_weights_workspace_bytes(ctypes.byref(cache.desc if isinstance(cache, Cache) else cache)))


def decode_tree_workspace_bytes(cache: "Cache | qp_cache", T: int) -> int:
    return int(lib().qp_decode_tree_workspace_bytes(ctypes.byref(cache.desc if isinstance(cache, Cache) else cache), T))


def _dev(t: torch.Tensor, dtype: torch.dtype, shape: tuple) -> None:
    """Contiguous, of this type and shape, and on the device the kernels are launched on."""
    assert (t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.is_cuda
            and t.get_device() == _current_device()), (t.device, t.dtype, t.shape, shape)


def _scratch(t: torch.Tensor) -> tuple:
    """Address and bytes of a workspace: contiguous, of any type, and on the device the kernels are launched on."""
    assert t.get_device() == _current_device() and t.is_contiguous(), (t.device, t.shape)
    return t.data_ptr(), t.numel() * t.element_size()


def _dev_cache(cache: Cache) -> None:
    assert cache.k_codes.get_device() == _current_device(), "cache not on the current device"


def _ref(strategy: "Strategy | None"):
    return None if strategy is None else ctypes.byref(strategy.desc)


def _state_shape(cache: Cache) -> tuple:
    d = cache.desc
    return d.batch, d.n_kv_heads, d.n_cap or d.n_keep


def prompt_weights(Q: torch.Tensor, K: torch.Tensor, q_start: int = 0, weights: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None) -> torch.Tensor:
    """qp_prompt_weights: the attention weight each key of K [Bt,Hkv,L,D] has received from the query rows Q [Bt,Hq,n_q,D] at
    positions q_start .. q_start+n_q-1, fp32 [Bt,Hkv,L].  Given ``weights`` they are added to (a prompt in chunks)."""
    Bt, Hkv, L, D = K.shape
    _, Hq, nq, _ = Q.shape
    _dev(Q, torch.bfloat16, (Bt, Hq, nq, D)); _dev(K, torch.bfloat16, (Bt, Hkv, L, D))
    accumulate = weights is not None
    if weights is None:
        weights = torch.empty((Bt, Hkv, L), dtype=torch.float32, device=K.device)
    _dev(weights, torch.float32, (Bt, Hkv, L))
    if workspace is None:
        workspace = torch.empty(max(16, prompt_weights_workspace_bytes(Bt, Hq, Hkv, D, L, q_start, nq)), dtype=torch.uint8,
                                device=K.device)
    _check(lib().qp_prompt_weights(_ptr(Q), _ptr(K), Bt, Hq, Hkv, D, L, q_start, nq, 1 if accumulate else 0, _ptr(weights),
                                   *_scratch(workspace), _stream()), "qp_prompt_weights")
    return weights


def heavy_select(weights: torch.Tensor, w: int, n_keep_: int, n_cap: int = 0):
    """qp_heavy_select: weights fp32 [Bt,Hkv,L] -> (kept_idx int32 [Bt,Hkv,n_keep], weights fp32 and positions int32
    [Bt,Hkv,n_cap] of a cache that holds these tokens)."""
    Bt, Hkv, L = weights.shape
    _dev(weights, torch.float32, (Bt, Hkv, L))
    cap = n_cap or n_keep_
    kept = torch.empty((Bt, Hkv, n_keep_), dtype=torch.int32, device=weights.device)
    kw, kp = weights.new_empty((Bt, Hkv, cap)), kept.new_empty((Bt, Hkv, cap))
    _check(lib().qp_heavy_select(_ptr(weights), Bt, Hkv, L, w, n_keep_, cap, _ptr(kept), _ptr(kw), _ptr(kp), _stream()),
           "qp_heavy_select")
    return kept, kw, kp


def decode_attn_weights(q: torch.Tensor, cache: Cache, weights: torch.Tensor, strategy: "Strategy | None" = None,
                        out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """qp_decode_attn_weights: decode attention that adds its softmax weights, summed over a KV head's query heads, to
    ``weights`` fp32 [Bt,Hkv,n_cap] in place."""
    d = cache.desc
    _dev(q, torch.bfloat16, (d.batch, d.n_q_heads, d.head_dim))
    _dev(weights, torch.float32, _state_shape(cache))
    _dev_cache(cache)
    if out is None:
        out = torch.empty_like(q)
    else:
        _dev(out, torch.bfloat16, q.shape)
    if workspace is None:
        workspace = new_decode_workspace(decode_weights_workspace_bytes(cache), q.device)
    _check(lib().qp_decode_attn_weights(_ptr(q), ctypes.byref(d), _ref(strategy), _ptr(weights), _ptr(out), *_scratch(workspace),
                                        _stream()), "qp_decode_attn_weights")
    return out


def evict_kv(k_new: torch.Tensor, v_new: torch.Tensor, cache: Cache, weights: torch.Tensor, pos: torch.Tensor, new_pos: int,
             recent: int, strategy: "Strategy | None" = None, slots: torch.Tensor | None = None) -> torch.Tensor:
    """qp_evict_kv: the new token's rows [Bt,Hkv,D] take the slot of the lightest token that is not among the ``recent`` last
    positions (a 16-bit cache with room grows first); returns the slots int32 [Bt,Hkv].  cache, weights and pos are updated."""
    d = cache.desc
    Bt, Hkv = d.batch, d.n_kv_heads
    row, state = (Bt, Hkv, d.head_dim), (Bt, Hkv, d.n_cap or d.n_keep)
    _dev(k_new, torch.bfloat16, row); _dev(v_new, torch.bfloat16, row)
    _dev(weights, torch.float32, state); _dev(pos, torch.int32, state)
    _dev_cache(cache)
    if slots is None:
        slots = pos.new_empty((Bt, Hkv))
    else:
        _dev(slots, torch.int32, (Bt, Hkv))
    status = lib().qp_evict_kv(k_new.data_ptr(), v_new.data_ptr(), ctypes.byref(d), _ref(strategy), weights.data_ptr(),
                               pos.data_ptr(), new_pos, recent, slots.data_ptr(), _stream())
    if status:
        _check(status, "qp_evict_kv")
    return slots


@dataclass
class HeavyCache:
    """A cache kept at a fixed budget by accumulated attention weight, with its tokens' weights and positions."""
    cache: Cache
    strategy: "Strategy | None"
    weights: torch.Tensor    # fp32 [Bt,Hkv,n_cap]
    pos: torch.Tensor        # int32 [Bt,Hkv,n_cap]
    next_pos: int            # position of the next token


def compress_layer_heavy(K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, budget_bits: int, bits: int, group: int = 32,
                         recent: int = 32, n_cap: int = 0) -> HeavyCache:
    """The prefill-side path with accumulated weights in place of the observation window: qp_prompt_weights over all queries
    Q [Bt,Hq,L,D] -> qp_heavy_select -> qp_gather_quantize (16 bit) or qp_gather_quantize_ex with per-token keys."""
    Bt, Hkv, L, D = K.shape
    for t, heads in ((K, Hkv), (V, Hkv), (Q, Q.shape[1])):
        _dev(t, torch.bfloat16, (Bt, heads, L, D))
    n = n_keep(budget_bits, bits, group, L, recent)
    received = prompt_weights(Q, K)
    kept, weights, pos = heavy_select(received, recent, n, n_cap)
    cache = alloc_cache(Bt, Q.shape[1], Hkv, D, bits, group, n, K.device, n_cap)
    strategy = None
    if bits == 16:
        gather_quantize(K, V, kept, cache)
    else:
        strategy = make_strategy(cache, 1, None)
        gather_quantize_ex(K, V, kept, cache, strategy)
    return HeavyCache(cache, strategy, weights, pos, L)


def decode_step_heavy(q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, hc: HeavyCache, recent: int = 32,
                      out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """One generation step over a HeavyCache: qp_evict_kv, then qp_decode_attn_weights (the new token sees itself).  A step that
    is refused has changed nothing: what the second call asks for is looked at before the first takes the token in."""
    d = hc.cache.desc
    _dev(q, torch.bfloat16, (d.batch, d.n_q_heads, d.head_dim))
    if out is None:
        out = torch.empty_like(q)
    else:
        _dev(out, torch.bfloat16, q.shape)
    need = decode_weights_workspace_bytes(hc.cache)
    if workspace is None:
        workspace = new_decode_workspace(need, q.device)
    address, size = _scratch(workspace)
    if d.batch * d.n_kv_heads > 65535:
        raise QpError(2, "decode_step_heavy")
    if size < need:
        raise QpError(4, "decode_step_heavy")
    if (address | q.data_ptr() | out.data_ptr()) & 15:
        raise QpError(5, "decode_step_heavy")
    evict_kv(k_new, v_new, hc.cache, hc.weights, hc.pos, hc.next_pos, recent, hc.strategy)
    hc.next_pos += 1
    return decode_attn_weights(q, hc.cache, hc.weights, hc.strategy, out, workspace)


def tree_mask(parents: torch.Tensor) -> torch.Tensor:
    """Masks of a drafted tree for decode_attn_tree: parents int [Bt,T], parents[b,i] < i the node draft i hangs on, or -1 for
    the context -> int64 [Bt,T], bit j of mask[b,i] set for i itself and its ancestors.  Tensor code that waits for the device to
    look at the parents (not for a capture): a tree whose shape does not change from step to step needs it once."""
    Bt, T = parents.shape
    assert 1 <= T <= QP_MAX_DRAFTS
    i = torch.arange(T, device=parents.device)
    if not bool(((parents >= -1) & (parents < i)).all()):
        raise ValueError("every node hangs on an earlier one, or on the context (-1)")
    own, up = (torch.ones_like(i) << i).expand(Bt, T), parents.long()
    mask = own.clone()
    for _ in range(6):                                # after r rounds a mask spans 2^r levels; 2^6 = QP_MAX_DRAFTS
        above = torch.gather(mask, 1, up.clamp(min=0))
        mask = torch.where(up >= 0, mask | above, mask)
        up = torch.where(up >= 0, torch.gather(up, 1, up.clamp(min=0)), up)
    return mask


def decode_attn_tree(q: torch.Tensor, cache: Cache, k_draft: torch.Tensor, v_draft: torch.Tensor, mask: torch.Tensor,
                     tail: "Tail | None" = None, strategy: "Strategy | None" = None, out: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None) -> torch.Tensor:
    """qp_decode_attn_tree: q [Bt,T,Hq,D], drafts [Bt,T,Hkv,D], mask int64 [Bt,T] (see tree_mask) -> out [Bt,T,Hq,D]."""
    d = cache.desc
    T = q.shape[1]
    _dev(q, torch.bfloat16, (d.batch, T, d.n_q_heads, d.head_dim))
    for t in (k_draft, v_draft):
        _dev(t, torch.bfloat16, (d.batch, T, d.n_kv_heads, d.head_dim))
    _dev(mask, torch.int64, (d.batch, T))
    _dev_cache(cache)
    if tail is not None and tail.desc.n_tail and d.bits < 16:      # (an empty one needs no arrays)
        for t in (tail.k_tail, tail.v_tail):
            _dev(t, torch.bfloat16, (d.batch, d.n_kv_heads, d.group, d.head_dim))
    if out is None:
        out = torch.empty_like(q)
    else:
        _dev(out, torch.bfloat16, q.shape)
    if workspace is None:
        workspace = new_decode_workspace(decode_tree_workspace_bytes(cache, T), q.device)
    _check(lib().qp_decode_attn_tree(_ptr(q), T, ctypes.byref(d), _ref(strategy), None if tail is None else ctypes.byref(tail.desc),
                                     _ptr(k_draft), _ptr(v_draft), _ptr(mask), _ptr(out), *_scratch(workspace), _stream()),
           "qp_decode_attn_tree")
    return out


ROPE_KINDS = {"plain": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}
PAGED_FORMATS = {torch.float8_e4m3fn: 0, torch.int8: 1}


def rope(rot_dim: int, base: float = 10000.0, interleaved: bool = False, scaling: str = "plain", factor: float = 1.0,
         trained_len: int = 8192, freqs=None) -> qp_rope:
    """qp_rope_init: the rotation of ``rot_dim`` channels by position, plain or scaled for long contexts ("linear", "ntk", "yarn",
    "bands"); with ``freqs`` (rot_dim/2 numbers, radians a position) qp_rope_freqs, ``factor`` being what the rotated channels are
    multiplied by."""
    r = qp_rope()
    if freqs is not None:
        if len(freqs) != rot_dim // 2:
            raise ValueError("one frequency for each pair of channels")
        w = (ctypes.c_double * max(1, len(freqs)))(*[float(x) for x in freqs])
        _check(lib().qp_rope_freqs(rot_dim, int(interleaved), w, factor, ctypes.byref(r)), "qp_rope_freqs")
    else:
        _check(lib().qp_rope_init(rot_dim, int(interleaved), base, ROPE_KINDS[scaling], factor, trained_len, ctypes.byref(r)),
               "qp_rope_init")
    return r


_contiguous, _empty_like, _bf16, _int32 = torch.contiguous_format, torch.empty_like, torch.bfloat16, torch.int32


@functools.lru_cache(maxsize=256)
def _int64x3(a: int, b: int, c: int):
    """A host array of these numbers for the library to read."""
    return (ctypes.c_int64 * 3)(a, b, c)


def _strides(t: torch.Tensor, b: int, h: int, n: int, device: int):
    """Strides of batch, head and token as qp_rotary takes them (0 where there is one only)."""
    sb, sh, sn, sd = t.stride()
    assert t.dtype is _bf16 and t.get_device() == device and sd == 1, (t.device, t.dtype, t.stride())
    return _int64x3(sb if b > 1 else 0, sh if h > 1 else 0, sn if n > 1 else 0)


def rotary(x: torch.Tensor, pos: torch.Tensor, rope_: qp_rope, out: torch.Tensor | None = None, transpose: bool = False) -> torch.Tensor:
    """qp_rotary: x [Bt,H,L,D] (any strides that keep a row's channels together: rows of a fused projection, seen head by head, do)
    rotated by pos int32 [L] or [Bt,L]; ``out`` may be x.  transpose: by the negative angles (the gradient; the way back where the
    rotation has no factor)."""
    Bt, H, L, D = x.shape
    device = _current_device()
    xs = _strides(x, Bt, H, L, device)
    if out is None:
        out = _empty_like(x, memory_format=_contiguous)
        to = _int64x3(H * L * D, L * D, D)
    else:
        assert out.shape == x.shape
        to = _strides(out, Bt, H, L, device)
        assert (to[0] or Bt == 1) and (to[1] or H == 1) and (to[2] or L == 1), "rows of out overlap"
    if pos.dim() == 1:
        _dev(pos, _int32, (L,))
        ps = 0
    else:
        _dev(pos, _int32, (Bt, L))
        ps = L
    status = lib().qp_rotary(x.data_ptr(), xs, out.data_ptr(), to, Bt, H, L, D, pos.data_ptr(), ps, ctypes.byref(rope_), int(transpose), _stream())
    if status:
        _check(status, "qp_rotary")
    return out


def compress_layer_rotary(K: torch.Tensor, V: torch.Tensor, Q_win: torch.Tensor, rope_: qp_rope, budget_bits: int, bits: int,
                          group: int = 32, pool: int = 7, first_pos: int = 0, **kw):
    """compress_layer for a prompt as it leaves the projections: K [Bt,Hkv,L,D] and Q_win [Bt,Hq,w,D] (any strides, see rotary) are
    rotated first, at positions first_pos .. first_pos+L-1, the window's at the last w of them."""
    L, w = K.shape[2], Q_win.shape[2]
    pos = torch.arange(first_pos, first_pos + L, dtype=torch.int32, device=K.device)
    return compress_layer(rotary(K, pos, rope_), V, rotary(Q_win, pos[L - w:], rope_), budget_bits, bits, group, pool, **kw)


@dataclass
class PagedCache:
    """Device buffers of one layer's paged 8-bit cache plus the C descriptor that points at them."""
    desc: qp_paged
    k_codes: torch.Tensor    # float8_e4m3fn or int8 [n_pages,Hkv,page,D]
    v_codes: torch.Tensor
    k_scale: torch.Tensor    # bf16 [n_pages,Hkv]
    v_scale: torch.Tensor
    k_tail: torch.Tensor     # bf16 [n_seqs,Hkv,page,D]
    v_tail: torch.Tensor

    def __post_init__(self):
        d = self.desc
        self.ref = ctypes.byref(d)                              # (nothing of the descriptor changes from call to call)
        self.heads, self.table, self.device = (d.n_q_heads, d.n_kv_heads, d.head_dim), (d.n_seqs, d.max_pages), self.k_codes.get_device()


def paged_layout(n_seqs: int, n_q_heads: int, n_kv_heads: int, head_dim: int, format: int, page: int, n_pages: int,
                 max_pages: int) -> qp_paged:
    c = qp_paged()
    _check(lib().qp_paged_layout(n_seqs, n_q_heads, n_kv_heads, head_dim, format, page, n_pages, max_pages, ctypes.byref(c)),
           "qp_paged_layout")
    return c


def paged_cache(n_q_heads: int, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                k_tail: torch.Tensor, v_tail: torch.Tensor, max_pages: int) -> PagedCache:
    """The cache that these arrays are (shapes as in PagedCache)."""
    n_pages, Hkv, page, D = k_codes.shape
    n_seqs = k_tail.shape[0]
    c = paged_layout(n_seqs, n_q_heads, Hkv, D, PAGED_FORMATS[k_codes.dtype], page, n_pages, max_pages)
    both = ((k_codes, v_codes, k_codes.dtype, (n_pages, Hkv, page, D)), (k_scale, v_scale, torch.bfloat16, (n_pages, Hkv)),
            (k_tail, v_tail, torch.bfloat16, (n_seqs, Hkv, page, D)))
    for k, v, dtype, shape in both:
        _dev(k, dtype, shape); _dev(v, dtype, shape)
    c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.k_tail, c.v_tail = map(_ptr, (k_codes, v_codes, k_scale, v_scale, k_tail, v_tail))
    return PagedCache(c, k_codes, v_codes, k_scale, v_scale, k_tail, v_tail)


def alloc_paged(n_seqs: int, n_q_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, max_pages: int, page: int = 64,
                dtype: torch.dtype = torch.float8_e4m3fn, device="cuda") -> PagedCache:
    """Allocates the buffers of ``qp_paged_layout`` with torch: a pool of n_pages pages for up to n_seqs sequences of up to
    max_pages pages each.  dtype: torch.float8_e4m3fn or torch.int8."""
    codes = lambda: torch.empty((n_pages, n_kv_heads, page, head_dim), dtype=dtype, device=device)
    wide = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=device)
    tail = (n_seqs, n_kv_heads, page, head_dim)
    return paged_cache(n_q_heads, codes(), codes(), wide(n_pages, n_kv_heads), wide(n_pages, n_kv_heads), wide(*tail), wide(*tail),
                       max_pages)


class PagedStep:
    """One step of a batch (qp_step), the same for all layers: sequence b's new tokens are rows start[b] .. start[b+1]-1 and stand
    behind the len[b] tokens it has; pages [n_seqs, max_pages] is the page table (int32 all, on the device).  The caller adds the
    new tokens to len after the last layer."""

    def __init__(self, start: torch.Tensor, len: torch.Tensor, pages: torch.Tensor, n_tokens: int, max_new: int):
        n_seqs, max_pages = pages.shape
        _dev(start, torch.int32, (n_seqs + 1,)); _dev(len, torch.int32, (n_seqs,)); _dev(pages, torch.int32, (n_seqs, max_pages))
        self.start, self.len, self.pages, self.n_tokens, self.max_new = start, len, pages, n_tokens, max_new
        self.shape, self.device = (n_seqs, max_pages), start.get_device()
        self.desc = qp_step(n_tokens, max_new, start.data_ptr(), len.data_ptr(), pages.data_ptr())
        self.ref = ctypes.byref(self.desc)


def _token_rows(t: torch.Tensor, n: int, heads: int, D: int, device: int) -> int:
    """bf16 rows [n, heads, D] whose heads lie one behind the other, on the device in use: elements from a row to the next."""
    row, head, one = t.stride()
    assert (t.dtype is _bf16 and t.shape == (n, heads, D) and t.get_device() == device and one == 1 and (head == D or heads == 1)), \
        (t.device, t.dtype, t.shape, t.stride())
    return row if n > 1 else heads * D


def _fits(cache: PagedCache, step: PagedStep) -> int:
    """The device in use, which both have to be on."""
    device = _current_device()
    assert step.shape == cache.table and step.device == device == cache.device, \
        "step and cache do not belong together, or are not on the current device"
    return device


def paged_append(k_new: torch.Tensor, v_new: torch.Tensor, cache: PagedCache, step: PagedStep, rope_: "qp_rope | None" = None,
                 pos: torch.Tensor | None = None, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None):
    """qp_paged_append: the step's keys and values [n_tokens,Hkv,D] go into the cache, keys rotated unless rope_ is None, at the
    tokens' positions in their sequences or at ``pos`` int32 [n_tokens]; returns the step's queries q [n_tokens,Hq,D] rotated, if
    they are given.  Rows may be parts of a fused projection's."""
    n, (Hq, Hkv, D), device = step.n_tokens, cache.heads, _fits(cache, step)
    ks, vs = _token_rows(k_new, n, Hkv, D, device), _token_rows(v_new, n, Hkv, D, device)
    qs, q_from, q_to = 0, None, None
    if q is not None:
        qs, q_from = _token_rows(q, n, Hq, D, device), q.data_ptr()
        if q_out is None:
            q_out = _empty_like(q, memory_format=_contiguous)
        else:
            _dev(q_out, _bf16, (n, Hq, D))
        q_to = q_out.data_ptr()
    if pos is not None:
        _dev(pos, _int32, (n,))
    status = lib().qp_paged_append(k_new.data_ptr(), ks, v_new.data_ptr(), vs, cache.ref, step.ref, None if rope_ is None else ctypes.byref(rope_),
                                   None if pos is None else pos.data_ptr(), q_from, qs, q_to, _stream())
    if status:
        _check(status, "qp_paged_append")
    return None if q is None else q_out


def paged_attn_workspace_bytes(cache: "PagedCache | qp_paged", n_tokens: int, max_new: int) -> int:
    return int(lib().qp_paged_attn_workspace_bytes(ctypes.byref(cache.desc if isinstance(cache, PagedCache) else cache), n_tokens, max_new))


def paged_attn(q: torch.Tensor, cache: PagedCache, step: PagedStep, out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """qp_paged_attn: attention of the step's tokens, which paged_append has taken in, over their sequences: q [n_tokens,Hq,D] ->
    out [n_tokens,Hq,D] (rows that are no sequence's are left as they are)."""
    n, (Hq, _, D), device = step.n_tokens, cache.heads, _fits(cache, step)
    qs = _token_rows(q, n, Hq, D, device)
    if out is None:
        out = _empty_like(q, memory_format=_contiguous)
    else:
        _dev(out, _bf16, (n, Hq, D))
    if workspace is None:
        workspace = new_decode_workspace(paged_attn_workspace_bytes(cache, n, step.max_new), q.device)
    address, size = _scratch(workspace)
    status = lib().qp_paged_attn(q.data_ptr(), qs, cache.ref, step.ref, out.data_ptr(), address, size, _stream())
    if status:
        _check(status, "qp_paged_attn")
    return out


def paged_layer_step(q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, cache: PagedCache, step: PagedStep,
                     rope_: "qp_rope | None" = None, pos: torch.Tensor | None = None, out: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None) -> torch.Tensor:
    """One layer of a step: qp_paged_append (with the queries, if there is a rotation), then qp_paged_attn.  A step that is refused
    has changed nothing: what the second call asks for is looked at before the first takes the tokens in."""
    n, (Hq, _, D), device = step.n_tokens, cache.heads, _fits(cache, step)
    stride = _token_rows(q, n, Hq, D, device)
    if out is None:
        out = _empty_like(q, memory_format=_contiguous)
    else:
        _dev(out, _bf16, (n, Hq, D))
    need = paged_attn_workspace_bytes(cache, n, step.max_new)
    if workspace is None:
        workspace = new_decode_workspace(need, q.device)
    address, size = _scratch(workspace)
    if need == 0:
        raise QpError(2 if 1 <= step.max_new <= n else 1, "paged_layer_step")
    if size < need:
        raise QpError(4, "paged_layer_step")
    if stride < Hq * D:
        raise QpError(1, "paged_layer_step")
    if (address | q.data_ptr() | out.data_ptr()) & 15 or stride & 7:
        raise QpError(5, "paged_layer_step")
    turned = paged_append(k_new, v_new, cache, step, rope_, pos, None if rope_ is None else q)
    return paged_attn(q if rope_ is None else turned, cache, step, out, workspace)


def debug_check() -> tuple[int, list[int]]:
    """qp_debug_check: (status, [1 + site of the first violation or 0, index, limit, violations]); status is
    QP_ERR_UNSUPPORTED (2) unless the loaded library is the range-checked build."""
    w = (ctypes.c_uint32 * 4)()
    st = lib().qp_debug_check(w)
    return st, list(w)


def debug_give_up(block: int) -> int:
    """qp_debug_give_up: the status; QP_ERR_UNSUPPORTED (2) unless the loaded library is the range-checked build."""
    return lib().qp_debug_give_up(block)


# the C entry points under their own names
qp_status_string = status_string
qp_n_keep = n_keep
qp_cache_layout = cache_layout
qp_compress_workspace_bytes = compress_workspace_bytes
qp_decode_workspace_bytes = decode_workspace_bytes
qp_window_scores = window_scores
qp_select_topk = select_topk
qp_gather_quantize = gather_quantize
qp_compress_layer = compress_layer
qp_compress_layers = compress_layers
qp_decode_attn = decode_attn
qp_decode_attn_layers = decode_attn_layers
qp_decode_attn_static = decode_attn_static
qp_decode_overlap = decode_overlap
qp_gather_quantize_ex = gather_quantize_ex
qp_decode_attn_ex = decode_attn_ex
qp_debug_check = debug_check
qp_debug_give_up = debug_give_up
qp_decode_attn_layers_ex = decode_attn_layers_ex
qp_head_budgets = head_budgets
qp_head_budgets_workspace_bytes = lambda *a: int(lib().qp_head_budgets_workspace_bytes(*a))
qp_cache_layout_cap = cache_layout_cap
qp_append_kv = append_kv
qp_append_kv_layers = append_kv_layers
qp_decode_attn_tail = decode_attn_tail
qp_decode_attn_tail_layers = decode_attn_tail_layers
qp_prompt_weights = prompt_weights
qp_prompt_weights_workspace_bytes = prompt_weights_workspace_bytes
qp_heavy_select = heavy_select
qp_decode_attn_weights = decode_attn_weights
qp_decode_weights_workspace_bytes = decode_weights_workspace_bytes
qp_evict_kv = evict_kv
qp_decode_attn_tree = decode_attn_tree
qp_decode_tree_workspace_bytes = decode_tree_workspace_bytes
qp_rope_init = rope
qp_rope_freqs = lambda rot_dim, interleaved, w, factor=1.0: rope(rot_dim, interleaved=interleaved, factor=factor, freqs=w)
qp_rotary = rotary
qp_paged_layout = paged_layout
qp_paged_append = paged_append
qp_paged_attn = paged_attn
qp_paged_attn_workspace_bytes = paged_attn_workspace_bytes
