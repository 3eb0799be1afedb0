"""Thin ctypes binding of libmagicpig.so: argument marshalling only.

Every function has the name and argument order of its C entry point (include/magicpig.h)
and takes torch tensors where the C call takes device pointers.  Work is enqueued on
torch's current HIP stream.  There is no fallback: if the library is missing, loading
raises; if a call returns a negative status, MagicpigError is raised.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# (MAGICPIG_LIB names another build of the library, e.g. one compiled with other options)
LIB_PATH = os.environ.get("MAGICPIG_LIB") or os.path.join(_PKG, "libmagicpig.so")

MAGICPIG_BF16, MAGICPIG_FP32 = 0, 1
MAGICPIG_KV_SAME, MAGICPIG_KV_FP8_E4M3, MAGICPIG_KV_MXFP4 = 0, 1, 4


class MagicpigError(RuntimeError):
    pass


class magicpig_params(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("K", ctypes.c_int32), ("L", ctypes.c_int32),
        ("min_hits", ctypes.c_int32), ("n_sink", ctypes.c_int32), ("n_local", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("n_ctx", ctypes.c_int64), ("n_cap", ctypes.c_int64),
        ("k_stride_b", ctypes.c_int64), ("k_stride_h", ctypes.c_int64), ("k_stride_n", ctypes.c_int64),
        ("v_stride_b", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("v_stride_n", ctypes.c_int64),
        ("n_ctx_dev", ctypes.c_void_p),
        ("kv_dtype", ctypes.c_int32),
    ]


class magicpig_paged_params(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
        ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_new", ctypes.c_int32),
        ("n_sink", ctypes.c_int32), ("n_local", ctypes.c_int32), ("scale", ctypes.c_float),
        ("n_pages", ctypes.c_int64), ("max_tokens", ctypes.c_int64),
        ("k_stride_page", ctypes.c_int64), ("k_stride_key", ctypes.c_int64), ("k_stride_head", ctypes.c_int64),
        ("v_stride_page", ctypes.c_int64), ("v_stride_key", ctypes.c_int64), ("v_stride_head", ctypes.c_int64),
        ("q_stride_token", ctypes.c_int64), ("q_stride_head", ctypes.c_int64),
        ("k_new_stride_token", ctypes.c_int64), ("k_new_stride_head", ctypes.c_int64),
        ("v_new_stride_token", ctypes.c_int64), ("v_new_stride_head", ctypes.c_int64),
    ]


EXPORTS = (
    "magicpig_code_words_per_key", "magicpig_code_words_per_query", "magicpig_key_code_bytes",
    "magicpig_query_code_bytes",
    "magicpig_key_code_index", "magicpig_workspace_bytes", "magicpig_key_mean",
    "magicpig_hash_keys", "magicpig_hash_query", "magicpig_sampled_attention",
    "magicpig_status_string", "magicpig_last_hip_error", "magicpig_profile_stage_events",
    "magicpig_hash_keys_stats_offset", "magicpig_table_bytes", "magicpig_build_tables",
    "magicpig_sampled_attention_tables", "magicpig_hash_decode_step", "magicpig_table_build_workspace_bytes",
    "magicpig_sampled_attention_noalloc",
    "magicpig_prepared_projector_bytes", "magicpig_prepare_projector", "magicpig_centering_bytes",
    "magicpig_prepare_centering", "magicpig_hash_query_prepared", "magicpig_hash_decode_step_prepared",
    "magicpig_paged_workspace_bytes", "magicpig_page_plan", "magicpig_page_append", "magicpig_paged_attention",
    "magicpig_page_append_mxfp", "magicpig_page_read_mxfp", "magicpig_paged_attention_mxfp",
    "magicpig_page_weights", "magicpig_page_keep", "magicpig_page_evict",
)

_lib = None


def lib() -> ctypes.CDLL:
    """Loads libmagicpig.so (built in-tree by paper_2410_16179_amd.build); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise MagicpigError(f"{LIB_PATH} is not built; run `python -m paper_2410_16179_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER(magicpig_params)
    vp, sz, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
    for name in ("magicpig_code_words_per_key", "magicpig_code_words_per_query", "magicpig_key_code_bytes",
                 "magicpig_query_code_bytes", "magicpig_workspace_bytes",
                 "magicpig_hash_keys_stats_offset", "magicpig_table_bytes", "magicpig_table_build_workspace_bytes",
                 "magicpig_prepared_projector_bytes", "magicpig_centering_bytes"):
        getattr(L, name).restype, getattr(L, name).argtypes = sz, [P]
    L.magicpig_key_code_index.restype = sz
    L.magicpig_key_code_index.argtypes = [P, i32, i32, i64, i32]
    L.magicpig_key_mean.restype = ctypes.c_int
    L.magicpig_key_mean.argtypes = [P, vp, vp, vp, sz, vp]
    L.magicpig_hash_keys.restype = ctypes.c_int
    L.magicpig_hash_keys.argtypes = [P, vp, vp, vp, i64, i64, vp, vp, sz, vp]
    L.magicpig_hash_query.restype = ctypes.c_int
    L.magicpig_hash_query.argtypes = [P, vp, vp, vp, vp, sz, vp]
    L.magicpig_hash_decode_step.restype = ctypes.c_int
    L.magicpig_hash_decode_step.argtypes = [P, vp, vp, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    L.magicpig_sampled_attention.restype = ctypes.c_int
    L.magicpig_sampled_attention.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp, sz, vp]
    L.magicpig_sampled_attention_noalloc.restype = ctypes.c_int
    L.magicpig_sampled_attention_noalloc.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp]
    L.magicpig_prepare_projector.restype = ctypes.c_int
    L.magicpig_prepare_projector.argtypes = [P, vp, vp, vp]
    L.magicpig_prepare_centering.restype = ctypes.c_int
    L.magicpig_prepare_centering.argtypes = [P, vp, vp, vp, vp]
    L.magicpig_hash_query_prepared.restype = ctypes.c_int
    L.magicpig_hash_query_prepared.argtypes = [P, vp, vp, vp, vp]
    L.magicpig_hash_decode_step_prepared.restype = ctypes.c_int
    L.magicpig_hash_decode_step_prepared.argtypes = [P, vp, vp, vp, vp, vp, i64, i64, vp, vp, vp]
    L.magicpig_build_tables.restype = ctypes.c_int
    L.magicpig_build_tables.argtypes = [P, vp, vp, vp, sz, vp]
    L.magicpig_sampled_attention_tables.restype = ctypes.c_int
    L.magicpig_sampled_attention_tables.argtypes = [P, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp, sz, vp]
    PP = ctypes.POINTER(magicpig_paged_params)
    L.magicpig_paged_workspace_bytes.restype, L.magicpig_paged_workspace_bytes.argtypes = sz, [PP]
    L.magicpig_page_plan.restype = ctypes.c_int
    L.magicpig_page_plan.argtypes = [PP] + [vp] * 11 + [sz, vp]
    L.magicpig_page_append.restype = ctypes.c_int
    L.magicpig_page_append.argtypes = [PP] + [vp] * 8
    L.magicpig_paged_attention.restype = ctypes.c_int
    L.magicpig_paged_attention.argtypes = [PP] + [vp] * 11 + [sz, vp]
    L.magicpig_page_append_mxfp.restype = ctypes.c_int
    L.magicpig_page_append_mxfp.argtypes = [PP] + [vp] * 8
    L.magicpig_page_read_mxfp.restype = ctypes.c_int
    L.magicpig_page_read_mxfp.argtypes = [PP] + [vp] * 8
    L.magicpig_paged_attention_mxfp.restype = ctypes.c_int
    L.magicpig_paged_attention_mxfp.argtypes = [PP] + [vp] * 11 + [sz, vp]
    L.magicpig_page_weights.restype = ctypes.c_int
    L.magicpig_page_weights.argtypes = [PP] + [vp] * 11 + [sz, vp]
    L.magicpig_page_keep.restype = ctypes.c_int
    L.magicpig_page_keep.argtypes = [PP] + [vp] * 4 + [i32] * 3 + [vp] * 3 + [sz, vp]
    L.magicpig_page_evict.restype = ctypes.c_int
    L.magicpig_page_evict.argtypes = [PP, vp, i32] + [vp] * 13 + [sz, vp]
    L.magicpig_status_string.restype, L.magicpig_status_string.argtypes = ctypes.c_char_p, [ctypes.c_int]
    L.magicpig_last_hip_error.restype, L.magicpig_last_hip_error.argtypes = ctypes.c_char_p, []
    L.magicpig_profile_stage_events.restype = None
    L.magicpig_profile_stage_events.argtypes = [ctypes.POINTER(ctypes.c_void_p)]
    _lib = L
    return L


def _check(status: int) -> None:
    if status != 0:
        msg = lib().magicpig_status_string(status).decode()
        if status == -4:
            msg += ": " + lib().magicpig_last_hip_error().decode()
        raise MagicpigError(f"magicpig status {status}: {msg}")


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def make_params(*, batch, n_q_heads, n_kv_heads, K, L, n_ctx, dtype, n_cap=None, min_hits=2,
                n_sink=4, n_local=64, head_dim=128, k_strides=None, v_strides=None,
                n_ctx_dev=None, kv_dtype=0) -> magicpig_params:
    """Parameter block; strides default to a contiguous [batch, n_kv_heads, n_cap, 128] cache.
    n_ctx_dev: an int64 device tensor holding the live context length, or None.
    kv_dtype: 0 (caches hold `dtype`), 1 or "fp8" (caches hold OCP e4m3 bytes)."""
    kv_dtype = {"fp8": MAGICPIG_KV_FP8_E4M3, "": 0, None: 0}.get(kv_dtype, kv_dtype)
    n_cap = n_ctx if n_cap is None else n_cap
    dense = (n_kv_heads * n_cap * head_dim, n_cap * head_dim, head_dim)
    ks = dense if k_strides is None else tuple(k_strides)
    vs = dense if v_strides is None else tuple(v_strides)
    code = {"bf16": MAGICPIG_BF16, "fp32": MAGICPIG_FP32, torch.bfloat16: MAGICPIG_BF16,
            torch.float32: MAGICPIG_FP32}.get(dtype, dtype)
    return magicpig_params(batch, n_q_heads, n_kv_heads, head_dim, K, L, min_hits, n_sink, n_local,
                           code, n_ctx, n_cap, ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                           None if n_ctx_dev is None else n_ctx_dev.data_ptr(), kv_dtype)


def magicpig_code_words_per_key(params) -> int:
    return lib().magicpig_code_words_per_key(ctypes.byref(params))


def magicpig_code_words_per_query(params) -> int:
    return lib().magicpig_code_words_per_query(ctypes.byref(params))


def magicpig_key_code_bytes(params) -> int:
    return lib().magicpig_key_code_bytes(ctypes.byref(params))


def magicpig_query_code_bytes(params) -> int:
    return lib().magicpig_query_code_bytes(ctypes.byref(params))


def magicpig_workspace_bytes(params) -> int:
    return lib().magicpig_workspace_bytes(ctypes.byref(params))


def magicpig_hash_keys_stats_offset(params) -> int:
    return lib().magicpig_hash_keys_stats_offset(ctypes.byref(params))


def hash_keys_stats(params, workspace) -> dict:
    """Reads the statistics a bf16 magicpig_hash_keys call left in its workspace (synchronises)."""
    off = magicpig_hash_keys_stats_offset(params)
    raw = workspace[off:off + 16].cpu().numpy().view(np.uint32)
    return {"w_max_norm": float(raw[:1].view(np.float32)[0]), "spilled": int(raw[1]),
            "overflowed": bool(raw[2]), "rechecked": int(raw[3])}


def magicpig_key_code_index(params, b, g, key, word) -> int:
    return lib().magicpig_key_code_index(ctypes.byref(params), b, g, key, word)


def magicpig_key_mean(params, K_cache, mu_out, workspace) -> None:
    _check(lib().magicpig_key_mean(ctypes.byref(params), _ptr(K_cache), _ptr(mu_out), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream()))


def magicpig_hash_keys(params, K_cache, mu, W, first_key, n_keys, key_codes, workspace) -> None:
    _check(lib().magicpig_hash_keys(ctypes.byref(params), _ptr(K_cache), _ptr(mu), _ptr(W), first_key,
                                    n_keys, _ptr(key_codes), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream()))


def magicpig_hash_query(params, q, W, q_codes, workspace=None) -> None:
    _check(lib().magicpig_hash_query(ctypes.byref(params), _ptr(q), _ptr(W), _ptr(q_codes),
                                     _ptr(workspace), _nbytes(workspace), _stream()))


def magicpig_hash_decode_step(params, q, K_cache, mu, W, first_key, n_keys, key_codes, q_codes, workspace=None) -> None:
    _check(lib().magicpig_hash_decode_step(ctypes.byref(params), _ptr(q), _ptr(K_cache), _ptr(mu), _ptr(W),
                                           first_key, n_keys, _ptr(key_codes), _ptr(q_codes), _ptr(workspace),
                                           _nbytes(workspace), _stream()))


def magicpig_prepared_projector_bytes(params) -> int:
    return lib().magicpig_prepared_projector_bytes(ctypes.byref(params))


def magicpig_centering_bytes(params) -> int:
    return lib().magicpig_centering_bytes(ctypes.byref(params))


def magicpig_prepare_projector(params, W, prepared) -> None:
    _check(lib().magicpig_prepare_projector(ctypes.byref(params), _ptr(W), _ptr(prepared), _stream()))


def magicpig_prepare_centering(params, mu, prepared, centering) -> None:
    _check(lib().magicpig_prepare_centering(ctypes.byref(params), _ptr(mu), _ptr(prepared), _ptr(centering), _stream()))


def magicpig_hash_query_prepared(params, q, prepared, q_codes) -> None:
    _check(lib().magicpig_hash_query_prepared(ctypes.byref(params), _ptr(q), _ptr(prepared), _ptr(q_codes), _stream()))


def magicpig_hash_decode_step_prepared(params, q, K_cache, mu, centering, prepared, first_key, n_keys, key_codes,
                                       q_codes) -> None:
    _check(lib().magicpig_hash_decode_step_prepared(ctypes.byref(params), _ptr(q), _ptr(K_cache), _ptr(mu),
                                                    _ptr(centering), _ptr(prepared), first_key, n_keys,
                                                    _ptr(key_codes), _ptr(q_codes), _stream()))


def magicpig_sampled_attention(params, q, K_cache, V_cache, mu, key_codes, q_codes, out,
                               dbg_counts=None, dbg_cand=None, dbg_ncand=None, workspace=None) -> None:
    cap = 0 if dbg_cand is None else dbg_cand.shape[-1]
    _check(lib().magicpig_sampled_attention(
        ctypes.byref(params), _ptr(q), _ptr(K_cache), _ptr(V_cache), _ptr(mu), _ptr(key_codes),
        _ptr(q_codes), _ptr(out), _ptr(dbg_counts), _ptr(dbg_cand), _ptr(dbg_ncand), cap,
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


def magicpig_sampled_attention_noalloc(params, q, K_cache, V_cache, mu, key_codes, q_codes, out) -> None:
    _check(lib().magicpig_sampled_attention_noalloc(
        ctypes.byref(params), _ptr(q), _ptr(K_cache), _ptr(V_cache), _ptr(mu), _ptr(key_codes),
        _ptr(q_codes), _ptr(out), _stream()))


def magicpig_table_bytes(params) -> int:
    return lib().magicpig_table_bytes(ctypes.byref(params))


def magicpig_build_tables(params, key_codes, tables, workspace=None) -> None:
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().magicpig_build_tables(ctypes.byref(params), _ptr(key_codes), _ptr(tables), _ptr(workspace),
                                       nbytes, _stream()))


def magicpig_sampled_attention_tables(params, q, K_cache, V_cache, mu, tables, n_indexed, key_codes, q_codes,
                                      out, dbg_counts=None, dbg_cand=None, dbg_ncand=None, workspace=None) -> None:
    cap = 0 if dbg_cand is None else dbg_cand.shape[-1]
    _check(lib().magicpig_sampled_attention_tables(
        ctypes.byref(params), _ptr(q), _ptr(K_cache), _ptr(V_cache), _ptr(mu), _ptr(tables),
        int(n_indexed), _ptr(key_codes), _ptr(q_codes), _ptr(out), _ptr(dbg_counts), _ptr(dbg_cand), _ptr(dbg_ncand), cap,
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


def magicpig_profile_stage_events(events) -> None:
    """events: None, or seven hipEvent_t handles (ints) attached to the decode kernels."""
    if events is None:
        lib().magicpig_profile_stage_events(None)
    else:
        assert len(events) == 7
        arr = (ctypes.c_void_p * 7)(*events)
        lib().magicpig_profile_stage_events(arr)


# ---- paged cache -----------------------------------------------------------------------------
def make_paged_params(*, batch, n_q_heads, n_kv_heads, dtype, page_size, max_pages, n_pages, max_tokens=None, max_new=1,
                      kv_dtype=0, n_sink=0, n_local=0, scale=0.0, head_dim=128, k_strides=None, v_strides=None,
                      q_strides=None, k_new_strides=None, v_new_strides=None) -> magicpig_paged_params:
    """Parameter block of the paged calls.  Element strides default to contiguous pools
    [n_pages, page_size, n_kv_heads, 128] and contiguous token arrays [max_tokens, heads, 128]; pool strides
    are (page, key, head), those of token arrays (token, head).  max_tokens defaults to batch.  kv_dtype: "" (pools hold
    `dtype`), "fp8" or "mxfp4"; strides of pools in four bits count elements, two of which are a byte of the tensor."""
    kv_dtype = {"fp8": MAGICPIG_KV_FP8_E4M3, "mxfp4": MAGICPIG_KV_MXFP4, "": 0, None: 0}.get(kv_dtype, kv_dtype)
    code = {"bf16": MAGICPIG_BF16, "fp32": MAGICPIG_FP32, torch.bfloat16: MAGICPIG_BF16,
            torch.float32: MAGICPIG_FP32}.get(dtype, dtype)
    row = n_kv_heads * head_dim
    pool, new = (page_size * row, row, head_dim), (row, head_dim)
    either = lambda given, default: default if given is None else tuple(given)
    return magicpig_paged_params(batch, n_q_heads, n_kv_heads, head_dim, code, kv_dtype, page_size, max_pages, max_new,
                                 n_sink, n_local, scale, n_pages, max(batch, 1) if max_tokens is None else max_tokens,
                                 *either(k_strides, pool), *either(v_strides, pool),
                                 *either(q_strides, (n_q_heads * head_dim, head_dim)),
                                 *either(k_new_strides, new), *either(v_new_strides, new))


_DTYPES = {MAGICPIG_BF16: torch.bfloat16, MAGICPIG_FP32: torch.float32}


class _PagedSizes:
    """What the paged calls' tensors have to be by a parameter block: types, and elements from the first to the last one used."""

    def __init__(self, p):
        reach = lambda *dims: p.head_dim + sum(stride * (size - 1) for stride, size in dims)
        self.dtype = _DTYPES.get(p.dtype)
        self.four = p.kv_dtype == MAGICPIG_KV_MXFP4
        self.pool_dtype = {MAGICPIG_KV_FP8_E4M3: (torch.float8_e4m3fn, torch.uint8),
                           MAGICPIG_KV_MXFP4: (torch.uint8, torch.float4_e2m1fn_x2)}.get(p.kv_dtype, (self.dtype,))
        self.batch, self.heads, self.n_pages, self.tokens, self.table = p.batch, p.n_kv_heads, p.n_pages, p.max_tokens, p.batch * p.max_pages
        self.k_pages = reach((p.k_stride_page, p.n_pages), (p.k_stride_key, p.page_size), (p.k_stride_head, p.n_kv_heads))
        self.v_pages = reach((p.v_stride_page, p.n_pages), (p.v_stride_key, p.page_size), (p.v_stride_head, p.n_kv_heads))
        if self.four:                                        # (entries of the tensors: two elements, and a block's scale)
            self.k_block, self.v_block = self.k_pages // 32, self.v_pages // 32
            self.k_pages, self.v_pages = self.k_pages // 2, self.v_pages // 2
        self.q = reach((p.q_stride_token, p.max_tokens), (p.q_stride_head, p.n_q_heads))
        self.k_new = reach((p.k_new_stride_token, p.max_tokens), (p.k_new_stride_head, p.n_kv_heads))
        self.v_new = reach((p.v_new_stride_token, p.max_tokens), (p.v_new_stride_head, p.n_kv_heads))
        self.weights = p.n_pages * p.n_kv_heads * p.page_size
        self.lse = p.max_tokens * p.n_q_heads
        self.out = self.lse * p.head_dim


def _paged_sizes(p) -> _PagedSizes:
    """Worked out once per block and kept with it, next to the bytes they stand for: a block that was changed, in whatever way, or a copy
    that was, gets its own.  Nothing in them refers to the block."""
    fields, kept = bytes(p), p.__dict__.get("sizes")
    if kept is None or kept[0] != fields:
        kept = p.__dict__["sizes"] = fields, _PagedSizes(p)
    return kept[1]


def _dense(t, device, dtype, elements) -> bool:
    """Whether t is read as it should be where the call takes it for one run of elements."""
    return t.get_device() == device and t.dtype is dtype and t.numel() >= elements and t.is_contiguous()


def _strided(t, device, dtypes, elements) -> bool:
    """The same where the call goes by the strides of the parameters: so many elements lie behind the tensor's first one."""
    if t.get_device() != device or t.dtype not in dtypes:
        return False
    return t.untyped_storage().nbytes() >= (t.storage_offset() + elements) * t.element_size()


def _refuse(device, **tensors):
    """Says what is wrong: name=(tensor, dtypes, elements, dense, optional)."""
    for name, (t, dtypes, elements, dense, optional) in tensors.items():
        if t is None:
            if optional:
                continue
            raise MagicpigError(f"{name} is missing")
        if t.get_device() != device:
            raise MagicpigError(f"{name} is on device {t.device}, the call runs on cuda:{device}")
        if t.dtype not in dtypes:
            raise MagicpigError(f"{name} has dtype {t.dtype}, not {dtypes[0]}")
        if dense and not t.is_contiguous():
            raise MagicpigError(f"{name} is not contiguous")
        if dense and t.numel() < elements:
            raise MagicpigError(f"{name} has {t.numel()} elements, the parameters say {elements}")
        if not dense and not _strided(t, device, dtypes, elements):
            raise MagicpigError(f"{name} ends before the {elements} elements that the parameters' strides reach")
    raise MagicpigError("a tensor does not fit the parameters")


def _paged_device(t, workspace=None) -> int:
    device = -1 if t is None else t.get_device()
    if device < 0:
        raise MagicpigError("the paged calls take tensors on a GPU")
    if workspace is not None and workspace.get_device() != device:
        raise MagicpigError(f"the workspace is on device {workspace.device}, the call runs on cuda:{device}")
    return device


def _paged_call(device, fn, *args) -> None:
    """fn(*args, stream) with the tensors' device current, on that device's current stream."""
    if device == torch.cuda.current_device():
        status = fn(*args, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(device))
    if status != 0:
        _check(status)


def magicpig_paged_workspace_bytes(params) -> int:
    return lib().magicpig_paged_workspace_bytes(ctypes.byref(params))


def magicpig_page_plan(params, new_tokens, lengths, block_table, free_pages, n_free, lengths_out, n_free_out, token_start,
                       slots, status, workspace=None) -> None:
    s, device, i32 = _paged_sizes(params), _paged_device(lengths, workspace), torch.int32
    n, of = s.batch, lambda t, count: (t, (i32,), count, True, False)
    try:
        fits = (_dense(new_tokens, device, i32, n) and _dense(lengths, device, i32, n) and _dense(block_table, device, i32, s.table)
                and _dense(free_pages, device, i32, s.n_pages) and _dense(n_free, device, i32, 1) and _dense(lengths_out, device, i32, n)
                and _dense(n_free_out, device, i32, 1) and _dense(token_start, device, i32, n + 1)
                and _dense(slots, device, torch.int64, s.tokens) and _dense(status, device, i32, 1))
    except AttributeError:                                   # (None)
        fits = False
    if not fits:
        _refuse(device, new_tokens=of(new_tokens, n), lengths=of(lengths, n), block_table=of(block_table, s.table),
                free_pages=of(free_pages, s.n_pages), n_free=of(n_free, 1), lengths_out=of(lengths_out, n), n_free_out=of(n_free_out, 1),
                token_start=of(token_start, n + 1), slots=(slots, (torch.int64,), s.tokens, True, False), status=of(status, 1))
    _paged_call(device, lib().magicpig_page_plan, ctypes.byref(params), new_tokens.data_ptr(), lengths.data_ptr(), block_table.data_ptr(),
                free_pages.data_ptr(), n_free.data_ptr(), lengths_out.data_ptr(), n_free_out.data_ptr(), token_start.data_ptr(),
                slots.data_ptr(), status.data_ptr(), _ptr(workspace), _nbytes(workspace))


def magicpig_page_append(params, k_new, v_new, slots, k_scale, v_scale, k_pages, v_pages) -> None:
    s, device, f32 = _paged_sizes(params), _paged_device(k_pages), torch.float32
    try:
        fits = (_strided(k_new, device, (s.dtype,), s.k_new) and _strided(v_new, device, (s.dtype,), s.v_new)
                and _dense(slots, device, torch.int64, s.tokens) and _strided(k_pages, device, s.pool_dtype, s.k_pages)
                and _strided(v_pages, device, s.pool_dtype, s.v_pages) and (k_scale is None or _dense(k_scale, device, f32, s.heads))
                and (v_scale is None or _dense(v_scale, device, f32, s.heads)))
    except AttributeError:
        fits = False
    if not fits:
        _refuse(device, k_new=(k_new, (s.dtype,), s.k_new, False, False), v_new=(v_new, (s.dtype,), s.v_new, False, False),
                slots=(slots, (torch.int64,), s.tokens, True, False), k_pages=(k_pages, s.pool_dtype, s.k_pages, False, False),
                v_pages=(v_pages, s.pool_dtype, s.v_pages, False, False), k_scale=(k_scale, (f32,), s.heads, True, True),
                v_scale=(v_scale, (f32,), s.heads, True, True))
    _paged_call(device, lib().magicpig_page_append, ctypes.byref(params), k_new.data_ptr(), v_new.data_ptr(), slots.data_ptr(), _ptr(k_scale),
                _ptr(v_scale), k_pages.data_ptr(), v_pages.data_ptr())


def magicpig_paged_attention(params, q, k_pages, v_pages, k_scale, v_scale, block_table, lengths, token_start, out, lse=None,
                             workspace=None) -> None:
    s, device, i32, f32 = _paged_sizes(params), _paged_device(q, workspace), torch.int32, torch.float32
    try:
        fits = (_strided(q, device, (s.dtype,), s.q) and _strided(k_pages, device, s.pool_dtype, s.k_pages)
                and _strided(v_pages, device, s.pool_dtype, s.v_pages) and _dense(block_table, device, i32, s.table)
                and _dense(lengths, device, i32, s.batch) and (token_start is None or _dense(token_start, device, i32, s.batch + 1))
                and _dense(out, device, s.dtype, s.out) and (lse is None or _dense(lse, device, f32, s.lse))
                and (k_scale is None or _dense(k_scale, device, f32, s.heads)) and (v_scale is None or _dense(v_scale, device, f32, s.heads)))
    except AttributeError:
        fits = False
    if not fits:
        _refuse(device, q=(q, (s.dtype,), s.q, False, False), k_pages=(k_pages, s.pool_dtype, s.k_pages, False, False),
                v_pages=(v_pages, s.pool_dtype, s.v_pages, False, False), k_scale=(k_scale, (f32,), s.heads, True, True),
                v_scale=(v_scale, (f32,), s.heads, True, True), block_table=(block_table, (i32,), s.table, True, False),
                lengths=(lengths, (i32,), s.batch, True, False), token_start=(token_start, (i32,), s.batch + 1, True, True),
                out=(out, (s.dtype,), s.out, True, False), lse=(lse, (f32,), s.lse, True, True))
    _paged_call(device, lib().magicpig_paged_attention, ctypes.byref(params), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scale),
                _ptr(v_scale), block_table.data_ptr(), lengths.data_ptr(), _ptr(token_start), out.data_ptr(), _ptr(lse), _ptr(workspace),
                _nbytes(workspace))


_SCALES = (torch.uint8, torch.float8_e8m0fnu)


def _four_bit_sizes(params) -> _PagedSizes:
    s = _paged_sizes(params)
    if not s.four:
        raise MagicpigError("the parameters' kv_dtype is not MAGICPIG_KV_MXFP4")
    return s


def _rows_mxfp4(params, k_rows, v_rows, slots, k_pages, v_pages, k_block_scales, v_block_scales, names) -> int:
    """The device of a call between rows and pools in four bits, when everything fits."""
    s, device = _four_bit_sizes(params), _paged_device(k_pages)
    try:
        fits = (_strided(k_rows, device, (s.dtype,), s.k_new) and _strided(v_rows, device, (s.dtype,), s.v_new)
                and _dense(slots, device, torch.int64, s.tokens) and _strided(k_pages, device, s.pool_dtype, s.k_pages)
                and _strided(v_pages, device, s.pool_dtype, s.v_pages) and _strided(k_block_scales, device, _SCALES, s.k_block)
                and _strided(v_block_scales, device, _SCALES, s.v_block))
    except AttributeError:
        fits = False
    if not fits:
        _refuse(device, **{names[0]: (k_rows, (s.dtype,), s.k_new, False, False), names[1]: (v_rows, (s.dtype,), s.v_new, False, False)},
                slots=(slots, (torch.int64,), s.tokens, True, False), k_pages=(k_pages, s.pool_dtype, s.k_pages, False, False),
                v_pages=(v_pages, s.pool_dtype, s.v_pages, False, False), k_block_scales=(k_block_scales, _SCALES, s.k_block, False, False),
                v_block_scales=(v_block_scales, _SCALES, s.v_block, False, False))
    return device


def magicpig_page_append_mxfp(params, k_new, v_new, slots, k_pages, v_pages, k_block_scales, v_block_scales) -> None:
    device = _rows_mxfp4(params, k_new, v_new, slots, k_pages, v_pages, k_block_scales, v_block_scales, ("k_new", "v_new"))
    _paged_call(device, lib().magicpig_page_append_mxfp, ctypes.byref(params), k_new.data_ptr(), v_new.data_ptr(), slots.data_ptr(),
                k_pages.data_ptr(), v_pages.data_ptr(), k_block_scales.data_ptr(), v_block_scales.data_ptr())


def magicpig_page_read_mxfp(params, k_pages, v_pages, k_block_scales, v_block_scales, slots, k_out, v_out) -> None:
    device = _rows_mxfp4(params, k_out, v_out, slots, k_pages, v_pages, k_block_scales, v_block_scales, ("k_out", "v_out"))
    _paged_call(device, lib().magicpig_page_read_mxfp, ctypes.byref(params), k_pages.data_ptr(), v_pages.data_ptr(), k_block_scales.data_ptr(),
                v_block_scales.data_ptr(), slots.data_ptr(), k_out.data_ptr(), v_out.data_ptr())


def magicpig_paged_attention_mxfp(params, q, k_pages, v_pages, k_block_scales, v_block_scales, block_table, lengths, token_start, out,
                                   lse=None, workspace=None) -> None:
    s, device, i32, f32 = _four_bit_sizes(params), _paged_device(q, workspace), torch.int32, torch.float32
    try:
        fits = (_strided(q, device, (s.dtype,), s.q) and _strided(k_pages, device, s.pool_dtype, s.k_pages)
                and _strided(v_pages, device, s.pool_dtype, s.v_pages) and _strided(k_block_scales, device, _SCALES, s.k_block)
                and _strided(v_block_scales, device, _SCALES, s.v_block) and _dense(block_table, device, i32, s.table)
                and _dense(lengths, device, i32, s.batch) and (token_start is None or _dense(token_start, device, i32, s.batch + 1))
                and _dense(out, device, s.dtype, s.out) and (lse is None or _dense(lse, device, f32, s.lse)))
    except AttributeError:
        fits = False
    if not fits:
        _refuse(device, q=(q, (s.dtype,), s.q, False, False), k_pages=(k_pages, s.pool_dtype, s.k_pages, False, False),
                v_pages=(v_pages, s.pool_dtype, s.v_pages, False, False), k_block_scales=(k_block_scales, _SCALES, s.k_block, False, False),
                v_block_scales=(v_block_scales, _SCALES, s.v_block, False, False), block_table=(block_table, (i32,), s.table, True, False),
                lengths=(lengths, (i32,), s.batch, True, False), token_start=(token_start, (i32,), s.batch + 1, True, True),
                out=(out, (s.dtype,), s.out, True, False), lse=(lse, (f32,), s.lse, True, True))
    _paged_call(device, lib().magicpig_paged_attention_mxfp, ctypes.byref(params), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                k_block_scales.data_ptr(), v_block_scales.data_ptr(), block_table.data_ptr(), lengths.data_ptr(), _ptr(token_start),
                out.data_ptr(), _ptr(lse), _ptr(workspace), _nbytes(workspace))


def _block(t, device, s, elements) -> bool:
    """Whether block scales are there exactly where the pools are in four bits."""
    return _strided(t, device, _SCALES, elements) if s.four else t is None


def _refuse_block(s, **tensors):
    for name, t in tensors.items():
        if t is not None and not s.four:
            raise MagicpigError(f"{name} belongs to pools of kv_dtype MAGICPIG_KV_MXFP4")


def magicpig_page_weights(params, q, k_pages, k_scale, k_block_scales, block_table, lengths, token_start, lse, counted, weights,
                          workspace=None) -> None:
    s, device, i32, f32 = _paged_sizes(params), _paged_device(q, workspace), torch.int32, torch.float32
    try:
        fits = (_strided(q, device, (s.dtype,), s.q) and _strided(k_pages, device, s.pool_dtype, s.k_pages)
                and _block(k_block_scales, device, s, s.four and s.k_block) and _dense(block_table, device, i32, s.table)
                and _dense(lengths, device, i32, s.batch) and (token_start is None or _dense(token_start, device, i32, s.batch + 1))
                and _dense(lse, device, f32, s.lse) and (counted is None or _dense(counted, device, i32, s.batch))
                and _dense(weights, device, f32, s.weights) and (k_scale is None or _dense(k_scale, device, f32, s.heads)))
    except AttributeError:
        fits = False
    if not fits:
        _refuse_block(s, k_block_scales=k_block_scales)
        _refuse(device, q=(q, (s.dtype,), s.q, False, False), k_pages=(k_pages, s.pool_dtype, s.k_pages, False, False),
                k_scale=(k_scale, (f32,), s.heads, True, True), k_block_scales=(k_block_scales, _SCALES, s.four and s.k_block, False, not s.four),
                block_table=(block_table, (i32,), s.table, True, False), lengths=(lengths, (i32,), s.batch, True, False),
                token_start=(token_start, (i32,), s.batch + 1, True, True), lse=(lse, (f32,), s.lse, True, False),
                counted=(counted, (i32,), s.batch, True, True), weights=(weights, (f32,), s.weights, True, False))
    _paged_call(device, lib().magicpig_page_weights, ctypes.byref(params), q.data_ptr(), k_pages.data_ptr(), _ptr(k_scale), _ptr(k_block_scales),
                block_table.data_ptr(), lengths.data_ptr(), _ptr(token_start), lse.data_ptr(), _ptr(counted), weights.data_ptr(), _ptr(workspace),
                _nbytes(workspace))


def magicpig_page_keep(params, weights, block_table, lengths, budgets, n_first, n_last, kept, lengths_out, workspace=None) -> None:
    """max_keep is the last dimension of `kept`, [batch, n_kv_heads, max_keep]."""
    s, device, i32, f32 = _paged_sizes(params), _paged_device(weights, workspace), torch.int32, torch.float32
    try:
        most = kept.shape[-1]
        fits = (_dense(weights, device, f32, s.weights) and _dense(block_table, device, i32, s.table) and _dense(lengths, device, i32, s.batch)
                and _dense(budgets, device, i32, s.batch) and _dense(kept, device, i32, s.batch * s.heads * most)
                and _dense(lengths_out, device, i32, s.batch))
    except (AttributeError, IndexError):
        most, fits = 1, False
    if not fits:
        _refuse(device, weights=(weights, (f32,), s.weights, True, False), block_table=(block_table, (i32,), s.table, True, False),
                lengths=(lengths, (i32,), s.batch, True, False), budgets=(budgets, (i32,), s.batch, True, False),
                kept=(kept, (i32,), s.batch * s.heads * most, True, False), lengths_out=(lengths_out, (i32,), s.batch, True, False))
    _paged_call(device, lib().magicpig_page_keep, ctypes.byref(params), weights.data_ptr(), block_table.data_ptr(), lengths.data_ptr(),
                budgets.data_ptr(), n_first, n_last, most, kept.data_ptr(), lengths_out.data_ptr(), _ptr(workspace), _nbytes(workspace))


def magicpig_page_evict(params, kept, lengths, lengths_kept, block_table, free_pages, n_free, k_pages, v_pages, k_block_scales, v_block_scales,
                        weights, n_free_out, status, workspace=None) -> None:
    """max_keep is the last dimension of `kept`, [batch, n_kv_heads, max_keep]; kept and weights may be None."""
    s, device, i32, f32 = _paged_sizes(params), _paged_device(k_pages, workspace), torch.int32, torch.float32
    try:
        most = 0 if kept is None else kept.shape[-1]
        fits = ((kept is None or _dense(kept, device, i32, s.batch * s.heads * most)) and _dense(lengths, device, i32, s.batch)
                and _dense(lengths_kept, device, i32, s.batch) and _dense(block_table, device, i32, s.table)
                and _dense(free_pages, device, i32, s.n_pages) and _dense(n_free, device, i32, 1) and _strided(k_pages, device, s.pool_dtype, s.k_pages)
                and _strided(v_pages, device, s.pool_dtype, s.v_pages) and _block(k_block_scales, device, s, s.four and s.k_block)
                and _block(v_block_scales, device, s, s.four and s.v_block) and (weights is None or _dense(weights, device, f32, s.weights))
                and _dense(n_free_out, device, i32, 1) and _dense(status, device, i32, 1))
    except (AttributeError, IndexError):
        most, fits = 1, False
    if not fits:
        _refuse_block(s, k_block_scales=k_block_scales, v_block_scales=v_block_scales)
        of = lambda t, count: (t, (i32,), count, True, False)
        _refuse(device, kept=(kept, (i32,), s.batch * s.heads * most, True, True), lengths=of(lengths, s.batch), lengths_kept=of(lengths_kept, s.batch),
                block_table=of(block_table, s.table), free_pages=of(free_pages, s.n_pages), n_free=of(n_free, 1),
                k_pages=(k_pages, s.pool_dtype, s.k_pages, False, False), v_pages=(v_pages, s.pool_dtype, s.v_pages, False, False),
                k_block_scales=(k_block_scales, _SCALES, s.four and s.k_block, False, not s.four),
                v_block_scales=(v_block_scales, _SCALES, s.four and s.v_block, False, not s.four),
                weights=(weights, (f32,), s.weights, True, True), n_free_out=of(n_free_out, 1), status=of(status, 1))
    _paged_call(device, lib().magicpig_page_evict, ctypes.byref(params), _ptr(kept), most, lengths.data_ptr(), lengths_kept.data_ptr(),
                block_table.data_ptr(), free_pages.data_ptr(), n_free.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_block_scales),
                _ptr(v_block_scales), _ptr(weights), n_free_out.data_ptr(), status.data_ptr(), _ptr(workspace), _nbytes(workspace))


# ---- buffer helpers (allocation and layout only) ---------------------------------------------
def alloc_key_codes(params, device="cuda") -> torch.Tensor:
    return torch.zeros(max(magicpig_key_code_bytes(params) // 4, 4), dtype=torch.int32, device=device)


def alloc_query_codes(params, device="cuda") -> torch.Tensor:
    return torch.zeros(max(magicpig_query_code_bytes(params) // 4, 4), dtype=torch.int32, device=device)


def alloc_tables(params, device="cuda") -> torch.Tensor:
    nbytes = magicpig_table_bytes(params)
    if nbytes == 0:
        raise MagicpigError("hash tables are not supported for these parameters")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def magicpig_table_build_workspace_bytes(params) -> int:
    return lib().magicpig_table_build_workspace_bytes(ctypes.byref(params))


def alloc_table_build_workspace(params, device="cuda") -> torch.Tensor:
    return torch.empty(max(magicpig_table_build_workspace_bytes(params), 256), dtype=torch.uint8, device=device)


def alloc_prepared_projector(params, device="cuda") -> torch.Tensor:
    return torch.empty(max(magicpig_prepared_projector_bytes(params), 256), dtype=torch.uint8, device=device)


def alloc_centering(params, device="cuda") -> torch.Tensor:
    return torch.empty(max(magicpig_centering_bytes(params), 256), dtype=torch.uint8, device=device)


def alloc_workspace(params, device="cuda") -> torch.Tensor:
    return torch.empty(max(magicpig_workspace_bytes(params), 256), dtype=torch.uint8, device=device)


def alloc_paged_workspace(params, device="cuda") -> torch.Tensor:
    return torch.zeros(max(magicpig_paged_workspace_bytes(params), 256), dtype=torch.uint8, device=device)


def key_code_gather_index(params) -> np.ndarray:
    """u32 index of every (b, g, key < n_cap, word) in the key-code buffer, built from
    magicpig_key_code_index on one block and the block stride it implies."""
    NW = magicpig_code_words_per_key(params)
    n_cap = params.n_cap
    slot = np.array([[magicpig_key_code_index(params, 0, 0, r, x) for x in range(NW)]
                     for r in range(min(64, n_cap))], dtype=np.int64)
    nblk = (n_cap + 63) // 64
    keys = np.arange(n_cap)
    per_unit = (keys // 64)[:, None] * (64 * NW) + slot[keys % 64]          # [n_cap, NW]
    units = np.arange(params.batch * params.n_kv_heads, dtype=np.int64) * (nblk * 64 * NW)
    idx = units[:, None, None] + per_unit[None]
    return idx.reshape(params.batch, params.n_kv_heads, n_cap, NW)


def key_plane_words(words: np.ndarray, K: int, L: int) -> np.ndarray:
    """[..., NW] words of key codes -> [..., K*ceil(L/32)] plane words: the last table group,
    stored as one bit string of K planes, is spread out again (tables >= L read 0)."""
    words = np.asarray(words).astype(np.uint32)
    Wd = (L + 31) // 32
    Lt, xs = L - 32 * (Wd - 1), K * (Wd - 1)
    out = np.zeros(words.shape[:-1] + (K * Wd,), np.uint32)
    out[..., :xs] = words[..., :xs]
    tail = words[..., xs:].astype(np.uint64)
    for b in range(K):
        pos = b * Lt
        wi, sh = pos // 32, pos % 32
        v = tail[..., wi] >> np.uint64(sh)
        if sh + Lt > 32:
            v = v | (tail[..., wi + 1] << np.uint64(32 - sh))
        out[..., xs + b] = (v & np.uint64((1 << Lt) - 1)).astype(np.uint32)
    return out


def key_words_from_planes(planes: np.ndarray, K: int, L: int) -> np.ndarray:
    """Inverse of key_plane_words: [..., K*ceil(L/32)] plane words -> [..., NW] key-code words."""
    planes = np.asarray(planes).astype(np.uint32)
    Wd = (L + 31) // 32
    Lt, xs = L - 32 * (Wd - 1), K * (Wd - 1)
    nt = (K * Lt + 31) // 32
    out = np.zeros(planes.shape[:-1] + (xs + nt,), np.uint32)
    out[..., :xs] = planes[..., :xs]
    acc = np.zeros(planes.shape[:-1] + (nt + 1,), np.uint64)
    for b in range(K):
        pos = b * Lt
        wi, sh = pos // 32, pos % 32
        v = (planes[..., xs + b].astype(np.uint64) & np.uint64((1 << Lt) - 1)) << np.uint64(sh)
        acc[..., wi] |= v & np.uint64(0xffffffff)
        acc[..., wi + 1] |= v >> np.uint64(32)
    out[..., xs:] = acc[..., :nt].astype(np.uint32)
    return out


def table_codes_from_words(words: np.ndarray, K: int, L: int) -> np.ndarray:
    """[..., K*ceil(L/32)] plane words (word w*K+b, bit beta <-> table 32w+beta) -> [..., L]
    integers sum_b bit_b 2^b, the canonical per-table form."""
    words = np.asarray(words).astype(np.uint32)
    Wd = (L + 31) // 32
    w = words.reshape(*words.shape[:-1], Wd, K)
    beta = np.arange(32, dtype=np.uint32)
    bits = (w[..., None] >> beta) & np.uint32(1)                 # [..., Wd, K, 32]
    weights = (np.uint32(1) << np.arange(K, dtype=np.uint32))[:, None]
    codes = (bits * weights).sum(axis=-2)                        # [..., Wd, 32]
    return codes.reshape(*words.shape[:-1], Wd * 32)[..., :L].astype(np.int32)
