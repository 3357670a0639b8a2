"""ctypes binding of liblsa.so: same names as include/lsa.h, argument marshalling only.

Every function takes torch tensors (device memory, plumbing) or None, passes their data pointers to
the C ABI and raises LsaError on a negative status.  Nothing is computed here, and there is no
fallback: a missing or unloadable library raises at first use.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_char_p, c_float, c_int, c_int32, c_int64, c_size_t, c_uint32, c_void_p

import torch

from .configs import LsaConfig

_LIB = None
# LSA_LIBRARY selects another build of the same library (the checking build liblsa_check.so, see build.py)
LIB_PATH = os.environ.get("LSA_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "liblsa.so")

LSA_KEY_BF16, LSA_KEY_E4M3 = 0, 1
LSA_POOL_MEAN, LSA_POOL_MINMAX = 0, 1
KERNEL_CLASSES = ("block_means", "coarse_score", "fine_select", "select", "convert", "sparse_attn", "merge_splits")


class LsaError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: {code} ({lib().lsa_strerror(code).decode()}) {detail}")


class LsaParams(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("n_heads_idx", c_int32), ("d_idx", c_int32), ("key_dtype", c_int32),
                ("page", c_int32), ("sub_block", c_int32), ("keep_pages", c_int32), ("k_sparse", c_int32),
                ("k_sink", c_int32), ("k_swa", c_int32), ("n_heads", c_int32), ("d_qk", c_int32), ("d_v", c_int32),
                ("sm_scale", c_float), ("n_layers", c_int32), ("q_chunk", c_int32), ("hi_enable", c_int32),
                ("paged", c_int32), ("kv_page", c_int32), ("pooling", c_int32)]


class LsaKvParams(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("dtype", c_int32), ("cache_e4m3", c_int32), ("latent", c_int32), ("n_heads", c_int32),
                ("n_kv_heads", c_int32), ("d_qk", c_int32), ("d_v", c_int32), ("kv_page", c_int32), ("d_rope", c_int32),
                ("rope_at", c_int32), ("rope_interleaved", c_int32), ("k_sink", c_int32), ("k_swa", c_int32), ("sm_scale", c_float)]


EXPORTS = {
    "lsa_create": (c_int, [POINTER(c_void_p), c_int, c_void_p, c_void_p, c_size_t]),
    "lsa_destroy": (c_int, [c_void_p]),
    "lsa_workspace_bytes": (c_int, [POINTER(LsaParams), c_int64, c_int64, c_int, POINTER(c_size_t)]),
    "lsa_status": (c_int, [c_void_p, POINTER(c_int)]),
    "lsa_strerror": (c_char_p, [c_int]),
    "lsa_last_cuda_error": (c_char_p, [c_void_p]),
    "lsa_launch_count": (c_int64, [c_void_p]),
    "lsa_tune": (c_int, [c_void_p, c_int, c_int]),
    "lsa_selftest_wait": (c_int, [c_void_p, c_int64]),
    "lsa_profile_enable": (c_int, [c_void_p, c_int]),
    "lsa_profile_read": (c_int, [c_void_p, POINTER(ctypes.c_double), POINTER(c_int64)]),
    "lsa_block_means": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_int64, c_void_p, c_int64,
                                c_void_p, c_int, c_void_p]),
    "lsa_index": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64,
                          c_int64, c_int64, c_void_p, c_int64, c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
    "lsa_index_static": (c_int, [c_int, c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_int64, c_int64, c_int64, c_void_p, c_void_p]),
    "lsa_index_static_status": (c_int, [c_int, c_void_p, POINTER(c_int)]),
    "lsa_select": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int64,
                           c_int32, c_int32, c_void_p, c_void_p]),
    "lsa_convert": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_int64, c_int64, c_void_p, c_int64,
                            c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
    "lsa_sparse_attn": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_void_p, c_int64, c_int64,
                                c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int64, c_void_p, c_int,
                                c_void_p, c_void_p]),
    "lsa_append": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64,
                           c_void_p, c_int, c_void_p, c_int, POINTER(c_void_p), POINTER(c_void_p), c_int64]),
    "lsa_merge": (c_int, [c_void_p, POINTER(LsaParams), c_int, POINTER(c_void_p), POINTER(c_void_p), c_int64, c_void_p,
                          c_void_p]),
    "lsa_layer_group": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_int64, c_int64, c_int64, c_void_p, c_int64, c_void_p, c_int, POINTER(c_void_p),
                                POINTER(c_void_p), POINTER(c_void_p), c_int64, c_int64, POINTER(c_void_p),
                                POINTER(c_void_p), c_void_p, c_void_p]),
    "lsa_layer_group_host": (c_int, [c_void_p, POINTER(LsaParams), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                     c_int64, c_int64, c_int64, POINTER(c_void_p), POINTER(c_void_p), POINTER(c_void_p),
                                     c_int64, c_int64, POINTER(c_void_p), c_int64, POINTER(c_void_p), c_size_t]),
    "lsa_kv_workspace_bytes": (c_int, [POINTER(LsaKvParams), POINTER(c_size_t)]),
    "lsa_kv_append": (c_int, [c_void_p, POINTER(LsaKvParams), c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                              c_int64, c_int64, c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                              c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int, c_void_p]),
    "lsa_paged_attn": (c_int, [c_void_p, POINTER(LsaKvParams), c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                               c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int, c_void_p, c_int64, c_void_p]),
    "lsa_host_stage_bytes": (c_int, [POINTER(LsaParams), c_int64, POINTER(c_size_t)]),
}


def lib() -> ctypes.CDLL:
    """The loaded library.  Raises if it has not been built: there is no other implementation."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2608_01662_b200.build` "
                               "(the CUDA library is the only implementation of this path)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _LIB = handle
    return _LIB


def make_params(cfg: LsaConfig) -> LsaParams:
    return LsaParams(ctypes.sizeof(LsaParams), cfg.H_I, cfg.d_I, LSA_KEY_E4M3 if cfg.key_dtype == "e4m3" else LSA_KEY_BF16,
                     cfg.P, cfg.B, cfg.M, cfg.Ksp, cfg.S, cfg.W, cfg.H, cfg.d_qk, cfg.d_v, cfg.sm_scale, cfg.R,
                     cfg.q_chunk, 1 if cfg.hi_enable else 0, 1 if cfg.mode == "decode" else 0, cfg.kv_page,
                     LSA_POOL_MINMAX if cfg.pooling == "minmax" else LSA_POOL_MEAN)


def _p(t):
    if t is None:
        return None
    if isinstance(t, int):
        return c_void_p(t)
    assert t.is_contiguous() or t.dim() == 2, "tensors are passed by base pointer"
    return c_void_p(t.data_ptr())


def _parr(ts):
    if ts is None:
        return None
    return (c_void_p * len(ts))(*[None if t is None else (t if isinstance(t, int) else t.data_ptr()) for t in ts])


def workspace_bytes(params: LsaParams, n_query: int, n_key_max: int, batch: int = 1) -> int:
    out = c_size_t(0)
    r = lib().lsa_workspace_bytes(ctypes.byref(params), n_query, n_key_max, batch, ctypes.byref(out))
    if r != 0:
        raise LsaError(r, "lsa_workspace_bytes")
    return out.value


def host_stage_bytes(params: LsaParams, stage_queries: int) -> int:
    out = c_size_t(0)
    r = lib().lsa_host_stage_bytes(ctypes.byref(params), stage_queries, ctypes.byref(out))
    if r != 0:
        raise LsaError(r, "lsa_host_stage_bytes")
    return out.value


_KV_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def make_kv_params(n_heads: int, n_kv_heads: int, d_qk: int, d_v: int, kv_page: int, latent: bool = False, dtype: str = "bf16",
                   e4m3: bool = False, d_rope: int = 0, rope_at: int = 0, rope_interleaved: bool = False, sink: int = 0,
                   window: int = 0, sm_scale: float | None = None) -> LsaKvParams:
    """lsa_kv_params: a paged key-value cache and the heads that read it.  sm_scale defaults to 1 / sqrt(d_qk)."""
    return LsaKvParams(ctypes.sizeof(LsaKvParams), tuple(_KV_DTYPES).index(dtype), int(e4m3), int(latent), n_heads, n_kv_heads, d_qk, d_v,
                       kv_page, d_rope, rope_at, int(rope_interleaved), sink, window, d_qk ** -0.5 if sm_scale is None else sm_scale)


def kv_workspace_bytes(kv: LsaKvParams) -> int:
    out = c_size_t(0)
    r = lib().lsa_kv_workspace_bytes(ctypes.byref(kv), ctypes.byref(out))
    if r != 0:
        raise LsaError(r, "lsa_kv_workspace_bytes")
    return out.value


def _kv_rows(t, heads: int, dims: int, dtype, where: str, rows: int, device: int = -1):
    """(pointer, elements from one row to the next) of rows of heads * dims elements, given as [rows, heads, dims] or [rows, heads * dims]
    on the device of that number (-1: the host)."""
    if t is None:
        return None, 0
    if t.dtype is dtype and t.shape == (rows, heads, dims) and t.get_device() == device and t.is_contiguous():   # (most calls end here)
        return t.data_ptr(), heads * dims
    st, sh = t.stride(), tuple(t.shape)
    if t.get_device() != device:
        raise LsaError(-1, where, f"a tensor on {t.device}: another device than the context's")
    inner = (sh == (rows, heads, dims) and (heads == 1 or st[1] == dims)) or sh == (rows, heads * dims)
    if not inner or st[-1] != 1 or t.dtype is not dtype:
        raise LsaError(-1, where, f"{rows} rows of {heads} heads of {dims} {dtype} wanted: got {sh} {t.dtype}, strides {st}")
    return t.data_ptr(), (st[0] if rows > 1 else max(st[0], heads * dims))


def _kv_flat(t, dtype, count: int, where: str, device: int = -1):
    """Pointer to a contiguous array of `count` elements."""
    if t is None:
        return None
    if t.get_device() != device:
        raise LsaError(-1, where, f"a tensor on {t.device}: another device than the context's")
    if t.dtype is not dtype or t.numel() != count or not t.is_contiguous():
        raise LsaError(-1, where, f"{count} contiguous {dtype} wanted: got {tuple(t.shape)} {t.dtype}")
    return t.data_ptr()


def _kv_table(t, where: str, device: int = -1):
    """(rows, entries from one row to the next, pointer) of a page table.  A row's length limit is its pitch: all of the last one has to
    lie in the tensor's memory, which it may not in a view of some columns."""
    sh = t.shape
    if t.dtype is not torch.int32 or len(sh) != 2 or t.get_device() != device:
        raise LsaError(-1, where, f"page_table: int32 [batch, pages] on the context's device wanted, got {tuple(sh)} {t.dtype} on {t.device}")
    if sh[0] <= 1 or t.is_contiguous():
        if sh[1] > 1 and t.stride(1) != 1:
            raise LsaError(-1, where, "page_table: contiguous rows wanted")
        return sh[0], sh[1], t.data_ptr()
    pitch = t.stride(0)
    if t.stride(1) != 1 or pitch < sh[1] or 4 * (t.storage_offset() + sh[0] * pitch) > t.untyped_storage().nbytes():
        raise LsaError(-1, where, f"page_table: contiguous rows wanted, the last one's whole pitch in memory; strides {t.stride()}")
    return sh[0], pitch, t.data_ptr()


STATIC_SCRATCH_BYTES = 8 << 20


def index_static(params: LsaParams, q_idx, w, k_idx, k_scale, kmean, q_pos0, n_query, n_key, sparse_idx, n_sparse,
                 stream=None):
    """lsa_index_static: the prefill indexer with its scratch inside the library (no context, no workspace)."""
    dev = q_idx.device
    stream = stream if stream is not None else torch.cuda.current_stream(dev)
    r = lib().lsa_index_static(dev.index or 0, c_void_p(stream.cuda_stream), ctypes.byref(params), _p(q_idx), _p(w),
                               _p(k_idx), _p(k_scale), _p(kmean), q_pos0, n_query, n_key, _p(sparse_idx), _p(n_sparse))
    if r != 0:
        raise LsaError(r, "lsa_index_static")


def index_static_status(device, stream=None) -> int:
    """lsa_index_static_status: waits for the stream, returns and clears the status word of lsa_index_static."""
    dev = _numbered(device)
    stream = stream if stream is not None else torch.cuda.current_stream(dev)
    st = c_int(0)
    r = lib().lsa_index_static_status(dev.index, c_void_p(stream.cuda_stream), ctypes.byref(st))
    if r != 0:
        raise LsaError(r, "lsa_index_static_status")
    return st.value


def _numbered(device) -> torch.device:
    """A CUDA device with its number: one without ("cuda") is the current one, as it is where tensors are made."""
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device


class Context:
    """lsa_ctx bound to the current torch CUDA stream; owns its workspace tensor."""

    def __init__(self, params: LsaParams | None, n_query: int, n_key_max: int, batch: int = 1, device=None, stream=None,
                 kv: LsaKvParams | None = None):
        """params: the sparse path's (None: the context serves kv_append and paged_attn only); kv: those calls' parameters."""
        if params is None and kv is None:
            raise LsaError(-1, "Context", "neither the sparse path's parameters nor those of a key-value cache")
        self.params, self.kv = params, kv
        self.device = _numbered(device if device is not None else "cuda:0")
        nbytes = workspace_bytes(params, n_query, n_key_max, batch) if params is not None else 0
        if kv is not None:
            nbytes = max(nbytes, kv_workspace_bytes(kv))
            # what every call needs of them (an attribute of a ctypes structure costs more than one of an object)
            self._kv_ref, self._kv_page, self._kv_rope = ctypes.byref(kv), kv.kv_page, kv.d_rope
            self._kv_dtype = tuple(_KV_DTYPES.values())[kv.dtype]
            self._kv_codes = {torch.float8_e4m3fn: torch.float8_e4m3fn} if kv.cache_e4m3 else None   # (else bytes)
            self._kv_k, self._kv_v, self._kv_q, self._kv_o = (kv.n_kv_heads, kv.d_qk), (kv.n_kv_heads, kv.d_v), (kv.n_heads, kv.d_qk), (kv.n_heads, kv.d_v)
            self._kv_dev, self._kv_append, self._paged_attn = self.device.index, lib().lsa_kv_append, lib().lsa_paged_attn
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = c_void_p()
        r = lib().lsa_create(ctypes.byref(h), self.device.index, c_void_p(self.stream.cuda_stream),
                             c_void_p(self.workspace.data_ptr()), nbytes)
        if r != 0:
            raise LsaError(r, "lsa_create")
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            lib().lsa_destroy(self.h)
            self.h = None

    __del__ = close

    def _chk(self, r, where):
        if r != 0:
            raise LsaError(r, where, lib().lsa_last_cuda_error(self.h).decode())

    def _sparse(self, where, params=None):
        """A sparse call's parameters: its own, or the context's."""
        params = params if params is not None else self.params
        if params is None:
            raise LsaError(-1, where, "the context was made without the sparse path's parameters")
        return ctypes.byref(params)

    def status(self) -> int:
        out = c_int(0)
        self._chk(lib().lsa_status(self.h, ctypes.byref(out)), "lsa_status")
        return out.value

    def launch_count(self) -> int:
        return lib().lsa_launch_count(self.h)

    def selftest_wait(self, budget_cycles: int):
        """lsa_selftest_wait: a bounded device-side wait that runs out (status() then returns LSA_ERR_TIMEOUT)."""
        self._chk(lib().lsa_selftest_wait(self.h, budget_cycles), "lsa_selftest_wait")

    def tune(self, knob: int, value: int):
        self._chk(lib().lsa_tune(self.h, knob, value), "lsa_tune")

    def profile_enable(self, on: bool):
        self._chk(lib().lsa_profile_enable(self.h, 1 if on else 0), "lsa_profile_enable")

    def profile_read(self) -> dict:
        """{kernel class: (total ms, launches)} since the last read."""
        n = len(KERNEL_CLASSES)
        ms, cnt = (ctypes.c_double * n)(), (c_int64 * n)()
        self._chk(lib().lsa_profile_read(self.h, ms, cnt), "lsa_profile_read")
        return {KERNEL_CLASSES[i]: (ms[i], cnt[i]) for i in range(n)}

    def block_means(self, k_idx, k_scale, n_key, kmean, page_table=None, ctx_len=None):
        pt_stride = page_table.shape[1] if page_table is not None else 0
        batch = page_table.shape[0] if page_table is not None else 1
        self._chk(lib().lsa_block_means(self.h, self._sparse("lsa_block_means"), _p(k_idx), _p(k_scale), n_key,
                                        _p(page_table), pt_stride, _p(ctx_len), batch, _p(kmean)), "lsa_block_means")

    def index(self, q_idx, w, k_idx, k_scale, kmean, q_pos0, n_query, n_key, sparse_idx, n_sparse, pages_out=None,
              page_table=None, ctx_len=None):
        pt_stride = page_table.shape[1] if page_table is not None else 0
        batch = page_table.shape[0] if page_table is not None else 1
        self._chk(lib().lsa_index(self.h, self._sparse("lsa_index"), _p(q_idx), _p(w), _p(k_idx), _p(k_scale),
                                  _p(kmean), q_pos0, n_query, n_key, _p(page_table), pt_stride, _p(ctx_len), batch,
                                  _p(sparse_idx), _p(n_sparse), _p(pages_out)), "lsa_index")

    def select(self, scores, cand_pos, q_pos0, k, apply_range, idx_out, n_out):
        n_query, n_cand = scores.shape
        self._chk(lib().lsa_select(self.h, self._sparse("lsa_select"), _p(scores), scores.stride(0), _p(cand_pos),
                                   q_pos0, n_query, n_cand, k, 1 if apply_range else 0, _p(idx_out), _p(n_out)),
                  "lsa_select")

    def convert(self, sparse_idx, n_sparse, q_pos0, n_query, rows_out, n_rows_out, runs_out=None, page_table=None,
                ctx_len=None):
        pt_stride = page_table.shape[1] if page_table is not None else 0
        batch = page_table.shape[0] if page_table is not None else 1
        self._chk(lib().lsa_convert(self.h, self._sparse("lsa_convert"), _p(sparse_idx), _p(n_sparse), q_pos0, n_query,
                                    _p(page_table), pt_stride, _p(ctx_len), batch, _p(rows_out), _p(n_rows_out),
                                    _p(runs_out)), "lsa_convert")

    def sparse_attn(self, q, k, v, sparse_idx, n_sparse, q_pos0, n_query, n_key, out, lse=None, rows=None,
                    n_rows=None, ctx_len=None, batch=1, params=None):
        self._chk(lib().lsa_sparse_attn(self.h, self._sparse("lsa_sparse_attn", params), _p(q), _p(k), _p(v), k.stride(0),
                                        v.stride(0), _p(sparse_idx), _p(n_sparse), _p(rows), _p(n_rows), q_pos0,
                                        n_query, n_key, _p(ctx_len), batch, _p(out), _p(lse)), "lsa_sparse_attn")

    def append(self, k_new, k_idx, k_scale, kmean, page_table, ctx_len, ctx_len_out=None, kv_new=(), kv_pool=()):
        batch = page_table.shape[0]
        row_bytes = kv_pool[0].stride(0) * kv_pool[0].element_size() if len(kv_pool) else 0
        self._chk(lib().lsa_append(self.h, self._sparse("lsa_append"), _p(k_new), _p(k_idx), _p(k_scale), _p(kmean),
                                   _p(page_table), page_table.shape[1], _p(ctx_len), batch, _p(ctx_len_out),
                                   len(kv_pool), _parr(list(kv_new)) if len(kv_pool) else None,
                                   _parr(list(kv_pool)) if len(kv_pool) else None, row_bytes), "lsa_append")

    def merge(self, outs, lses, n_query, out, lse=None, params=None):
        self._chk(lib().lsa_merge(self.h, self._sparse("lsa_merge", params), len(outs), _parr(outs), _parr(lses), n_query, _p(out),
                                  _p(lse)), "lsa_merge")

    def layer_group(self, q_idx, w, k_idx, k_scale, kmean, q_pos0, n_query, n_key, q, k, v, out, lse, sparse_idx,
                    n_sparse, page_table=None, ctx_len=None):
        pt_stride = page_table.shape[1] if page_table is not None else 0
        batch = page_table.shape[0] if page_table is not None else 1
        self._chk(lib().lsa_layer_group(self.h, self._sparse("lsa_layer_group"), _p(q_idx), _p(w), _p(k_idx), _p(k_scale),
                                        _p(kmean), q_pos0, n_query, n_key, _p(page_table), pt_stride, _p(ctx_len),
                                        batch, _parr(q), _parr(k), _parr(v), k[0].stride(0), v[0].stride(0),
                                        _parr(out), _parr(lse), _p(sparse_idx), _p(n_sparse)), "lsa_layer_group")

    def layer_group_host(self, q_idx_host, w_host, k_idx, k_scale, kmean, q_pos0, n_query, n_key, q_host, k, v, out_host,
                         stage_queries, stage):
        self._chk(lib().lsa_layer_group_host(self.h, self._sparse("lsa_layer_group_host"), _p(q_idx_host), _p(w_host), _p(k_idx),
                                             _p(k_scale), _p(kmean), q_pos0, n_query, n_key, _parr(q_host), _parr(k),
                                             _parr(v), k[0].stride(0), v[0].stride(0), _parr(out_host), stage_queries,
                                             _parr(stage), stage[0].numel()), "lsa_layer_group_host")

    def _kv_cache(self, k_pool, v_pool, k_scale, v_scale, page_table, ctx_len, where):
        """The arguments of a cache: pools as [rows, heads * dims] or [rows, heads, dims], scales as [rows, heads]."""
        if self.kv is None:
            raise LsaError(-1, where, "the context was made without kv parameters")
        dev, rows = self._kv_dev, k_pool.shape[0]
        n_pages, rest = divmod(rows, self._kv_page)
        if rest:
            raise LsaError(-1, where, f"a pool of {rows} rows is not a whole number of pages of {self._kv_page}")
        batch, pitch, pages = _kv_table(page_table, where, dev)
        cached = self._kv_codes.get(k_pool.dtype, torch.uint8) if self._kv_codes else self._kv_dtype
        k, ld_k = _kv_rows(k_pool, *self._kv_k, cached, where, rows, dev)
        v, ld_v = _kv_rows(v_pool, *self._kv_v, cached, where, rows, dev)
        ks, vs = (None, None) if k_scale is None and v_scale is None else (_kv_flat(x, torch.float32, rows * self._kv_k[0], where, dev) for x in (k_scale, v_scale))
        return (k, ld_k, v, ld_v, ks, vs, n_pages, pages, pitch, _kv_flat(ctx_len, torch.int32, batch, where, dev), batch)

    def kv_append(self, k_new, v_new, k_pool, v_pool, page_table, ctx_len, ctx_len_out=None, tok_start=None, q=None, q_out=None,
                  cos_sin=None, k_scale=None, v_scale=None):
        """lsa_kv_append: new tokens [n_tok, heads, dims] into the cache, rotated; q (optional) rotated into q_out."""
        where = "lsa_kv_append"
        cache = self._kv_cache(k_pool, v_pool, k_scale, v_scale, page_table, ctx_len, where)
        batch, dtype, n_pos, n_tok, dev = cache[-1], self._kv_dtype, 0, k_new.shape[0], self._kv_dev
        if cos_sin is not None:
            n_pos, width = cos_sin.shape if cos_sin.dim() == 2 else (0, -1)
            if width != self._kv_rope:
                raise LsaError(-1, where, f"cos_sin: [positions, {self._kv_rope}] wanted, got {tuple(cos_sin.shape)}")
        self._chk(self._kv_append(
            self.h, self._kv_ref, *_kv_rows(k_new, *self._kv_k, dtype, "k_new", n_tok, dev), *_kv_rows(v_new, *self._kv_v, dtype, "v_new", n_tok, dev),
            *_kv_rows(q, *self._kv_q, dtype, "q", n_tok, dev), *_kv_rows(q_out, *self._kv_q, dtype, "q_out", n_tok, dev), n_tok,
            _kv_flat(tok_start, torch.int32, batch + 1, "tok_start", dev), _kv_flat(cos_sin, torch.float32, n_pos * self._kv_rope, "cos_sin", dev), n_pos,
            *cache, _kv_flat(ctx_len_out, torch.int32, batch, "ctx_len_out", dev)), where)

    def paged_attn(self, q, k_pool, v_pool, page_table, ctx_len, out, lse=None, k_scale=None, v_scale=None):
        """lsa_paged_attn: q [batch, heads, d_qk] over each sequence's cached tokens -> out [batch, heads, d_v], lse [batch, heads]."""
        where = "lsa_paged_attn"
        cache = self._kv_cache(k_pool, v_pool, k_scale, v_scale, page_table, ctx_len, where)
        batch, dtype, dev = cache[-1], self._kv_dtype, self._kv_dev
        self._chk(self._paged_attn(self.h, self._kv_ref, *_kv_rows(q, *self._kv_q, dtype, "q", batch, dev), *cache,
                                   *_kv_rows(out, *self._kv_o, dtype, "out", batch, dev),
                                   _kv_flat(lse, torch.float32, batch * self._kv_o[0], "lse", dev)), where)
