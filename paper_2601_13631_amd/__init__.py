"""Python binding of libckv, the MI355X (gfx950) Re-Prefill hot path of ContiguousKV.

Argument marshalling only: every function forwards to the C ABI declared in
``include/ckv.h`` (same names without the ``ckv_`` prefix).  Every step of the
path runs in the library's HIP kernels; torch supplies device memory and
streams.  There is no fallback: if ``libckv.so`` is missing or fails to load,
importing this package raises.

Tensor arguments are torch tensors on the current HIP device (or, where the C
ABI allows host memory, pinned host tensors); they are passed by data pointer.
``stream`` defaults to torch's current stream.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libckv.so")

OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM, ESTATE = range(6)
DTYPE_F32, DTYPE_BF16, DTYPE_E4M3 = 0, 1, 2
CTX_HOST_PREFIX, CTX_MATERIALIZE, CTX_STAGE_TIMING, CTX_SCORE_TIMING = 0x1, 0x2, 0x4, 0x8
CACHE_ATTENTION, CACHE_LFU, CACHE_LOADS = 0, 1, 2
STORE_DIRECT = 0x1
TIER_NONE, TIER_CPU, TIER_GPU = 0, 1, 2
STAGES = ("score", "finalize", "select", "move", "attn")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libckv.so not built at {LIB_PATH}; run `python paper_2601_13631_amd/build.py`")
# torch first: libckv.so then binds to the HIP runtime that torch has loaded.  The
# other way round the process holds two, and what one allocates the other faults on.
import torch  # noqa: E402,F401

_lib = ctypes.CDLL(LIB_PATH)


class Dims(ctypes.Structure):
    """``ckv_dims``: the problem shape."""
    _fields_ = [
        ("n_prefix", ctypes.c_int64),
        ("n_suffix", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("chunk_size", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("sm_scale", ctypes.c_float),
    ]

    @property
    def n_chunks(self) -> int:
        return num_chunks(self.n_prefix, self.chunk_size)


class LayerIO(ctypes.Structure):
    """``ckv_layer_io``."""
    _fields_ = [(f, ctypes.c_void_p) for f in (
        "q", "k_suffix", "v_suffix", "k_probe", "k_prefix", "v_prefix", "kv_host", "kv_host_next",
        "out", "chunk_scores", "sel_idx", "stream", "pred_idx")] + [("n_pred", ctypes.c_int64)]


class LayerStats(ctypes.Structure):
    """``ckv_layer_stats``."""
    _fields_ = [(f, ctypes.c_int64) for f in (
        "k", "hits", "misses", "wasted", "bytes_prefetch", "bytes_demand", "bytes_gathered",
        "cache_hits", "bytes_cache_fill", "bytes_storage")]

    def as_dict(self) -> dict:
        return {f: int(getattr(self, f)) for f, _ in self._fields_}


class IoCounts(ctypes.Structure):
    """``ckv_io_counts``."""
    _fields_ = [(f, ctypes.c_int64) for f in ("tokens_selected", "runs", "blocks", "tokens_block")]


class CacheCounts(ctypes.Structure):
    """``ckv_cache_counts``."""
    _fields_ = [(f, ctypes.c_int64) for f in ("hits_gpu", "hits_cpu", "misses", "demoted", "dropped")]


class _PagePool(ctypes.Structure):
    """``ckv_page_pool``."""
    _fields_ = [(f, ctypes.c_void_p) for f in ("k", "v", "k_scale", "v_scale")] + [
        (f, ctypes.c_int64) for f in ("n_pages", "page_stride")] + [
        (f, ctypes.c_int32) for f in ("page_size", "n_kv_heads", "head_dim", "dtype")]


class _PageBatch(ctypes.Structure):
    """``ckv_page_batch``."""
    _fields_ = [(f, ctypes.c_void_p) for f in ("table", "lens", "tok_off")] + [
        (f, ctypes.c_int64) for f in ("table_stride", "n_tokens")] + [
        (f, ctypes.c_int32) for f in ("n_seqs", "max_pages", "max_tokens", "max_len")]


class _PageGroups(ctypes.Structure):
    """``ckv_page_groups``."""
    _fields_ = [(f, ctypes.c_void_p) for f in ("grp_off", "shared")] + [
        (f, ctypes.c_int32) for f in ("n_groups", "max_tokens", "max_shared")]


class _PageTables(ctypes.Structure):
    """``ckv_page_tables``."""
    _fields_ = [(f, ctypes.c_void_p) for f in (
        "table", "table_out", "lens", "lens_out", "refs", "refs_out")] + [
        (f, ctypes.c_int64) for f in ("table_stride", "table_out_stride", "n_pages")] + [
        (f, ctypes.c_int32) for f in ("n_seqs", "n_out", "max_pages", "page_size")]


class _SeqRows(ctypes.Structure):
    """``ckv_seq_rows``."""
    _fields_ = [(f, ctypes.c_void_p) for f in ("src", "dst")] + [
        (f, ctypes.c_int64) for f in ("row_bytes", "src_stride", "dst_stride")]


class _PageStep(ctypes.Structure):
    """``ckv_page_step``."""
    _fields_ = [(f, ctypes.c_void_p) for f in (
        "tok_off", "slots", "positions", "seqs", "copy_src", "copy_dst", "counts")] + [("n_tokens", ctypes.c_int64)]


class _Beams(ctypes.Structure):
    """``ckv_beams``."""
    _fields_ = [(f, ctypes.c_void_p) for f in ("logits", "scores", "done")] + [("row_stride", ctypes.c_int64)] + [
        (f, ctypes.c_int32) for f in ("n_reqs", "n_beams", "vocab", "keep", "eos", "dtype")]


_P = ctypes.c_void_p
_DP = ctypes.POINTER(Dims)
_PP = ctypes.POINTER(_PagePool)
_BP = ctypes.POINTER(_PageBatch)
_GP = ctypes.POINTER(_PageGroups)
_TP = ctypes.POINTER(_PageTables)
_I32, _I64, _SZ = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_SIG = {
    "ckv_last_error": ([], ctypes.c_char_p),
    "ckv_version": ([], ctypes.c_char_p),
    "ckv_num_chunks": ([ctypes.c_int64, ctypes.c_int32], ctypes.c_int64),
    "ckv_num_keep": ([ctypes.c_int64, ctypes.c_double], ctypes.c_int64),
    "ckv_score_workspace_bytes": ([_DP], ctypes.c_size_t),
    "ckv_score_chunks": ([_DP, _P, _P, _P, _P, ctypes.c_size_t, _P], ctypes.c_int32),
    "ckv_select_workspace_bytes": ([ctypes.c_int64], ctypes.c_size_t),
    "ckv_select_topk_chunks": ([_P, ctypes.c_int64, ctypes.c_int64, _P, _P, ctypes.c_size_t, _P],
                               ctypes.c_int32),
    "ckv_gather_chunks": ([_DP, _P, _P, _P, ctypes.c_int64, _P, _P, _P], ctypes.c_int32),
    "ckv_attn_workspace_bytes": ([_DP, ctypes.c_int64], ctypes.c_size_t),
    "ckv_debug_attn_wide_addressing": ([ctypes.c_int32], ctypes.c_int32),
    "ckv_sparse_prefill_attn": ([_DP, _P, _P, _P, _P, ctypes.c_int64, _P, _P, _P, _P,
                                 ctypes.c_size_t, _P], ctypes.c_int32),
    "ckv_ctx_create": ([_DP, ctypes.c_int32, ctypes.c_double, ctypes.c_int32, ctypes.POINTER(_P)],
                       ctypes.c_int32),
    "ckv_ctx_set_host_layers": ([_P, ctypes.POINTER(_P), ctypes.c_int32], ctypes.c_int32),
    "ckv_ctx_inject_copy_error": ([_P, ctypes.c_int32], ctypes.c_int32),
    "ckv_ctx_destroy": ([_P], ctypes.c_int32),
    "ckv_ctx_reset": ([_P], ctypes.c_int32),
    "ckv_ctx_set_period": ([_P, ctypes.c_int32], ctypes.c_int32),
    "ckv_ctx_attach_cache": ([_P, _P], ctypes.c_int32),
    "ckv_ctx_attach_store": ([_P, _P], ctypes.c_int32),
    "ckv_ctx_set_subperiod": ([_P, ctypes.c_int32], ctypes.c_int32),
    "ckv_store_open": ([ctypes.c_char_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                        ctypes.POINTER(_P)], ctypes.c_int32),
    "ckv_store_close": ([_P], ctypes.c_int32),
    "ckv_store_read": ([_P, _P, ctypes.c_int64, _P], ctypes.c_int32),
    "ckv_ctx_stage_times": ([_P, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)],
                            ctypes.c_int32),
    "ckv_reprefill_layer": ([_P, ctypes.c_int32, ctypes.POINTER(LayerIO),
                             ctypes.POINTER(LayerStats)], ctypes.c_int32),
    "ckv_reprefill_layer_noalloc": ([_DP, ctypes.c_double, _P, _P, _P, _P, _P, _P, _P, _P, _P],
                                    ctypes.c_int32),
    "ckv_io_account": ([ctypes.c_int64, ctypes.c_int32, _P, ctypes.c_int64, ctypes.c_int32,
                        ctypes.POINTER(IoCounts)], ctypes.c_int32),
    "ckv_cache_create": ([ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32,
                          ctypes.POINTER(_P)], ctypes.c_int32),
    "ckv_cache_destroy": ([_P], ctypes.c_int32),
    "ckv_cache_access": ([_P, _P, _P, ctypes.c_int64, _P, ctypes.POINTER(CacheCounts)],
                         ctypes.c_int32),
    "ckv_cache_lookup": ([_P, _P, ctypes.c_int64, _P], ctypes.c_int32),
    "ckv_cache_state": ([_P, _P, _P, _P], ctypes.c_int32),
    "ckv_cache_resident": ([_P, ctypes.c_int32, _P, ctypes.c_int64, ctypes.POINTER(ctypes.c_int64)],
                           ctypes.c_int32),
    "ckv_page_append": ([_PP, _BP, _P, _P, _P], _I32),
    "ckv_page_attn_workspace_bytes": ([_PP, _BP, _I32, _I32, _I32], _SZ),
    "ckv_page_attn": ([_PP, _BP, _P, _I32, ctypes.c_float, _I32, _I32, _P, _P, _SZ, _P], _I32),
    "ckv_page_copy": ([_PP, _I32, _P, _P, _I64, _P], _I32),
    "ckv_page_compact_workspace_bytes": ([_I64], _SZ),
    "ckv_page_compact": ([_PP, _I32, _P, _P, _I64, _P, _P, _I64, _P, _P, _SZ, _P], _I32),
    "ckv_page_share_ints": ([_I32, _I32], _I64),
    "ckv_page_share": ([_I32, _BP, _GP, _P], _I32),
    "ckv_page_attn_shared_workspace_bytes": ([_PP, _BP, _GP, _I32], _SZ),
    "ckv_page_attn_shared": ([_PP, _BP, _GP, _P, _I32, ctypes.c_float, _P, _P, _SZ, _P], _I32),
    "ckv_page_fork": ([_TP, _P, ctypes.POINTER(_SeqRows), _I32, _P], _I32),
    "ckv_page_extend_workspace_bytes": ([_I64, _I32], _SZ),
    "ckv_page_extend": ([_TP, _P, ctypes.POINTER(_PageStep), _P, _SZ, _P], _I32),
    "ckv_beam_select_workspace_bytes": ([ctypes.POINTER(_Beams)], _SZ),
    "ckv_beam_select": ([ctypes.POINTER(_Beams), _P, _P, _P, _P, _P, _SZ, _P], _I32),
}
for _name, (_args, _res) in _SIG.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _res

EXPORTED = tuple(_SIG)

# a valid host address for an empty caller prediction (n_pred = 0 with a
# non-NULL pred_idx); nothing is read from it
_EMPTY_PRED = (ctypes.c_int32 * 1)()
_EMPTY_PRED_ADDR = ctypes.addressof(_EMPTY_PRED)


class CkvError(RuntimeError):
    def __init__(self, status: int, what: str):
        msg = _lib.ckv_last_error().decode(errors="replace")
        super().__init__(f"{what} returned {status}: {msg}")
        self.status = status


def _check(status: int, what: str) -> None:
    if status != OK:
        raise CkvError(status, what)


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        # (the number alone: a torch.cuda.Stream made and asked for it takes 3 us)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def version() -> str:
    return _lib.ckv_version().decode()


def last_error() -> str:
    return _lib.ckv_last_error().decode(errors="replace")


def num_chunks(n: int, c: int) -> int:
    return int(_lib.ckv_num_chunks(n, c))


def num_keep(m: int, r: float) -> int:
    return int(_lib.ckv_num_keep(m, r))


def make_dims(n_prefix, n_suffix, n_q_heads, n_kv_heads, head_dim, chunk_size, dtype=DTYPE_BF16,
              sm_scale=0.0) -> Dims:
    return Dims(n_prefix, n_suffix, n_q_heads, n_kv_heads, head_dim, chunk_size, dtype, sm_scale)


def score_workspace_bytes(dims: Dims) -> int:
    return int(_lib.ckv_score_workspace_bytes(ctypes.byref(dims)))


def score_chunks(dims: Dims, q, k_prefix, chunk_scores, ws, stream=None) -> None:
    _check(_lib.ckv_score_chunks(ctypes.byref(dims), _ptr(q), _ptr(k_prefix), _ptr(chunk_scores),
                                 _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0,
                                 _stream(stream)), "ckv_score_chunks")


def select_workspace_bytes(m: int) -> int:
    return int(_lib.ckv_select_workspace_bytes(m))


def select_topk_chunks(chunk_scores, m: int, k: int, sel_idx, ws=None, stream=None) -> None:
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check(_lib.ckv_select_topk_chunks(_ptr(chunk_scores), m, k, _ptr(sel_idx), _ptr(ws), nbytes,
                                       _stream(stream)), "ckv_select_topk_chunks")


def gather_chunks(dims: Dims, k_src, v_src, sel_idx, k: int, k_sel, v_sel, stream=None) -> None:
    _check(_lib.ckv_gather_chunks(ctypes.byref(dims), _ptr(k_src), _ptr(v_src), _ptr(sel_idx), k,
                                  _ptr(k_sel), _ptr(v_sel), _stream(stream)), "ckv_gather_chunks")


def attn_workspace_bytes(dims: Dims, k: int) -> int:
    return int(_lib.ckv_attn_workspace_bytes(ctypes.byref(dims), k))


def debug_attn_wide_addressing(force_wide: bool) -> None:
    """Test hook: every later attention launch reads K/V through 64-bit row
    addresses (the form sources past 4 GiB take) instead of 32-bit offsets."""
    _check(_lib.ckv_debug_attn_wide_addressing(1 if force_wide else 0),
           "ckv_debug_attn_wide_addressing")


def sparse_prefill_attn(dims: Dims, q, k_sel, v_sel, sel_idx, k: int, k_suffix, v_suffix, out,
                        ws=None, stream=None) -> None:
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check(_lib.ckv_sparse_prefill_attn(ctypes.byref(dims), _ptr(q), _ptr(k_sel), _ptr(v_sel),
                                        _ptr(sel_idx), k, _ptr(k_suffix), _ptr(v_suffix), _ptr(out),
                                        _ptr(ws), nbytes, _stream(stream)),
           "ckv_sparse_prefill_attn")


NOALLOC_SCRATCH_BYTES = 64 << 20


def reprefill_layer_noalloc(dims: Dims, keep_ratio: float, q, k_prefix, v_prefix, k_suffix, v_suffix,
                            out, chunk_scores=None, sel_idx=None, stream=None) -> None:
    """``ckv_reprefill_layer_noalloc``: one HBM-resident layer step that allocates
    nothing (scratch in the library's fixed device array)."""
    _check(_lib.ckv_reprefill_layer_noalloc(ctypes.byref(dims), keep_ratio, _ptr(q), _ptr(k_prefix),
                                            _ptr(v_prefix), _ptr(k_suffix), _ptr(v_suffix),
                                            _ptr(out), _ptr(chunk_scores), _ptr(sel_idx),
                                            _stream(stream)),
           "ckv_reprefill_layer_noalloc")


class Context:
    """``ckv_ctx``: owns workspace, streams, events and (host-resident prefix) HBM slots."""

    def __init__(self, dims: Dims, n_layers: int, keep_ratio: float, flags: int = 0):
        self.dims = dims
        self._h = ctypes.c_void_p()
        _check(_lib.ckv_ctx_create(ctypes.byref(dims), n_layers, keep_ratio, flags,
                                   ctypes.byref(self._h)), "ckv_ctx_create")
        self.n_layers = n_layers
        self.k = num_keep(dims.n_chunks, keep_ratio)

    def reprefill_layer(self, layer: int, q, k_suffix, v_suffix, k_probe, out, k_prefix=None,
                        v_prefix=None, kv_host=None, kv_host_next=None, chunk_scores=None,
                        sel_idx=None, stream=None, pred_idx=None) -> dict:
        """``pred_idx``: this layer's predicted chunks (ascending; a host numpy
        array or sequence, possibly empty), or None for the context's own."""
        pred = None
        if pred_idx is not None:
            import numpy as np
            pred = np.ascontiguousarray(pred_idx, np.int32)
            if pred.size == 0:
                pred = np.zeros(1, np.int32)[:0]
        io = LayerIO(_ptr(q), _ptr(k_suffix), _ptr(v_suffix), _ptr(k_probe), _ptr(k_prefix),
                     _ptr(v_prefix), _ptr(kv_host), _ptr(kv_host_next), _ptr(out),
                     _ptr(chunk_scores), _ptr(sel_idx), _stream(stream),
                     None if pred is None else (pred.ctypes.data or _EMPTY_PRED_ADDR),
                     0 if pred is None else pred.size)
        st = LayerStats()
        _check(_lib.ckv_reprefill_layer(self._h, layer, ctypes.byref(io), ctypes.byref(st)),
               "ckv_reprefill_layer")
        return st.as_dict()

    def stage_times(self) -> tuple:
        """(per-stage total ms dict, number of layers) since creation or reset."""
        ms = (ctypes.c_double * len(STAGES))()
        n = ctypes.c_int64()
        _check(_lib.ckv_ctx_stage_times(self._h, ms, ctypes.byref(n)), "ckv_ctx_stage_times")
        return dict(zip(STAGES, list(ms))), int(n.value)

    def reset(self) -> None:
        _check(_lib.ckv_ctx_reset(self._h), "ckv_ctx_reset")

    def set_period(self, period: int) -> None:
        """Layers p*i .. p*i+p-1 share the set selected at layer p*i."""
        _check(_lib.ckv_ctx_set_period(self._h, period), "ckv_ctx_set_period")

    def attach_cache(self, cache) -> None:
        """Keeps the GPU tier of ``cache`` (a :class:`Cache`, or None to detach)
        in HBM slots for this host-resident context."""
        self._cache = cache  # the context must not outlive the cache it uses
        _check(_lib.ckv_ctx_attach_cache(self._h, cache._h if cache is not None else None),
               "ckv_ctx_attach_cache")

    def set_host_layers(self, stores) -> None:
        """Registers the pinned host store of every layer (a list of n_layers
        pinned tensors), or unregisters them (None)."""
        self._host_layers = stores  # kept alive while registered
        if stores is None:
            _check(_lib.ckv_ctx_set_host_layers(self._h, None, 0), "ckv_ctx_set_host_layers")
            return
        arr = (_P * len(stores))(*[_ptr(t) for t in stores])
        _check(_lib.ckv_ctx_set_host_layers(self._h, arr, len(stores)), "ckv_ctx_set_host_layers")

    def inject_copy_error(self, layer: int) -> None:
        """Test hook: the next run of ``layer`` fails at its demand copies (-1 disarms)."""
        _check(_lib.ckv_ctx_inject_copy_error(self._h, layer), "ckv_ctx_inject_copy_error")

    def set_subperiod(self, subperiod: int) -> None:
        """Storage reads up to subperiod - 1 layers ahead inside a Period."""
        _check(_lib.ckv_ctx_set_subperiod(self._h, subperiod), "ckv_ctx_set_subperiod")

    def attach_store(self, store) -> None:
        """Takes the chunks of this host-resident context from ``store`` (a
        :class:`Store`, or None to detach)."""
        self._store = store  # the context must not outlive the store it reads
        _check(_lib.ckv_ctx_attach_store(self._h, store._h if store is not None else None),
               "ckv_ctx_attach_store")

    def close(self) -> None:
        if self._h:
            _check(_lib.ckv_ctx_destroy(self._h), "ckv_ctx_destroy")
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _host_ptr(a) -> int | None:
    """Address of a contiguous host numpy array."""
    return a.ctypes.data if a is not None and a.size else None


def io_account(n: int, c: int, sel_idx, block_tokens: int = 64) -> dict:
    """``ckv_io_account``: tokens read for the ascending chunk indices sel_idx (host)
    by a ContiguousChunk store and by a store of block_tokens-token blocks."""
    import numpy as np
    sel = np.ascontiguousarray(sel_idx, np.int32)
    out = IoCounts()
    _check(_lib.ckv_io_account(n, c, _host_ptr(sel), sel.size, block_tokens, ctypes.byref(out)),
           "ckv_io_account")
    return {f: int(getattr(out, f)) for f, _ in out._fields_}


class Cache:
    """``ckv_cache``: the attention-guided two-tier chunk cache (host memory)."""

    def __init__(self, n_keys: int, gpu_slots: int, cpu_slots: int, policy: int = CACHE_ATTENTION):
        self.n_keys = n_keys
        self._h = ctypes.c_void_p()
        _check(_lib.ckv_cache_create(n_keys, gpu_slots, cpu_slots, policy, ctypes.byref(self._h)),
               "ckv_cache_create")

    def access(self, keys, scores):
        """One request's used chunks; returns (tier each was found in, totals dict)."""
        import numpy as np
        keys = np.ascontiguousarray(keys, np.int64)
        scores = np.ascontiguousarray(scores, np.float64)
        if keys.size != scores.size:
            raise ValueError("keys and scores differ in length")
        where = np.zeros(keys.size, np.int8)
        cnt = CacheCounts()
        _check(_lib.ckv_cache_access(self._h, _host_ptr(keys), _host_ptr(scores), keys.size,
                                     _host_ptr(where), ctypes.byref(cnt)), "ckv_cache_access")
        return where, {f: int(getattr(cnt, f)) for f, _ in cnt._fields_}

    def lookup(self, keys):
        import numpy as np
        keys = np.ascontiguousarray(keys, np.int64)
        tier = np.zeros(keys.size, np.int8)
        _check(_lib.ckv_cache_lookup(self._h, _host_ptr(keys), keys.size, _host_ptr(tier)),
               "ckv_cache_lookup")
        return tier

    def state(self):
        """(I, F, tier) arrays over every key."""
        import numpy as np
        I = np.zeros(self.n_keys, np.float64)
        F = np.zeros(self.n_keys, np.int64)
        tier = np.zeros(self.n_keys, np.int8)
        _check(_lib.ckv_cache_state(self._h, _host_ptr(I), _host_ptr(F), _host_ptr(tier)),
               "ckv_cache_state")
        return I, F, tier

    def resident(self, tier: int):
        import numpy as np
        n = ctypes.c_int64()
        keys = np.zeros(self.n_keys, np.int64)
        _check(_lib.ckv_cache_resident(self._h, tier, _host_ptr(keys), keys.size, ctypes.byref(n)),
               "ckv_cache_resident")
        return keys[: n.value].copy()

    def close(self) -> None:
        if self._h:
            _check(_lib.ckv_cache_destroy(self._h), "ckv_cache_destroy")
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Store:
    """``ckv_store``: a file of fixed-size spans read by I/O threads (the storage tier)."""

    def __init__(self, path: str, n_keys: int, span_bytes: int, io_threads: int = 8, flags: int = 0):
        self.span_bytes = span_bytes
        self._h = ctypes.c_void_p()
        _check(_lib.ckv_store_open(os.fsencode(path), n_keys, span_bytes, io_threads, flags,
                                   ctypes.byref(self._h)), "ckv_store_open")

    def read(self, keys, dst) -> None:
        """Spans ``keys`` into ``dst`` (a host numpy array or tensor of len(keys) spans)."""
        import numpy as np
        keys = np.ascontiguousarray(keys, np.int64)
        nbytes = dst.nbytes if hasattr(dst, "nbytes") else dst.numel() * dst.element_size()
        if nbytes < keys.size * self.span_bytes:
            raise ValueError("destination smaller than the spans read")
        ptr = dst.ctypes.data if hasattr(dst, "ctypes") else dst.data_ptr()
        _check(_lib.ckv_store_read(self._h, _host_ptr(keys), keys.size, ptr), "ckv_store_read")

    def close(self) -> None:
        if self._h:
            _check(_lib.ckv_store_close(self._h), "ckv_store_close")
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _need(t, what: str, dtype, shape=None):
    """``t`` if it is a contiguous tensor of the current HIP device, of this type and shape."""
    # (of a device tensor: torch.cuda.current_device() without its look whether HIP has begun)
    if (t.dtype is dtype and t.is_cuda and t.get_device() == torch._C._cuda_getDevice()
            and (shape is None or t.shape == shape) and t.is_contiguous()):
        return t
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what} must be on the current device (it is on {t.device})")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype} (it is {t.dtype})")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)} (it has {tuple(t.shape)})")
    raise ValueError(f"{what} must be contiguous")


def _together(t, *handles) -> int:
    """The device of ``t``, the current one, where the handles' tensors have to be as well."""
    device = t.get_device()
    for h in handles:
        if h._device != device:
            raise ValueError(f"the {type(h).__name__} is on device {h._device}, the call's tensors on {device}")
    return device


def _current(device: int) -> int:
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"the call's tensors are on device {device}, not the current one")
    return device


def _stream_on(device: int, stream) -> int | None:
    """``_stream`` where the current device is known."""
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)


def _workspace(ws, t):
    """Address and bytes of a workspace, on the device of ``t``."""
    if ws is None:
        return None, 0
    if ws.get_device() != t.get_device() or not ws.is_contiguous():
        raise ValueError(f"the workspace must be contiguous and on the call's device (it is on {ws.device})")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _int32(x, what: str) -> int:
    """``x`` as a C int that is not negative."""
    if not 0 <= x < 1 << 31:
        raise ValueError(f"{what} must be in [0, 2^31) (it is {x})")
    return int(x)


_PAGE_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float8_e4m3fn: DTYPE_E4M3}


class PagePool:
    """``ckv_page_pool``: one layer's pages.

    ``k`` and ``v``: float32, bfloat16 or float8_e4m3fn tensors
    [n_pages, page_size, n_kv_heads, head_dim] of the current device, whose pages are
    contiguous and may lie apart (``stride(0)``, the same for both); with
    float8_e4m3fn, ``k_scale`` and ``v_scale``: contiguous uint8 tensors
    [n_pages, n_kv_heads].  Keeps the tensors alive; make it once and keep it (2 to 3 us).
    """

    def __init__(self, k, v, k_scale=None, v_scale=None):
        shape, dtype, stride, v_stride = k.shape, k.dtype, k.stride(), v.stride()
        if len(shape) != 4 or v.shape != shape or v.dtype is not dtype:
            raise ValueError("k and v must be of one type and shape [n_pages, page_size, n_kv_heads, head_dim]")
        number = _PAGE_DTYPES.get(dtype)
        if number is None:
            raise ValueError(f"pages are float32, bfloat16 or float8_e4m3fn (not {dtype})")
        n_pages, page_size, hkv, d = shape
        for t in (k, v):
            if not t.is_cuda or t.get_device() != torch._C._cuda_getDevice():
                raise ValueError(f"pages must be on the current device (they are on {t.device})")
        if hkv == 1:  # (where there is one head, its stride is not used)
            stride, v_stride = ((*s[:2], d, s[3]) for s in (stride, v_stride))
        if stride[1:] != (hkv * d, d, 1) or (v_stride != stride if n_pages > 1 else v_stride[1:] != stride[1:]):
            raise ValueError("a page's rows must be contiguous, and K and V pages equally far apart")
        if n_pages > 1 and stride[0] < page_size * hkv * d:  # (0, of an expanded tensor, would mean dense)
            raise ValueError(f"pages must not overlap (they are {stride[0]} elements apart)")
        if (number == DTYPE_E4M3) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            raise ValueError("k_scale and v_scale belong to float8_e4m3fn pages, and to those only")
        if k_scale is not None:
            _need(k_scale, "k_scale", torch.uint8, (n_pages, hkv))
            _need(v_scale, "v_scale", torch.uint8, (n_pages, hkv))
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.page_size, self.n_kv_heads, self.head_dim = n_pages, page_size, hkv, d
        self._device = k.get_device()
        self.token_dtype = torch.float32 if number == DTYPE_F32 else torch.bfloat16
        self._c = _PagePool(k.data_ptr(), v.data_ptr(), _ptr(k_scale), _ptr(v_scale), n_pages,
                            stride[0] if n_pages > 1 else 0, page_size, hkv, d, number)


class PageLayers:
    """The pools of a model's layers (same shapes throughout) as one handle for
    :func:`page_copy` and :func:`page_compact`."""

    def __init__(self, pools):
        self.pools = tuple(pools)
        self.n_pages = self.pools[0].n_pages if self.pools else 0
        self._device = self.pools[0]._device if self.pools else None
        if any(p._device != self._device for p in self.pools):
            raise ValueError("the pools must be on one device")
        self._c = (_PagePool * len(self.pools))(*(p._c for p in self.pools))


class PageBatch:
    """``ckv_page_batch``: the sequences of one call.

    ``table`` (int32 [n_seqs, max_pages], rows may lie apart), ``lens`` (int32
    [n_seqs]) and ``tok_off`` (int32 [n_seqs + 1]) are device tensors, read when the
    call's kernels run; ``n_tokens`` is the number of rows of the call's token
    tensors.  ``max_tokens`` and ``max_len``: about the most tokens of a sequence
    and the greatest length (0: not known, taken for ``n_tokens`` and the table's: say
    1 for decoding, which is otherwise given the kernel for prompts).  Keeps the tensors
    alive; one handle serves every call on the same tensors.
    """

    def __init__(self, table, lens, tok_off, n_tokens: int, max_tokens: int = 0, max_len: int = 0):
        if table.dim() != 2 or (table.shape[0] > 0 and table.stride(1) != 1 and table.shape[1] > 1):
            raise ValueError("table must be [n_seqs, max_pages] with contiguous rows")
        n_seqs, width = table.shape
        if table.dtype != torch.int32 or not table.is_cuda or table.device.index != torch.cuda.current_device():
            raise ValueError("table must be an int32 tensor of the current device")
        _need(lens, "lens", torch.int32, (n_seqs,))
        _need(tok_off, "tok_off", torch.int32, (n_seqs + 1,))
        stride = table.stride(0) if n_seqs > 1 else width
        if stride < width:
            raise ValueError("the table's rows must not overlap")
        _int32(n_tokens, "n_tokens")
        self.table, self.lens, self.tok_off = table, lens, tok_off
        self.n_seqs, self.n_tokens = n_seqs, int(n_tokens)
        self._device = table.get_device()
        self._c = _PageBatch(_ptr(table), _ptr(lens), _ptr(tok_off), stride, n_tokens, n_seqs, width,
                             _int32(max_tokens, "max_tokens"), _int32(max_len, "max_len"))


def page_append(pool: PagePool, batch: PageBatch, k_new, v_new, stream=None) -> None:
    """``ckv_page_append``: the batch's tokens' K and V rows (``[n_tokens, n_kv_heads,
    head_dim]``, float32 for a float32 pool, else bfloat16) into their pages."""
    shape = (batch.n_tokens, pool.n_kv_heads, pool.head_dim)
    _need(k_new, "k_new", pool.token_dtype, shape)
    _need(v_new, "v_new", pool.token_dtype, shape)
    device = _together(k_new, pool, batch)
    _check(_lib.ckv_page_append(pool._c, batch._c, k_new.data_ptr(), v_new.data_ptr(),
                                _stream_on(device, stream)),
           "ckv_page_append")


def page_attn_workspace_bytes(pool: PagePool, batch: PageBatch, n_q_heads: int, window: int = 0,
                              n_sinks: int = 0) -> int:
    return int(_lib.ckv_page_attn_workspace_bytes(pool._c, batch._c, _int32(n_q_heads, "n_q_heads"),
                                                  _int32(window, "window"), _int32(n_sinks, "n_sinks")))


def page_attn(pool: PagePool, batch: PageBatch, q, out, ws=None, window: int = 0, n_sinks: int = 0,
              sm_scale: float = 0.0, stream=None) -> None:
    """``ckv_page_attn``: attention of the batch's tokens over their sequences' pages.

    ``q`` and ``out``: ``[n_tokens, n_q_heads, head_dim]``, float32 for a float32
    pool, else bfloat16.  ``ws``: a uint8 tensor of
    :func:`page_attn_workspace_bytes` bytes (None where that is 0).
    """
    shape = q.shape
    if len(shape) != 3 or shape[0] != batch.n_tokens or shape[2] != pool.head_dim:
        raise ValueError("q must be [n_tokens, n_q_heads, head_dim]")
    _need(q, "q", pool.token_dtype)
    _need(out, "out", pool.token_dtype, shape)
    device = _together(q, pool, batch)
    ws_ptr, nbytes = _workspace(ws, q)
    _check(_lib.ckv_page_attn(pool._c, batch._c, q.data_ptr(), shape[1], sm_scale,
                              _int32(window, "window"), _int32(n_sinks, "n_sinks"), out.data_ptr(), ws_ptr,
                              nbytes, _stream_on(device, stream)), "ckv_page_attn")


def page_copy(layers: PageLayers, src, dst, stream=None) -> None:
    """``ckv_page_copy``: page ``src[i]`` to page ``dst[i]`` (int32 device tensors) in
    every layer."""
    _need(src, "src", torch.int32)
    _need(dst, "dst", torch.int32, src.shape)
    device = _together(src, layers) if layers.pools else src.get_device()
    _check(_lib.ckv_page_copy(layers._c, len(layers.pools), src.data_ptr(), dst.data_ptr(), src.numel(),
                              _stream_on(device, stream)), "ckv_page_copy")


def page_compact_workspace_bytes(n_pages: int) -> int:
    return int(_lib.ckv_page_compact_workspace_bytes(n_pages))


def page_compact(layers: PageLayers, refs, refs_out, table, table_out, n_live, ws, stream=None) -> None:
    """``ckv_page_compact``: the pages in use (``refs`` > 0) to the front of every layer's
    pool.  ``refs``, ``refs_out``: int32 [n_pages]; ``table``, ``table_out``: int32 tensors of
    one shape (or None); ``n_live``: int32 [1]; ``ws``: a uint8 tensor of
    :func:`page_compact_workspace_bytes` bytes.  The outputs may be the inputs."""
    _need(refs, "refs", torch.int32)
    _need(refs_out, "refs_out", torch.int32, refs.shape)
    _need(n_live, "n_live", torch.int32, (1,))
    if table is not None:
        _need(table, "table", torch.int32)
        _need(table_out, "table_out", torch.int32, table.shape)
    device = _together(refs, layers) if layers.pools else refs.get_device()
    ws_ptr, nbytes = _workspace(ws, refs)
    _check(_lib.ckv_page_compact(layers._c, len(layers.pools), refs.data_ptr(), refs_out.data_ptr(),
                                 refs.numel(), _ptr(table), _ptr(table_out) if table is not None else None,
                                 table.numel() if table is not None else 0, n_live.data_ptr(), ws_ptr,
                                 nbytes, _stream_on(device, stream)), "ckv_page_compact")


class PageGroups:
    """``ckv_page_groups``: the groups of a batch whose sequences share their first pages.

    ``grp_off`` (int32 [n_groups + 1], device): group g is the sequences ``grp_off[g]`` to
    ``grp_off[g + 1] - 1``.  ``shared``: an int32 tensor of :func:`page_share_ints` numbers,
    which :func:`page_share` writes.  ``max_tokens`` and ``max_shared``: about the most tokens
    of one group's sequences together, and the most that one shares (0: not known).  Keeps
    the tensors alive; one handle serves every step on the same tensors.
    """

    def __init__(self, grp_off, shared, max_tokens: int = 0, max_shared: int = 0):
        if grp_off.dim() != 1 or grp_off.shape[0] < 1:
            raise ValueError("grp_off must be [n_groups + 1]")
        _need(grp_off, "grp_off", torch.int32)
        _need(shared, "shared", torch.int32)
        self.grp_off, self.shared = grp_off, shared
        self.n_groups = grp_off.shape[0] - 1
        self._device = grp_off.get_device()
        self._c = _PageGroups(_ptr(grp_off), _ptr(shared), self.n_groups, _int32(max_tokens, "max_tokens"),
                              _int32(max_shared, "max_shared"))

    def _fits(self, batch: PageBatch) -> None:
        if self.shared.numel() < 2 * self.n_groups + batch.n_seqs:
            raise ValueError(f"shared must have {2 * self.n_groups + batch.n_seqs} numbers (it has "
                             f"{self.shared.numel()})")


def page_share_ints(n_groups: int, n_seqs: int) -> int:
    return int(_lib.ckv_page_share_ints(_int32(n_groups, "n_groups"), _int32(n_seqs, "n_seqs")))


def page_share(page_size: int, batch: PageBatch, groups: PageGroups, stream=None) -> None:
    """``ckv_page_share``: what each group's sequences share, for :func:`page_attn_shared` in
    every layer; again whenever the table, the lengths or the offsets have changed."""
    groups._fits(batch)
    device = _current(_together(groups.grp_off, groups, batch))
    _check(_lib.ckv_page_share(_int32(page_size, "page_size"), batch._c, groups._c, _stream_on(device, stream)),
           "ckv_page_share")


def page_attn_shared_workspace_bytes(pool: PagePool, batch: PageBatch, groups: PageGroups, n_q_heads: int) -> int:
    return int(_lib.ckv_page_attn_shared_workspace_bytes(pool._c, batch._c, groups._c,
                                                         _int32(n_q_heads, "n_q_heads")))


def page_attn_shared(pool: PagePool, batch: PageBatch, groups: PageGroups, q, out, ws=None, sm_scale: float = 0.0,
                     stream=None) -> None:
    """``ckv_page_attn_shared``: :func:`page_attn` without a window, the pages that a group's
    sequences share read once for all of them (``groups`` as :func:`page_share` left it).

    ``ws``: a uint8 tensor of :func:`page_attn_shared_workspace_bytes` bytes (None where that is 0).
    """
    shape = q.shape
    if len(shape) != 3 or shape[0] != batch.n_tokens or shape[2] != pool.head_dim:
        raise ValueError("q must be [n_tokens, n_q_heads, head_dim]")
    _need(q, "q", pool.token_dtype)
    _need(out, "out", pool.token_dtype, shape)
    groups._fits(batch)
    device = _together(q, pool, batch, groups)
    ws_ptr, nbytes = _workspace(ws, q)
    _check(_lib.ckv_page_attn_shared(pool._c, batch._c, groups._c, q.data_ptr(), shape[1], sm_scale,
                                     out.data_ptr(), ws_ptr, nbytes, _stream_on(device, stream)),
           "ckv_page_attn_shared")


def _rows(t, what: str) -> int:
    """Elements between the rows of an int32 table of the current device."""
    if t.dim() != 2 or t.dtype != torch.int32 or not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what} must be an int32 tensor [n_seqs, max_pages] of the current device")
    n, width = t.shape
    if n > 0 and width > 1 and t.stride(1) != 1:
        raise ValueError(f"{what} must have contiguous rows")
    stride = t.stride(0) if n > 1 else width
    if stride < width:
        raise ValueError(f"the rows of {what} must not overlap")
    return stride


def _tables(page_size, table, table_out, lens, lens_out, refs, refs_out) -> _PageTables:
    stride, out_stride = _rows(table, "table"), _rows(table_out, "table_out")
    if table_out.shape[1] != table.shape[1]:
        raise ValueError("table and table_out must be equally wide")
    _need(lens, "lens", torch.int32, table.shape[:1])
    _need(lens_out, "lens_out", torch.int32, table_out.shape[:1])
    _need(refs, "refs", torch.int32)
    _need(refs_out, "refs_out", torch.int32, refs.shape)
    return _PageTables(_ptr(table), _ptr(table_out), _ptr(lens), _ptr(lens_out), _ptr(refs), _ptr(refs_out),
                       stride, out_stride, refs.numel(), table.shape[0], table_out.shape[0], table.shape[1],
                       _int32(page_size, "page_size"))


class PageFork:
    """What :func:`page_fork` reads and writes, as one handle.

    ``table`` [n_seqs, max_pages], ``lens`` [n_seqs] and ``refs`` [n_pages] (int32, device) are the
    sequences as they are, ``table_out`` [n_out, max_pages], ``lens_out`` [n_out] and ``refs_out`` (which
    may be ``refs``) those after the call.  ``states``: pairs of tensors [n_seqs, ...] and
    [n_out, ...] of one type whose rows follow the sequences, up to eight; a row is
    contiguous, rows may lie apart.  What is written shares no memory with the rest, but ``refs_out`` with
    ``refs``.  Keeps the tensors alive; make it once per pair of buffers.
    """

    def __init__(self, page_size: int, table, table_out, lens, lens_out, refs, refs_out, states=()):
        self._c = _tables(page_size, table, table_out, lens, lens_out, refs, refs_out)
        self.n_seqs, self.n_out = table.shape[0], table_out.shape[0]
        self._device = refs.get_device()
        self._tensors = (table, table_out, lens, lens_out, refs, refs_out, *(t for pair in states for t in pair))
        rows = []
        for src, dst in states:
            if src.dtype != dst.dtype or src.shape[1:] != dst.shape[1:]:
                raise ValueError("a state's tensors must be of one type and row shape")
            if src.dim() < 1 or src.shape[0] != self.n_seqs or dst.shape[0] != self.n_out:
                raise ValueError(f"a state needs {self.n_seqs} rows, and {self.n_out} to write")
            strides = []
            for t in (src, dst):
                if not t.is_cuda or t.get_device() != self._device:
                    raise ValueError(f"states must be on the current device (one is on {t.device})")
                if t.shape[0] > 0 and not t[0].is_contiguous():
                    raise ValueError("a state's rows must be contiguous")
                strides.append(t.stride(0) * t.element_size() if t.shape[0] > 1 else 0)
            nbytes = src[0].numel() * src.element_size() if self.n_seqs > 0 else 0
            if nbytes == 0:
                continue
            if any(t.shape[0] > 1 and s < nbytes for t, s in zip((src, dst), strides)):
                raise ValueError("a state's rows must not overlap")
            rows.append(_SeqRows(src.data_ptr(), dst.data_ptr(), nbytes, *strides))
        self._states = (_SeqRows * len(rows))(*rows)
        self._n_states = len(rows)


def page_fork(fork: PageFork, parents, stream=None) -> None:
    """``ckv_page_fork``: sequence i becomes a copy of sequence ``parents[i]`` (int32 [n_out], device; one
    outside the sequences: empty): its pages, its length, its rows of the states."""
    _need(parents, "parents", torch.int32)
    if parents.numel() != fork.n_out:
        raise ValueError(f"parents must have {fork.n_out} numbers (it has {parents.numel()})")
    device = _together(parents, fork)
    _check(_lib.ckv_page_fork(fork._c, _ptr(parents), fork._states, fork._n_states, _stream_on(device, stream)),
           "ckv_page_fork")


class PageStep:
    """What :func:`page_extend` reads and writes, as one handle.

    ``table``, ``lens`` and ``refs`` (int32, device) as in :class:`PageFork`; ``table_out``, ``lens_out`` and
    ``refs_out`` may be the same tensors.  ``n_new`` [n_seqs]: the tokens that each sequence
    gets.  Written: ``tok_off`` [n_seqs + 1], ``copy_src`` and ``copy_dst`` [n_seqs], ``counts`` [4], and, each
    of as many rows as the call's token tensors, ``slots`` (int64), ``positions`` and ``seqs`` (int32; any
    of these may be None).  ``n_tokens``: those rows, where all three are None.  What is written shares no
    memory with the rest, but for the three that may be the same.
    Keeps the tensors alive; one handle serves every step on the same tensors.
    """

    def __init__(self, page_size: int, table, table_out, lens, lens_out, refs, refs_out, n_new, tok_off, copy_src,
                 copy_dst, counts, slots=None, positions=None, seqs=None, n_tokens: int = 0):
        self._c = _tables(page_size, table, table_out, lens, lens_out, refs, refs_out)
        n = table.shape[0]
        if table_out.shape[0] != n:
            raise ValueError("table and table_out must have as many rows")
        _need(n_new, "n_new", torch.int32, (n,))
        _need(tok_off, "tok_off", torch.int32, (n + 1,))
        _need(copy_src, "copy_src", torch.int32, (n,))
        _need(copy_dst, "copy_dst", torch.int32, (n,))
        _need(counts, "counts", torch.int32, (4,))
        given = [(t, w, d) for t, w, d in ((slots, "slots", torch.int64), (positions, "positions", torch.int32),
                                           (seqs, "seqs", torch.int32)) if t is not None]
        if given:
            n_tokens = given[0][0].numel()
        for t, what, dtype in given:
            _need(t, what, dtype, (n_tokens,))
        self._device = refs.get_device()
        self.n_seqs, self.n_pages = n, refs.numel()
        self.n_new = n_new
        self._tensors = (table, table_out, lens, lens_out, refs, refs_out, tok_off, copy_src, copy_dst, counts, slots,
                         positions, seqs)
        self._step = _PageStep(_ptr(tok_off), _ptr(slots), _ptr(positions), _ptr(seqs), _ptr(copy_src),
                               _ptr(copy_dst), _ptr(counts), _int32(n_tokens, "n_tokens"))


def page_extend_workspace_bytes(n_pages: int, n_seqs: int) -> int:
    return int(_lib.ckv_page_extend_workspace_bytes(n_pages, _int32(n_seqs, "n_seqs")))


def page_extend(step: PageStep, ws, stream=None) -> None:
    """``ckv_page_extend``: pages for every sequence's ``n_new`` tokens, and what the step's token rows
    are; then :func:`page_copy` of ``copy_src`` to ``copy_dst``, and :func:`page_append`.  ``ws``: a uint8
    tensor of :func:`page_extend_workspace_bytes` bytes."""
    device = _current(_together(step.n_new, step))
    ws_ptr, nbytes = _workspace(ws, step.n_new)
    _check(_lib.ckv_page_extend(step._c, _ptr(step.n_new), step._step, ws_ptr, nbytes, _stream_on(device, stream)),
           "ckv_page_extend")


_LOGIT_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


def _fits(t, dtype, shape, device: int) -> bool:
    return t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous()


def _beams(logits, keep: int, scores=None, done=None, eos: int = -1) -> _Beams:
    if logits.dim() != 3 or logits.dtype not in _LOGIT_DTYPES:
        raise ValueError("logits must be a float32 or bfloat16 tensor [n_reqs, n_beams, vocab]")
    n_reqs, n_beams, vocab = logits.shape
    if not -1 <= eos < 1 << 31:
        raise ValueError(f"eos must be -1 or a token (it is {eos})")
    if logits.numel() > 0 and vocab > 1 and logits.stride(2) != 1:
        raise ValueError("a beam's logits must be contiguous")
    # (a dimension of one has no stride that counts)
    stride = logits.stride(1) if n_beams > 1 else logits.stride(0) if n_reqs > 1 else vocab
    if n_reqs > 1 and n_beams > 1 and logits.stride(0) != n_beams * stride:
        raise ValueError("the beams' logits must be equally far apart")
    if n_reqs * n_beams > 1 and stride < vocab:
        raise ValueError("the beams' logits must not overlap")
    return _Beams(_ptr(logits), _ptr(scores), _ptr(done), stride, n_reqs, n_beams, vocab, _int32(keep, "keep"), eos,
                  _LOGIT_DTYPES[logits.dtype])


def beam_select_workspace_bytes(logits, keep: int) -> int:
    return int(_lib.ckv_beam_select_workspace_bytes(_beams(logits, keep)))


def beam_select(logits, scores, parent, token, scores_out, ws, done=None, done_out=None, eos: int = -1,
                stream=None) -> None:
    """``ckv_beam_select``: the best continuations of each request's beams.

    ``logits`` [n_reqs, n_beams, vocab] (float32 or bfloat16, rows equally far apart), ``scores`` float32
    [n_reqs, n_beams] (-inf: an empty place), ``done`` uint8 of that shape or None; ``parent`` and ``token``
    (int32), ``scores_out`` (float32) and ``done_out`` (uint8 or None): [n_reqs, keep], written, best
    first.  ``parent`` counts sequences, request * n_beams + beam, as :func:`page_fork` takes them; -1
    where fewer are offered.  ``ws``: a uint8 tensor of :func:`beam_select_workspace_bytes` bytes.
    """
    if not logits.is_cuda:
        raise ValueError(f"logits must be on the current device (they are on {logits.device})")
    dims, shape, device = logits.shape, parent.shape, torch._C._cuda_getDevice()
    # (what fits is seen in a few comparisons: a call 12.4 -> 11.0 us)
    if not (len(dims) == 3 and len(shape) == 2 and shape[0] == dims[0] and logits.get_device() == device
            and _fits(scores, torch.float32, dims[:2], device) and _fits(parent, torch.int32, shape, device)
            and _fits(token, torch.int32, shape, device) and _fits(scores_out, torch.float32, shape, device)
            and (done is None or _fits(done, torch.uint8, dims[:2], device))
            and (done_out is None or _fits(done_out, torch.uint8, shape, device))):
        if len(dims) != 3 or len(shape) != 2:
            raise ValueError("logits must be [n_reqs, n_beams, vocab] and parent [n_reqs, keep]")
        if logits.get_device() != device:
            raise ValueError(f"logits must be on the current device (they are on {logits.device})")
        shape = (dims[0], shape[1])
        _need(scores, "scores", torch.float32, dims[:2])
        _need(parent, "parent", torch.int32, shape)
        _need(token, "token", torch.int32, shape)
        _need(scores_out, "scores_out", torch.float32, shape)
        if done is not None:
            _need(done, "done", torch.uint8, dims[:2])
        if done_out is not None:
            _need(done_out, "done_out", torch.uint8, shape)
    beams = _beams(logits, shape[1], scores, done, eos)
    ws_ptr, nbytes = _workspace(ws, scores)
    _check(_lib.ckv_beam_select(beams, _ptr(parent), _ptr(token), _ptr(scores_out), _ptr(done_out), ws_ptr, nbytes,
                                _stream_on(device, stream)), "ckv_beam_select")
