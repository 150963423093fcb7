"""ctypes binding of the C ABI in ``include/sp.h``.

Argument marshalling only: every function takes torch tensors (device memory
owned by the caller) and plain integers, passes raw pointers to the library and
turns a non-zero status into :class:`SpError`. Nothing is computed here and
there is no fallback: if ``libsp_amd.so`` is missing the call raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

SP_LAYER_MEAN = 0
SP_LAYER_MAX = 1
SP_CACHE_BF16 = 0
SP_CACHE_E4M3 = 1
SP_CACHE_MX4 = 3
SP_CACHE_BLOCK = 32
SP_MX4_GROUP = 32
SP_ROTATE_HALF = 0
SP_ROTATE_PAIRS = 1
SP_LOGITS_F32 = 0
SP_LOGITS_BF16 = 1
SP_LOGPROBS_MAX_TOP = 32

_STATUS = {1: "SP_ERR_INVALID_ARG", 2: "SP_ERR_UNSUPPORTED", 3: "SP_ERR_WORKSPACE", 4: "SP_ERR_DEVICE"}

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG_DIR, "libsp_amd.so")

EXPORTS = (
    "sp_score_workspace", "sp_score", "sp_score_look", "sp_score_paged", "sp_score_fp8", "sp_score_is_fused", "sp_score_fp8_is_fused", "sp_score_batch", "sp_score_batch_is_fused", "sp_keep_count", "sp_select_workspace",
    "sp_select", "sp_select_static", "sp_select_batch_workspace", "sp_select_batch", "sp_select_budget_workspace", "sp_select_budget", "sp_project", "sp_project_batch",
    "sp_assemble_workspace", "sp_assemble", "sp_last_error", "sp_version",
    "sp_debug_fused_giveup", "sp_debug_score_path", "sp_hbm_read_probe",
    "sp_cache_append", "sp_attend_workspace", "sp_attend", "sp_logprobs_workspace", "sp_logprobs",
    "sp_attend_weights", "sp_cache_evict", "sp_mx4_quantise", "sp_mx4_matmul",
)


class SpError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status
        self.message = message


class ScoreDesc(ctypes.Structure):
    """Mirror of ``sp_score_desc``."""
    _fields_ = [
        ("n_layers", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("n_q", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("layer_agg", ctypes.c_int32),
        ("k_stride_token", ctypes.c_int64),
        ("k_stride_head", ctypes.c_int64),
    ]


class CacheDesc(ctypes.Structure):
    """Mirror of ``sp_cache_desc``."""
    _fields_ = [
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("cache_type", ctypes.c_int32),
        ("n_pages", ctypes.c_int64),
        ("page_tokens", ctypes.c_int64),
        ("page_stride", ctypes.c_int64),
        ("stride_head", ctypes.c_int64),
        ("stride_token", ctypes.c_int64),
    ]


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads ``libsp_amd.so`` (built in-tree by ``paper_2603_02631_amd/build.py``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2603_02631_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(_LIB_PATH)
    c = ctypes
    P = c.c_void_p
    D = c.POINTER(ScoreDesc)
    lib.sp_score_workspace.argtypes = [D, c.c_int64, c.c_int32, c.POINTER(c.c_size_t)]
    lib.sp_score.argtypes = [D, P, c.POINTER(P), c.c_int64, P, P, c.c_size_t, P]
    lib.sp_score_look.argtypes = [D, P, c.POINTER(P), c.c_int64, P, c.c_int32, P, P, c.c_size_t, P]
    lib.sp_score_paged.argtypes = [D, P, c.POINTER(P), P, c.c_int64, c.c_int64, c.c_int64, P, P, c.c_size_t, P]
    lib.sp_score_fp8.argtypes = [D, P, c.POINTER(P), P, c.c_int64, P, P, c.c_size_t, P]
    lib.sp_score_batch.argtypes = [D, P, c.POINTER(P), c.POINTER(c.c_int64), P, c.c_int32, P, P, c.c_size_t, P]
    lib.sp_score_batch_is_fused.argtypes = [D, c.POINTER(c.c_int64), c.c_int32]
    lib.sp_score_batch_is_fused.restype = c.c_int32
    lib.sp_score_is_fused.argtypes = [D, c.c_int64]
    lib.sp_score_is_fused.restype = c.c_int32
    lib.sp_score_fp8_is_fused.argtypes = [D, c.c_int64]
    lib.sp_score_fp8_is_fused.restype = c.c_int32
    lib.sp_keep_count.argtypes = [c.c_int64, c.c_int64, c.c_int64]
    lib.sp_keep_count.restype = c.c_int64
    lib.sp_select_workspace.argtypes = [c.c_int64, c.c_int32, c.POINTER(c.c_size_t)]
    lib.sp_select.argtypes = [P, c.c_int64, c.c_int32, c.c_int32, c.c_int64, P, P, P, P, P, c.c_size_t, P]
    lib.sp_select_static.argtypes = [P, c.c_int64, c.c_int32, c.c_int32, c.c_int64, P, P, P, P, P]
    I64P = c.POINTER(c.c_int64)
    lib.sp_select_batch_workspace.argtypes = [c.c_int64, c.c_int32, c.c_int32, c.POINTER(c.c_size_t)]
    lib.sp_select_batch.argtypes = [P, I64P, P, c.c_int32, c.c_int32, c.c_int32, I64P, P, P, P, P, P, P, c.c_size_t, P]
    lib.sp_project_batch.argtypes = [P, I64P, P, P, I64P, P, c.c_int32, P, P, I64P, P, P, P, P, P, P]
    lib.sp_select_budget_workspace.argtypes = [c.c_int64, c.c_int32, c.POINTER(c.c_size_t)]
    lib.sp_select_budget.argtypes = [P, c.c_int64, c.c_int32, c.c_int32, P, P, c.c_int64, c.c_int64, P, P, P, P, P, P,
                                     P, c.c_size_t, P]
    lib.sp_project.argtypes = [P, c.c_int64, P, c.c_int64, P, P, c.c_int32, P, P, P, P, P]
    lib.sp_assemble_workspace.argtypes = [c.c_int32, c.POINTER(c.c_size_t)]
    lib.sp_assemble.argtypes = [P, c.c_int64, P, P, c.c_int32, P, c.c_int32, c.c_int64, P, P, P, P, P, c.c_size_t, P]
    CD = c.POINTER(CacheDesc)
    lib.sp_cache_append.argtypes = [CD, P, c.c_int64, P, c.c_int64, P, c.c_int64, P, I64P, P, c.c_int32, P, P, P, c.c_int64,
                                    P, P, c.c_int64, c.c_int32, c.c_int32, P, P, P, P, P]
    lib.sp_attend_workspace.argtypes = [CD, I64P, c.c_int32, c.c_int64, c.POINTER(c.c_size_t)]
    lib.sp_attend.argtypes = [CD, P, I64P, P, c.c_int32, P, c.c_int64, P, c.c_int64, P, P, P, P, c.c_float, c.c_int32,
                              c.c_int64, P, P, P, c.c_size_t, P]
    lib.sp_attend_weights.argtypes = [CD, P, I64P, P, c.c_int32, P, c.c_int64, P, c.c_int64, P, P, c.c_float, c.c_int32, c.c_int64,
                                      P, P, P, c.c_int64, P]
    lib.sp_cache_evict.argtypes = [CD, c.c_int32, P, c.c_int64, P, c.c_int64, c.c_int64, c.c_int64, P, c.c_int64, P, c.c_int64,
                                   P, c.c_int64, P, P, P, P, P, P, P, P]
    lib.sp_mx4_quantise.argtypes = [P, c.c_int32, c.c_int64, c.c_int64, c.c_int64, P, P, P]
    lib.sp_mx4_matmul.argtypes = [P, P, c.c_int64, P, P, c.c_int64, c.c_int64, P, c.c_int32, c.c_int64, P]
    lib.sp_logprobs_workspace.argtypes = [c.c_int64, c.c_int64, c.c_int32, c.POINTER(c.c_size_t)]
    lib.sp_logprobs.argtypes = [P, c.c_int32, c.c_int64, c.c_int64, c.c_int64, P, c.c_int32, P, P, P, P, P, c.c_size_t, P]
    lib.sp_hbm_read_probe.argtypes = [P, c.c_size_t, P, P]
    lib.sp_hbm_read_probe.restype = c.c_int
    lib.sp_debug_fused_giveup.argtypes = [c.c_uint32, c.c_int32]
    lib.sp_debug_fused_giveup.restype = None
    lib.sp_debug_score_path.argtypes = []
    lib.sp_debug_score_path.restype = c.c_int32
    lib.sp_last_error.restype = c.c_char_p
    lib.sp_version.restype = c.c_char_p
    for name in ("sp_score_workspace", "sp_score", "sp_score_look", "sp_score_paged", "sp_score_fp8", "sp_score_is_fused", "sp_score_batch", "sp_select_workspace", "sp_select",
                 "sp_select_static", "sp_select_batch_workspace", "sp_select_batch", "sp_select_budget_workspace", "sp_select_budget", "sp_project",
                 "sp_project_batch", "sp_assemble_workspace", "sp_assemble", "sp_cache_append", "sp_attend_workspace", "sp_attend",
                 "sp_logprobs_workspace", "sp_logprobs"):
        getattr(lib, name).restype = c.c_int
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != 0:
        raise SpError(status, sp_last_error())


def _ptr(t, what: str = "buffer", nbytes: int = 0) -> Optional[int]:
    """Device address of a tensor; None passes NULL, an int is taken as a raw address.

    A tensor is checked before its address leaves Python: it has to live on the GPU, be contiguous
    and hold at least ``nbytes`` bytes (what the call will read or write), so that a short or
    host-side buffer becomes an :class:`SpError` instead of an out-of-bounds device access."""
    # a good tensor takes four attribute reads: a call of a dozen pointers costs more here than in its launches
    try:
        if t.is_cuda and t.is_contiguous() and t.nbytes >= nbytes:
            return t.data_ptr()
    except AttributeError:
        pass
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not getattr(t, "is_cuda", False):
        raise SpError(1, f"{what} is not a device tensor")
    if not t.is_contiguous():
        raise SpError(1, f"{what} is not contiguous")
    have = t.numel() * t.element_size()
    if have < nbytes:
        raise SpError(1, f"{what} holds {have} bytes, the call needs {nbytes}")
    return t.data_ptr()


def _q_bytes(desc: "ScoreDesc", n_prompts: int = 1) -> int:
    return n_prompts * desc.n_layers * desc.n_q_heads * desc.n_q * desc.head_dim * 2


def _k_bytes(desc: "ScoreDesc", tokens: int) -> int:
    """Bytes a layer's K buffer must hold for `tokens` tokens under the desc's strides."""
    if tokens <= 0:
        return 0
    return ((desc.n_kv_heads - 1) * desc.k_stride_head + (tokens - 1) * desc.k_stride_token + desc.head_dim) * 2


_current_stream = None      # () -> handle of torch's current stream, resolved at the first use


def _resolve_current_stream():
    import torch
    torch.cuda.init()
    try:        # 1.5 us a call less than through a Stream object; not public, so a torch without them takes the other
        raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        raw(device())
    except (AttributeError, TypeError):
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(stream) -> Optional[int]:
    global _current_stream
    if stream is None:
        if _current_stream is None:
            _current_stream = _resolve_current_stream()
        return _current_stream() or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def sp_last_error() -> str:
    return load_library().sp_last_error().decode()


def sp_version() -> str:
    return load_library().sp_version().decode()


def sp_debug_fused_giveup(spin_limit: int = 1 << 20, force_miss: int = 0) -> None:
    """Test hook: see ``sp_debug_fused_giveup`` in ``include/sp.h``."""
    load_library().sp_debug_fused_giveup(int(spin_limit), int(force_miss))


def sp_debug_score_path() -> int:
    """Test hook: see ``sp_debug_score_path`` in ``include/sp.h``."""
    return int(load_library().sp_debug_score_path())


def sp_hbm_read_probe(buf, nbytes: int, sink, stream=None) -> None:
    _check(load_library().sp_hbm_read_probe(_ptr(buf, "buf", nbytes), nbytes, _ptr(sink, "sink", 8), _stream(stream)))


def sp_keep_count(n_chunks: int, keep_num: int, keep_den: int) -> int:
    return int(load_library().sp_keep_count(n_chunks, keep_num, keep_den))


def sp_score_workspace(desc: ScoreDesc, total_tokens: int, n_prompts: int = 1) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().sp_score_workspace(ctypes.byref(desc), total_tokens, n_prompts, ctypes.byref(n)))
    return int(n.value)


def sp_score_is_fused(desc: ScoreDesc, L: int) -> int:
    return int(load_library().sp_score_is_fused(ctypes.byref(desc), L))


def sp_score_fp8_is_fused(desc: ScoreDesc, L: int) -> int:
    return int(load_library().sp_score_fp8_is_fused(ctypes.byref(desc), L))


def sp_score_batch_is_fused(desc: ScoreDesc, offsets_host: Sequence[int]) -> int:
    B = len(offsets_host) - 1
    off = (ctypes.c_int64 * (B + 1))(*[int(v) for v in offsets_host])
    return int(load_library().sp_score_batch_is_fused(ctypes.byref(desc), off, B))


def _layer_array(k_layers: Sequence, nbytes: int = 0):
    return (ctypes.c_void_p * len(k_layers))(*[_ptr(k, f"k_layers[{i}]", nbytes) for i, k in enumerate(k_layers)])


def _ws_bytes(ws, ws_bytes: Optional[int]) -> int:
    have = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    if ws_bytes is None:
        return have
    if not isinstance(ws, int) and ws is not None and ws_bytes > have:
        raise SpError(3, f"ws_bytes = {ws_bytes} exceeds the workspace tensor ({have} bytes)")
    return ws_bytes


def sp_score(desc: ScoreDesc, q, k_layers: Sequence, L: int, scores, ws, ws_bytes: Optional[int] = None,
             stream=None) -> None:
    if len(k_layers) != desc.n_layers:
        raise SpError(1, f"k_layers has {len(k_layers)} entries, desc.n_layers is {desc.n_layers}")
    nbytes = _ws_bytes(ws, ws_bytes)
    _check(load_library().sp_score(ctypes.byref(desc), _ptr(q, "q", _q_bytes(desc)),
                                   _layer_array(k_layers, _k_bytes(desc, L)), L, _ptr(scores, "scores", 4 * max(L, 0)),
                                   _ptr(ws, "ws"), nbytes, _stream(stream)))


def sp_score_look(desc: ScoreDesc, q, k_layers: Sequence, L: int, k_look, look_self: int, scores, ws,
                  ws_bytes: Optional[int] = None, stream=None) -> None:
    if len(k_layers) != desc.n_layers:
        raise SpError(1, f"k_layers has {len(k_layers)} entries, desc.n_layers is {desc.n_layers}")
    nbytes = _ws_bytes(ws, ws_bytes)
    look_bytes = desc.n_layers * desc.n_kv_heads * desc.n_q * desc.head_dim * 2
    _check(load_library().sp_score_look(ctypes.byref(desc), _ptr(q, "q", _q_bytes(desc)),
                                        _layer_array(k_layers, _k_bytes(desc, L)), L, _ptr(k_look, "k_look", look_bytes),
                                        int(look_self), _ptr(scores, "scores", 4 * max(L, 0)), _ptr(ws, "ws"), nbytes,
                                        _stream(stream)))


def sp_score_paged(desc: ScoreDesc, q, k_pools: Sequence, block_table, page_tokens: int, page_stride: int, L: int,
                   scores, ws, ws_bytes: Optional[int] = None, stream=None) -> None:
    if len(k_pools) != desc.n_layers:
        raise SpError(1, f"k_pools has {len(k_pools)} entries, desc.n_layers is {desc.n_layers}")
    nbytes = _ws_bytes(ws, ws_bytes)
    n_pages = (max(L, 0) + page_tokens - 1) // page_tokens if page_tokens > 0 else 0
    _check(load_library().sp_score_paged(ctypes.byref(desc), _ptr(q, "q", _q_bytes(desc)), _layer_array(k_pools),
                                         _ptr(block_table, "block_table", 4 * n_pages), int(page_tokens),
                                         int(page_stride), L, _ptr(scores, "scores", 4 * max(L, 0)), _ptr(ws, "ws"),
                                         nbytes, _stream(stream)))


def sp_score_fp8(desc: ScoreDesc, q, k8_layers: Sequence, kscale, L: int, scores, ws, ws_bytes: Optional[int] = None,
                 stream=None) -> None:
    if len(k8_layers) != desc.n_layers:
        raise SpError(1, f"k8_layers has {len(k8_layers)} entries, desc.n_layers is {desc.n_layers}")
    nbytes = _ws_bytes(ws, ws_bytes)
    _check(load_library().sp_score_fp8(ctypes.byref(desc), _ptr(q, "q", _q_bytes(desc)),
                                       _layer_array(k8_layers, _k_bytes(desc, L) // 2),
                                       _ptr(kscale, "kscale", 4 * desc.n_layers * desc.n_kv_heads), L,
                                       _ptr(scores, "scores", 4 * max(L, 0)), _ptr(ws, "ws"), nbytes, _stream(stream)))


def sp_score_batch(desc: ScoreDesc, q, k_layers: Sequence, offsets_host: Sequence[int], offsets_dev, scores, ws,
                   ws_bytes: Optional[int] = None, stream=None) -> None:
    if len(k_layers) != desc.n_layers:
        raise SpError(1, f"k_layers has {len(k_layers)} entries, desc.n_layers is {desc.n_layers}")
    B = len(offsets_host) - 1
    off = (ctypes.c_int64 * (B + 1))(*[int(v) for v in offsets_host])
    nbytes = _ws_bytes(ws, ws_bytes)
    total = int(offsets_host[-1]) if B >= 0 else 0
    _check(load_library().sp_score_batch(ctypes.byref(desc), _ptr(q, "q", _q_bytes(desc, max(B, 0))),
                                         _layer_array(k_layers, _k_bytes(desc, total)), off,
                                         _ptr(offsets_dev, "offsets_dev", 8 * (B + 1)), B,
                                         _ptr(scores, "scores", 4 * max(total, 0)), _ptr(ws, "ws"), nbytes,
                                         _stream(stream)))


def sp_select_workspace(L: int, chunk: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().sp_select_workspace(L, chunk, ctypes.byref(n)))
    return int(n.value)


def sp_select(scores, L: int, pool_w: int, chunk: int, k: int, sel_chunks, spans, n_spans, chunk_scores, ws,
              ws_bytes: Optional[int] = None, stream=None) -> None:
    nbytes = _ws_bytes(ws, ws_bytes)
    C = (L + chunk - 1) // chunk if chunk > 0 and L > 0 else 0
    kk = max(int(k), 0)
    _check(load_library().sp_select(_ptr(scores, "scores", 4 * max(L, 0)), L, pool_w, chunk, k,
                                    _ptr(sel_chunks, "sel_chunks", 4 * kk), _ptr(spans, "spans", 16 * kk),
                                    _ptr(n_spans, "n_spans", 4), _ptr(chunk_scores, "chunk_scores", 4 * C),
                                    _ptr(ws, "ws"), nbytes, _stream(stream)))


def sp_select_static(scores, L: int, pool_w: int, chunk: int, k: int, sel_chunks, spans, n_spans, chunk_scores,
                     stream=None) -> None:
    C = (L + chunk - 1) // chunk if chunk > 0 and L > 0 else 0
    kk = max(int(k), 0)
    _check(load_library().sp_select_static(_ptr(scores, "scores", 4 * max(L, 0)), L, pool_w, chunk, k,
                                           _ptr(sel_chunks, "sel_chunks", 4 * kk), _ptr(spans, "spans", 16 * kk),
                                           _ptr(n_spans, "n_spans", 4), _ptr(chunk_scores, "chunk_scores", 4 * C),
                                           _stream(stream)))


def _host_i64(values: Sequence[int]):
    return (ctypes.c_int64 * len(values))(*[int(v) for v in values])


def sp_select_batch_workspace(total_tokens: int, B: int, chunk: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().sp_select_batch_workspace(total_tokens, B, chunk, ctypes.byref(n)))
    return int(n.value)


def sp_select_batch(scores, offsets_host: Sequence[int], offsets_dev, pool_w: int, chunk: int,
                    kept_off_host: Sequence[int], kept_off_dev, sel_chunks, spans, n_spans, chunk_scores, ws,
                    ws_bytes: Optional[int] = None, stream=None) -> None:
    B = len(offsets_host) - 1
    if len(kept_off_host) != B + 1:
        raise SpError(1, f"kept_off_host has {len(kept_off_host)} entries, offsets_host {B + 1}")
    total, kept = max(int(offsets_host[-1]), 0), max(int(kept_off_host[-1]), 0)
    n_cs = total // chunk + B + 1 if chunk > 0 else 0
    _check(load_library().sp_select_batch(
        _ptr(scores, "scores", 4 * total), _host_i64(offsets_host), _ptr(offsets_dev, "offsets_dev", 8 * (B + 1)), B,
        pool_w, chunk, _host_i64(kept_off_host), _ptr(kept_off_dev, "kept_off_dev", 8 * (B + 1)),
        _ptr(sel_chunks, "sel_chunks", 4 * kept), _ptr(spans, "spans", 16 * kept), _ptr(n_spans, "n_spans", 4 * B),
        _ptr(chunk_scores, "chunk_scores", 4 * n_cs), _ptr(ws, "ws"), _ws_bytes(ws, ws_bytes), _stream(stream)))


def sp_project_batch(draft_off, offsets_host: Sequence[int], offsets_dev, target_off, moffsets_host: Sequence[int],
                     moffsets_dev, spans, n_spans, kept_off_host: Sequence[int], kept_off_dev, tspans, n_tspans,
                     keep_mask, n_kept, stream=None) -> None:
    B = len(offsets_host) - 1
    if len(moffsets_host) != B + 1 or len(kept_off_host) != B + 1:
        raise SpError(1, "offsets_host, moffsets_host and kept_off_host must have the same length")
    total, m_total, kept = max(int(offsets_host[-1]), 0), max(int(moffsets_host[-1]), 0), max(int(kept_off_host[-1]), 0)
    _check(load_library().sp_project_batch(
        _ptr(draft_off, "draft_off", 8 * (total + B)), _host_i64(offsets_host),
        _ptr(offsets_dev, "offsets_dev", 8 * (B + 1)), _ptr(target_off, "target_off", 8 * (m_total + B)),
        _host_i64(moffsets_host), _ptr(moffsets_dev, "moffsets_dev", 8 * (B + 1)), B, _ptr(spans, "spans", 16 * kept),
        _ptr(n_spans, "n_spans", 4 * B), _host_i64(kept_off_host), _ptr(kept_off_dev, "kept_off_dev", 8 * (B + 1)),
        _ptr(tspans, "tspans", 16 * kept), _ptr(n_tspans, "n_tspans", 4 * B), _ptr(keep_mask, "keep_mask", m_total),
        _ptr(n_kept, "n_kept", 8 * B), _stream(stream)))


def sp_select_budget_workspace(L: int, chunk: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().sp_select_budget_workspace(L, chunk, ctypes.byref(n)))
    return int(n.value)


def sp_select_budget(scores, L: int, pool_w: int, chunk: int, draft_off, target_off, M: int, budget: int, sel_chunks,
                     spans, n_spans, k_out, n_kept, chunk_scores, ws, ws_bytes: Optional[int] = None,
                     stream=None) -> None:
    nbytes = _ws_bytes(ws, ws_bytes)
    C = (L + chunk - 1) // chunk if chunk > 0 and L > 0 else 0
    _check(load_library().sp_select_budget(_ptr(scores, "scores", 4 * max(L, 0)), L, pool_w, chunk,
                                           _ptr(draft_off, "draft_off", 8 * (max(L, 0) + 1)),
                                           _ptr(target_off, "target_off", 8 * (max(M, 0) + 1)), M, budget,
                                           _ptr(sel_chunks, "sel_chunks", 4 * C), _ptr(spans, "spans", 16 * C),
                                           _ptr(n_spans, "n_spans", 4), _ptr(k_out, "k_out", 8), _ptr(n_kept, "n_kept", 8),
                                           _ptr(chunk_scores, "chunk_scores", 4 * C), _ptr(ws, "ws"), nbytes,
                                           _stream(stream)))


def sp_project(draft_off, L: int, target_off, M: int, spans, n_spans, max_spans: int, tspans, n_tspans, keep_mask,
               n_kept, stream=None) -> None:
    cap = max(int(max_spans), 0)
    _check(load_library().sp_project(_ptr(draft_off, "draft_off", 8 * (max(L, 0) + 1)), L,
                                     _ptr(target_off, "target_off", 8 * (max(M, 0) + 1)), M,
                                     _ptr(spans, "spans", 16 * cap), _ptr(n_spans, "n_spans", 4), max_spans,
                                     _ptr(tspans, "tspans", 16 * cap), _ptr(n_tspans, "n_tspans", 4),
                                     _ptr(keep_mask, "keep_mask", max(M, 0)), _ptr(n_kept, "n_kept", 8), _stream(stream)))


def sp_assemble_workspace(max_spans: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().sp_assemble_workspace(max_spans, ctypes.byref(n)))
    return int(n.value)


def sp_assemble(target_ids, M: int, tspans, n_tspans, max_spans: int, delim_ids, n_delim: int, out_capacity: int,
                out_ids, out_pos, out_src, out_len, ws, ws_bytes: Optional[int] = None, stream=None) -> None:
    nbytes = _ws_bytes(ws, ws_bytes)
    cap = max(int(max_spans), 0)
    oc = max(int(out_capacity), 0)
    _check(load_library().sp_assemble(_ptr(target_ids, "target_ids", 4 * max(M, 0)), M, _ptr(tspans, "tspans", 16 * cap),
                                      _ptr(n_tspans, "n_tspans", 4), max_spans,
                                      _ptr(delim_ids, "delim_ids", 4 * max(int(n_delim), 0)), n_delim, out_capacity,
                                      _ptr(out_ids, "out_ids", 4 * oc), _ptr(out_pos, "out_pos", 4 * oc),
                                      _ptr(out_src, "out_src", 8 * oc), _ptr(out_len, "out_len", 8), _ptr(ws, "ws"),
                                      nbytes, _stream(stream)))


# ---- the draft model's forward pass: paged cache, attention over it, log probabilities ----

def host_offsets(values: Sequence[int]):
    """Offsets as the array that the library reads: made once, it saves the conversion of a list in every call."""
    return _host_i64(values)


def _offsets(values):
    return values if getattr(values, "_type_", None) is ctypes.c_int64 else _host_i64(values)


# Types that an argument may have: its own, and the integers of its width (its bits). Filled at the first tensor (torch is not imported before).
_INT32, _INT64, _FP32, _BF16, _E4M3, _BYTES = set(), set(), set(), set(), set(), set()


def _learn_types() -> None:
    import torch
    for known, names in ((_INT32, ("int32", "uint32")), (_INT64, ("int64", "uint64")), (_FP32, ("float32", "int32", "uint32")),
                         (_BF16, ("bfloat16", "int16", "uint16")), (_E4M3, ("float8_e4m3fn", "uint8", "int8")),
                         (_BYTES, ("uint8", "int8", "float4_e2m1fn_x2", "float8_e8m0fnu"))):
        known.update(getattr(torch, name) for name in names if hasattr(torch, name))


def _check_type(t, what: str, known: set, plain_bytes: bool) -> None:
    if not known:
        _learn_types()
    if t.dtype not in known and not (plain_bytes and str(t.dtype) == "torch.uint8"):
        raise SpError(1, f"{what} is of {t.dtype}, the call needs {' or '.join(sorted(str(x) for x in known))}")


def _typed(t, what: str, nbytes: int, known: set) -> Optional[int]:
    """As _ptr, for arguments whose elements could be misread: a tensor's type has to be one of `known`, or bytes."""
    if t is None:           # before anything raises: an exception takes longer than a tensor's checks
        return None
    try:
        if t.dtype in known and t.is_cuda and t.is_contiguous() and t.nbytes >= nbytes:
            return t.data_ptr()
    except AttributeError:
        pass
    p = _ptr(t, what, nbytes)
    if hasattr(t, "dtype"):
        _check_type(t, what, known, True)
    return p


def _rows(t, what: str, rows: int, width: int, stride: Optional[int], known: set):
    """(address, row stride in elements) of `rows` rows of `width` contiguous elements: a tensor of a type in `known` whose
    first dimension counts rows and whose others are dense, or an address with its stride."""
    if t is None:
        return None, 0
    # two dimensions, the second dense: what a projection's output and its parts are. Few attribute reads, as in _ptr
    try:
        st = t.stride()
        if t.is_cuda and len(st) == 2 and st[1] == 1 and stride is None and t.dtype in known:
            n, w = t.shape
            if n >= rows and w >= width:
                return t.data_ptr(), st[0] if rows > 1 else (width + 7) & ~7      # the stride of a single row means nothing
    except AttributeError:
        pass
    if isinstance(t, int):
        return t, width if stride is None else stride
    if not getattr(t, "is_cuda", False):
        raise SpError(1, f"{what} is not a device tensor")
    _check_type(t, what, known, False)
    shape, strides = t.shape, t.stride()
    if not shape or shape[0] < rows:
        raise SpError(1, f"{what} is {tuple(shape)}, the call needs {rows} rows")
    dense = 1
    for n, s in zip(reversed(shape[1:]), reversed(strides[1:])):
        if n != 1 and s != dense:
            raise SpError(1, f"{what} is not dense within a row")
        dense *= n
    if dense < width:
        raise SpError(1, f"{what} has {dense} elements a row, the call needs {width}")
    if stride is not None and stride != strides[0] and rows > 1:
        raise SpError(1, f"{what} has a row stride of {strides[0]}, the call says {stride}")
    return t.data_ptr(), (strides[0] if rows > 1 else (width + 7) & ~7)


def _rows_or_none(t, what: str, rows: int, width: int, stride: Optional[int], known: set):
    """As _rows; without rows the stride is the given one, or a dense row's. A stride of 0 stays one, which the library refuses."""
    if t is None:
        return None, width if stride is None else stride
    return _rows(t, what, rows, width, stride, known)


def _table(block_table, B: int, table_stride: Optional[int], what: str = "block_table"):
    """(address, entries of a request) of a dense [B][table_stride] int32 block table."""
    if isinstance(block_table, int) or block_table is None:
        return block_table, 0 if table_stride is None else table_stride
    if table_stride is None:
        if block_table.dim() != 2:
            raise SpError(1, f"{what} has to be [requests][entries]")
        table_stride = block_table.shape[1]
    return _typed(block_table, what, 4 * B * table_stride, _INT32), table_stride


_desc_fields = struct.Struct("4i5q").unpack_from        # all fields at once: half of what reading them one by one takes


def _cache_bytes(desc: CacheDesc):
    """Query heads, kv heads, head_dim, a pool's element types and those of its scales, and the bytes that a pool and its scales have to hold."""
    H, kv, d, kind, pages, page, page_stride, stride_head, stride_token = _desc_fields(desc)
    pool = (pages - 1) * page_stride + (kv - 1) * stride_head + (page - 1) * stride_token + d
    if kind == SP_CACHE_MX4:
        return H, kv, d, _BYTES, _BYTES, pool // 2, pages * kv * page * (d // SP_MX4_GROUP)
    scales = 4 * pages * kv * (page // SP_CACHE_BLOCK)
    return (H, kv, d, _E4M3, _FP32, pool, scales) if kind == SP_CACHE_E4M3 else (H, kv, d, _BF16, _FP32, 2 * pool, scales)


def _workspace(ws, ws_bytes: Optional[int]):
    """(address, bytes) of a workspace."""
    try:
        if ws_bytes is None and ws.is_cuda and ws.is_contiguous():
            return ws.data_ptr(), ws.nbytes
    except AttributeError:
        pass
    return _ptr(ws, "ws"), _ws_bytes(ws, ws_bytes)


def sp_cache_append(desc: CacheDesc, k, v, offsets_host, offsets_dev, start, block_table, k_pool, v_pool, k_scale=None,
                    v_scale=None, q=None, q_out=None, cos=None, sin=None, n_pos: Optional[int] = None, rot_dim: int = 0,
                    rot_style: int = SP_ROTATE_HALF, positions=None, k_stride: Optional[int] = None,
                    v_stride: Optional[int] = None, q_stride: Optional[int] = None, table_stride: Optional[int] = None,
                    stream=None) -> None:
    off = _offsets(offsets_host)
    B = len(off) - 1
    T = off[B] if B >= 0 and off[B] > 0 else 0
    H, kv, d, elems, of_scales, pool, scales = _cache_bytes(desc)
    kw, qw = kv * d, H * d
    kp, ks = _rows(k, "k", T, kw, k_stride, _BF16)
    vp, vs = _rows(v, "v", T, kw, v_stride, _BF16)
    qp, qs = _rows(q, "q", T, qw, q_stride, _BF16)
    tab, width = _table(block_table, B, table_stride)
    if n_pos is None:
        n_pos = 0 if cos is None or isinstance(cos, int) else cos.shape[0]
    trig = 2 * n_pos * rot_dim
    status = (_lib or load_library()).sp_cache_append(
        ctypes.byref(desc), kp, ks, vp, vs, qp, qs, _typed(q_out, "q_out", 2 * T * qw, _BF16), off,
        _typed(offsets_dev, "offsets_dev", 8 * (B + 1), _INT64), B, _typed(start, "start", 4 * B, _INT32),
        _typed(positions, "positions", 4 * T, _INT32), tab, width, _typed(cos, "cos", trig, _FP32), _typed(sin, "sin", trig, _FP32), n_pos, rot_dim, rot_style,
        _typed(k_pool, "k_pool", pool, elems), _typed(v_pool, "v_pool", pool, elems), _typed(k_scale, "k_scale", scales, of_scales),
        _typed(v_scale, "v_scale", scales, of_scales), _stream(stream))
    if status:
        _check(status)


def sp_attend_workspace(desc: CacheDesc, offsets_host, B: Optional[int] = None, max_len: int = 0) -> int:
    off = _offsets(offsets_host)
    n = ctypes.c_size_t(0)
    if B is None:
        B = len(off) - 1
    if B >= len(off):
        raise SpError(1, f"offsets_host has {len(off)} entries, {B} requests need {B + 1}")
    _check(load_library().sp_attend_workspace(ctypes.byref(desc), off, B, max_len, ctypes.byref(n)))
    return int(n.value)


def sp_attend(desc: CacheDesc, q, offsets_host, offsets_dev, lens, max_len: int, block_table, k_pool, v_pool, k_scale,
              v_scale, scale: float, out, lse, ws, causal: int = 1, window: int = 0, table_stride: Optional[int] = None,
              ws_bytes: Optional[int] = None, stream=None) -> None:
    off = _offsets(offsets_host)
    B = len(off) - 1
    T = off[B] if B >= 0 and off[B] > 0 else 0
    tab, width = _table(block_table, B, table_stride)
    H, _, d, elems, of_scales, pool, scales = _cache_bytes(desc)
    rows = T * H
    ws_at, ws_size = _workspace(ws, ws_bytes)
    status = (_lib or load_library()).sp_attend(
        ctypes.byref(desc), _typed(q, "q", 2 * rows * d, _BF16), off, _typed(offsets_dev, "offsets_dev", 8 * (B + 1), _INT64), B,
        _typed(lens, "lens", 4 * B, _INT32), max_len, tab, width, _typed(k_pool, "k_pool", pool, elems), _typed(v_pool, "v_pool", pool, elems),
        _typed(k_scale, "k_scale", scales, of_scales),
        _typed(v_scale, "v_scale", scales, of_scales), scale, causal, window,
        _typed(out, "out", 2 * rows * d, _BF16), _typed(lse, "lse", 4 * rows, _FP32), ws_at, ws_size,
        _stream(stream))
    if status:
        _check(status)


def sp_logprobs_workspace(n_rows: int, vocab: int, n_top: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().sp_logprobs_workspace(n_rows, vocab, n_top, ctypes.byref(n)))
    return int(n.value)


def sp_logprobs(logits, n_rows: int, vocab: int, targets, n_top: int, logprob, entropy, top_ids, top_logprobs, ws,
                dtype: Optional[int] = None, row_stride: Optional[int] = None, ws_bytes: Optional[int] = None,
                stream=None) -> None:
    if dtype is None:       # from the tensor
        if not hasattr(logits, "dtype"):
            raise SpError(1, "logits given as an address need a dtype")
        if not _BF16:
            _learn_types()
        dtype = SP_LOGITS_BF16 if logits.dtype in _BF16 else SP_LOGITS_F32        # which refuses what is neither
    x, stride = _rows_or_none(logits, "logits", n_rows, vocab, row_stride, _FP32 if dtype == SP_LOGITS_F32 else _BF16)
    n, k = max(n_rows, 0), max(n_top, 0)
    ws_at, ws_size = _workspace(ws, ws_bytes)
    status = (_lib or load_library()).sp_logprobs(
        x, dtype, n_rows, vocab, stride, _typed(targets, "targets", 4 * n, _INT32), n_top,
        _typed(logprob, "logprob", 4 * n, _FP32), _typed(entropy, "entropy", 4 * n, _FP32), _typed(top_ids, "top_ids", 4 * n * k, _INT32),
        _typed(top_logprobs, "top_logprobs", 4 * n * k, _FP32), ws_at, ws_size, _stream(stream))
    if status:
        _check(status)


def _line_stride(t, what: str, width: int, stride: Optional[int]) -> int:
    """Entries of a (request, kv head) line of a dense [requests][kv heads][entries] array."""
    if stride is not None:
        return stride
    if not hasattr(t, "shape"):
        return width
    if t.dim() != 3:
        raise SpError(1, f"{what} has to be [requests][kv heads][entries]")
    return t.shape[2]


def sp_attend_weights(desc: CacheDesc, q, offsets_host, offsets_dev, lens, max_len: int, block_table, k_pool, k_scale, scale: float, lse,
                      old, weights, causal: int = 1, window: int = 0, table_stride: Optional[int] = None,
                      weights_stride: Optional[int] = None, stream=None) -> None:
    off = _offsets(offsets_host)
    B = len(off) - 1
    T = off[B] if B >= 0 and off[B] > 0 else 0
    tab, width = _table(block_table, B, table_stride)
    H, kv, d, elems, of_scales, pool, scales = _cache_bytes(desc)
    entries = _line_stride(weights, "weights", max_len, weights_stride)
    if old is not None and entries != _line_stride(old, "old", max_len, weights_stride):
        raise SpError(1, "old and weights differ in shape")
    size = 4 * B * kv * max(entries, 0)
    status = (_lib or load_library()).sp_attend_weights(
        ctypes.byref(desc), _typed(q, "q", 2 * T * H * d, _BF16), off, _typed(offsets_dev, "offsets_dev", 8 * (B + 1), _INT64), B,
        _typed(lens, "lens", 4 * B, _INT32), max_len, tab, width, _typed(k_pool, "k_pool", pool, elems), _typed(k_scale, "k_scale", scales, of_scales),
        scale, causal, window, _typed(lse, "lse", 4 * T * H, _FP32), _typed(old, "old", size, _FP32), _typed(weights, "weights", size, _FP32), entries,
        _stream(stream))
    if status:
        _check(status)


def sp_cache_evict(desc: CacheDesc, lens, max_len: int, budget, max_budget: int, sinks: int, recent: int, weights, block_table, dst_table,
                   k_pool, v_pool, k_scale, v_scale, new_lens, kept, new_weights=None, B: Optional[int] = None,
                   weights_stride: Optional[int] = None, table_stride: Optional[int] = None, dst_stride: Optional[int] = None, stream=None) -> None:
    if B is None:
        if not hasattr(lens, "shape"):
            raise SpError(1, "lens given as an address needs B")
        B = lens.numel()
    n = max(B, 0)
    tab, width = _table(block_table, n, table_stride)
    dst, dst_width = _table(dst_table, n, dst_stride, "dst_table")
    _, kv, _, elems, of_scales, pool, scales = _cache_bytes(desc)
    entries = _line_stride(weights, "weights", max_len, weights_stride)
    held = 4 * n * kv * max(max_budget, 0)
    status = (_lib or load_library()).sp_cache_evict(
        ctypes.byref(desc), B, _typed(lens, "lens", 4 * n, _INT32), max_len, _typed(budget, "budget", 4 * n, _INT32), max_budget, sinks, recent,
        _typed(weights, "weights", 4 * n * kv * max(entries, 0), _FP32), entries, tab, width, dst, dst_width, _typed(k_pool, "k_pool", pool, elems),
        _typed(v_pool, "v_pool", pool, elems), _typed(k_scale, "k_scale", scales, of_scales), _typed(v_scale, "v_scale", scales, of_scales),
        _typed(new_lens, "new_lens", 4 * n, _INT32), _typed(kept, "kept", held, _INT32), _typed(new_weights, "new_weights", held, _FP32), _stream(stream))
    if status:
        _check(status)


def _float_kind(t, what: str, dtype: Optional[int]) -> int:
    """SP_LOGITS_BF16 or SP_LOGITS_F32, from the tensor if it is not given."""
    if dtype is not None:
        return dtype
    if not hasattr(t, "dtype"):
        raise SpError(1, f"{what} given as an address needs a dtype")
    if not _BF16:
        _learn_types()
    return SP_LOGITS_BF16 if t.dtype in _BF16 else SP_LOGITS_F32        # the caller refuses what is neither


def sp_mx4_quantise(x, rows: int, K: int, codes, scales, dtype: Optional[int] = None, row_stride: Optional[int] = None, stream=None) -> None:
    dtype = _float_kind(x, "x", dtype)
    at, stride = _rows_or_none(x, "x", rows, K, row_stride, _FP32 if dtype == SP_LOGITS_F32 else _BF16)
    n, k = max(rows, 0), max(K, 0)
    status = (_lib or load_library()).sp_mx4_quantise(at, dtype, rows, K, stride, _typed(codes, "codes", n * k // 2, _BYTES),
                                                      _typed(scales, "scales", n * (k // SP_MX4_GROUP), _BYTES), _stream(stream))
    if status:
        _check(status)


def sp_mx4_matmul(a_codes, a_scales, M: int, w_codes, w_scales, N: int, K: int, out, dtype: Optional[int] = None,
                  out_stride: Optional[int] = None, stream=None) -> None:
    dtype = _float_kind(out, "out", dtype)
    to, stride = _rows_or_none(out, "out", M, N, out_stride, _FP32 if dtype == SP_LOGITS_F32 else _BF16)
    m, n, k = max(M, 0), max(N, 0), max(K, 0)
    status = (_lib or load_library()).sp_mx4_matmul(
        _typed(a_codes, "a_codes", m * k // 2, _BYTES), _typed(a_scales, "a_scales", m * (k // SP_MX4_GROUP), _BYTES), M,
        _typed(w_codes, "w_codes", n * k // 2, _BYTES), _typed(w_scales, "w_scales", n * (k // SP_MX4_GROUP), _BYTES), N, K, to, dtype,
        stride, _stream(stream))
    if status:
        _check(status)
