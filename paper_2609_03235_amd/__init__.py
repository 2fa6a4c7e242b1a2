"""SGD-KV hot path on AMD Instinct MI355X (gfx950).

Thin ctypes binding over ``libsgdkv.so`` (the C ABI declared in
``include/sgdkv.h``): every step of the path runs in the library's HIP
kernels; this module only converts tensors to pointers, allocates the output
tensors with torch, and passes torch's current stream. If the library is not
built, every call raises -- there is no fallback implementation.

Entry points (same names as the C ABI without the ``sgdkv_`` prefix):
  allocate_budgets, total_from_ratio, reduce_query_head_scores   (host)
  compress_workspace_size, compress_layer                        (device)
  decode_workspace_size, decode_attention                        (device)
  page_update, paged_store, norm_rope_store                      (device)
  paged_attention_workspace_size, paged_attention                (device)
"""
from __future__ import annotations

import ctypes
import math
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsgdkv.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, 1, 2, 3, 4
DTYPE_F32, DTYPE_BF16 = 0, 1
SYMBOLS = ("sgdkv_last_error", "sgdkv_version", "sgdkv_reduce_query_head_scores", "sgdkv_total_from_ratio",
           "sgdkv_allocate_budgets", "sgdkv_allocate_budgets_variant", "sgdkv_segment_offsets",
           "sgdkv_compress_workspace_size",
           "sgdkv_compress_layer", "sgdkv_compress_layer_ex",
           "sgdkv_decode_workspace_size", "sgdkv_decode_attention", "sgdkv_decode_workspace_size_ex",
           "sgdkv_decode_attention_ex", "sgdkv_decode_attention_noalloc", "sgdkv_append_kv", "sgdkv_page_update",
           "sgdkv_paged_store", "sgdkv_norm_rope_store", "sgdkv_paged_attention_workspace_size",
           "sgdkv_paged_attention", "sgdkv_profile_enable",
           "sgdkv_profile_reset", "sgdkv_profile_read")


class SgdkvError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"sgdkv status {status}: {message}")
        self.status = status
        self.message = message


class CompressDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("obs_window", ctypes.c_int32), ("pool_kernel", ctypes.c_int32),
                ("seq_len", ctypes.c_int64), ("b_sink", ctypes.c_int64), ("b_window", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class CompressOpts(ctypes.Structure):
    _fields_ = [("group_agg", ctypes.c_int32), ("reserved", ctypes.c_int32), ("qhead_scores", ctypes.c_void_p),
                ("window_pos", ctypes.c_int64), ("gather_stream", ctypes.c_void_p)]


class DecodeDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("kv_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("scale", ctypes.c_float)]


_lib = None


def load_library():
    """Load libsgdkv.so (after torch, so both share torch's HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() or "
                          "python paper_2609_03235_amd/build.py")
    try:
        import torch  # noqa: F401  -- binds the HIP runtime torch ships before ours resolves it
    except ImportError:
        pass
    lib = ctypes.CDLL(LIB_PATH)
    P, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
    lib.sgdkv_last_error.restype = ctypes.c_char_p
    lib.sgdkv_last_error.argtypes = []
    lib.sgdkv_version.restype = i32
    lib.sgdkv_version.argtypes = []
    sigs = {
        "sgdkv_reduce_query_head_scores": [P, i32, i32, i32, P],
        "sgdkv_total_from_ratio": [f64, i32, i32, i64, i64, i64, i32, P],
        "sgdkv_allocate_budgets": [P, i32, i32, i64, i64, i64, i64, i32, P],
        "sgdkv_allocate_budgets_variant": [P, P, i32, i32, i64, i64, i64, i64, i32, i32, f64, P],
        "sgdkv_segment_offsets": [P, i32, i32, P],
        "sgdkv_compress_workspace_size": [P, P],
        "sgdkv_compress_layer": [P, P, P, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P],
        "sgdkv_compress_layer_ex": [P, P, P, P, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P],
        "sgdkv_decode_workspace_size": [P, P, P],
        "sgdkv_decode_attention": [P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P],
        "sgdkv_decode_workspace_size_ex": [P, P, i64, P],
        "sgdkv_decode_attention_ex": [P, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P],
        "sgdkv_decode_attention_noalloc": [P, P, P, P, P, P, P, P, P, P],
        "sgdkv_append_kv": [P, P, P, P, P, i64, i64, P],
        "sgdkv_page_update": [P, P, P, P, P, P, P, P, P, P, P, P],
        "sgdkv_paged_store": [P, P, P, P, i64, P],
        "sgdkv_norm_rope_store": [P, P, P, P, P, P, P, P, P, P, P, P],
        "sgdkv_paged_attention_workspace_size": [P, P, P],
        "sgdkv_paged_attention": [P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P],
        "sgdkv_profile_enable": [i32],
        "sgdkv_profile_reset": [],
        "sgdkv_profile_read": [i32, P, P, P, P],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = i32
    _lib = lib
    return lib


def _check(status: int):
    if status != OK:
        raise SgdkvError(status, load_library().sgdkv_last_error().decode())


def version() -> int:
    return int(load_library().sgdkv_version())


def _np_ptr(a: np.ndarray):
    return a.ctypes.data_as(ctypes.c_void_p)


# ------------------------------------------------------------------ host
def reduce_query_head_scores(per_qhead, num_kv_heads: int) -> np.ndarray:
    a = np.ascontiguousarray(np.asarray(per_qhead, dtype=np.float64))
    L, Hq = a.shape
    out = np.zeros((L, num_kv_heads), dtype=np.float64)
    _check(load_library().sgdkv_reduce_query_head_scores(_np_ptr(a), L, Hq, num_kv_heads, _np_ptr(out)))
    return out


def total_from_ratio(R: float, L: int, H: int, C: int, b_sink: int, b_window: int, of_middle: int = 0) -> int:
    t = ctypes.c_int64(0)
    _check(load_library().sgdkv_total_from_ratio(float(R), L, H, C, b_sink, b_window, int(of_middle),
                                                 ctypes.byref(t)))
    return int(t.value)


def allocate_budgets(scores, L: int, H: int, C: int, b_sink: int, b_window: int, total: int,
                     mode: int = 0) -> np.ndarray:
    sc = np.ascontiguousarray(np.asarray(scores, dtype=np.float64).reshape(-1))
    if sc.size != L * H:
        raise SgdkvError(ERR_INVALID_ARG, "scores must hold L*H values")
    out = np.zeros(L * H, dtype=np.int64)
    _check(load_library().sgdkv_allocate_budgets(_np_ptr(sc), L, H, C, b_sink, b_window, int(total), int(mode),
                                                 _np_ptr(out)))
    return out


ALLOC_PLAIN, ALLOC_THR, ALLOC_REVERSE, ALLOC_MIX, ALLOC_BINARY, ALLOC_BINARY_REVERSE = range(6)


def allocate_budgets_variant(scores, L: int, H: int, C: int, b_sink: int, b_window: int, total: int,
                             variant: int, mode: int = 0, scores2=None, full_fraction: float = 0.0) -> np.ndarray:
    sc = np.ascontiguousarray(np.asarray(scores, dtype=np.float64).reshape(-1))
    if sc.size != L * H:
        raise SgdkvError(ERR_INVALID_ARG, "scores must hold L*H values")
    s2 = None
    if scores2 is not None:
        s2 = np.ascontiguousarray(np.asarray(scores2, dtype=np.float64).reshape(-1))
        if s2.size != L * H:
            raise SgdkvError(ERR_INVALID_ARG, "scores2 must hold L*H values")
    out = np.zeros(L * H, dtype=np.int64)
    _check(load_library().sgdkv_allocate_budgets_variant(
        _np_ptr(sc), _np_ptr(s2) if s2 is not None else None, L, H, C, b_sink, b_window, int(total), int(mode),
        int(variant), float(full_fraction), _np_ptr(out)))
    return out


def segment_offsets(layer_budgets, batch: int) -> np.ndarray:
    """Host copy of the ragged cache's row offsets [batch * Hkv + 1] for one layer's budgets
    (sgdkv_segment_offsets): the values compress_layer writes to its device offsets."""
    bud = np.ascontiguousarray(np.asarray(layer_budgets, dtype=np.int64).reshape(-1))
    out = np.zeros(int(batch) * bud.size + 1, dtype=np.int64)
    _check(load_library().sgdkv_segment_offsets(_np_ptr(bud), int(batch), bud.size, _np_ptr(out)))
    return out


# ---------------------------------------------------------------- device
def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    if t.dtype == torch.float32:
        return DTYPE_F32
    raise SgdkvError(ERR_INVALID_ARG, f"unsupported dtype {t.dtype}")


def _ptr(t):
    if t is None:
        return None
    if not t.is_contiguous():
        raise SgdkvError(ERR_INVALID_ARG, "tensors must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def compress_desc(q_win, k, *, obs_window=None, pool_kernel: int, b_sink: int, b_window: int,
                  scale: float = 0.0) -> CompressDesc:
    B, Hq, w, d = q_win.shape
    Bk, Hkv, C, dk = k.shape
    if Bk != B or dk != d or (obs_window is not None and obs_window != w):
        raise SgdkvError(ERR_INVALID_ARG, f"shape mismatch q_win {tuple(q_win.shape)} k {tuple(k.shape)}")
    return CompressDesc(B, Hq, Hkv, d, w, pool_kernel, C, b_sink, b_window, _dtype_code(k), float(scale))


def compress_workspace_size(desc: CompressDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().sgdkv_compress_workspace_size(ctypes.byref(desc), ctypes.byref(n)))
    return int(n.value)


def alloc_workspace(nbytes: int, device):
    """Device workspace as a uint8 tensor (torch's allocator returns 256-byte aligned blocks)."""
    import torch
    ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    return ws


GROUP_MEAN, GROUP_IPT_MAX, GROUP_IPT_MEAN, GROUP_IPT_ONLY = range(4)


def compress_layer(q_win, k, v, layer_budgets, *, pool_kernel: int, b_sink: int, b_window: int,
                   scale: float = 0.0, window_lse=None, scores_only: bool = False, with_scores: bool = True,
                   group_agg: int = GROUP_MEAN, qhead_scores=None, window_pos: int = -1,
                   workspace=None, out: dict | None = None, stream=None, gather_stream=None) -> dict:
    """Compress one layer (sgdkv_compress_layer_ex). group_agg selects the plain group mean or an
    Ipt. aggregation with the layer's per-query-head scores; window_pos places the first window
    row (-1: the last obs_window prompt tokens). gather_stream (optional) takes the copy of the
    kept rows into k_c and v_c, which are then complete only on that stream. Returns k_c, v_c,
    kept_pos, offsets, offsets_host, scores (scores: [B, Hkv, window position]). With gather_stream, the
    tensors the copy reads or writes (k, v, k_c, v_c, kept_pos) are marked as in use on that stream (for a
    torch.cuda.Stream; a raw stream handle leaves keeping them alive to the caller), so torch's allocator
    does not hand their memory to other work before the copy is done."""
    import torch
    desc = compress_desc(q_win, k, pool_kernel=pool_kernel, b_sink=b_sink, b_window=b_window, scale=scale)
    B, Hkv, C, d = k.shape
    dev = k.device
    budgets = None if layer_budgets is None else np.ascontiguousarray(np.asarray(layer_budgets, dtype=np.int64))
    if budgets is not None and budgets.size != Hkv:
        raise SgdkvError(ERR_INVALID_ARG, "layer_budgets must hold num_kv_heads values")
    res = dict(out or {})
    if not scores_only:
        T = int(budgets.sum())
        # only what the caller did not bring is allocated (eagerly evaluated defaults cost a 2K layer
        # four allocations, about 8 us of host time, per call)
        for name, shape, dtype in (("k_c", (B * T, d), k.dtype), ("v_c", (B * T, d), None),
                                   ("kept_pos", B * T, torch.int32), ("offsets", B * Hkv + 1, torch.int64)):
            if name not in res:
                res[name] = torch.empty(shape, dtype=v.dtype if dtype is None else dtype, device=dev)
        res["offsets_host"] = segment_offsets(budgets, B)
    n_scored = C - q_win.shape[2] if window_pos == -1 else int(window_pos)
    if (with_scores or scores_only) and "scores" not in res:
        res["scores"] = torch.empty((B, Hkv, max(n_scored, 0)), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = alloc_workspace(compress_workspace_size(desc), dev)
    qs = None
    if qhead_scores is not None:
        qs = np.ascontiguousarray(np.asarray(qhead_scores, dtype=np.float64).reshape(-1))
        if qs.size != q_win.shape[1]:
            raise SgdkvError(ERR_INVALID_ARG, "qhead_scores must hold num_q_heads values")
    opts = CompressOpts(int(group_agg), 0, None if qs is None else qs.ctypes.data, int(window_pos),
                        None if gather_stream is None else _stream(gather_stream).value)
    st = load_library().sgdkv_compress_layer_ex(
        ctypes.byref(desc), ctypes.byref(opts), None if budgets is None else _np_ptr(budgets), _ptr(q_win), _ptr(k),
        _ptr(v) if v is not None else None, _ptr(window_lse), _ptr(res.get("k_c")), _ptr(res.get("v_c")),
        _ptr(res.get("kept_pos")), _ptr(res.get("offsets")), _ptr(res.get("scores")), _ptr(workspace),
        workspace.numel(), _stream(stream))
    _check(st)
    if isinstance(gather_stream, torch.cuda.Stream) and not scores_only:
        for t in (k, v, res["k_c"], res["v_c"], res["kept_pos"]):
            t.record_stream(gather_stream)
    return res


def decode_desc(q, num_kv_heads: int, out_dtype=None, scale: float = 0.0) -> DecodeDesc:
    B, Hq, d = q.shape
    od = _dtype_code(q) if out_dtype is None else (DTYPE_BF16 if "bfloat16" in str(out_dtype) else DTYPE_F32)
    return DecodeDesc(B, Hq, num_kv_heads, d, _dtype_code(q), od, float(scale))


def decode_workspace_size(desc: DecodeDesc, offsets_host, capacity: int = 0) -> int:
    oh = np.ascontiguousarray(np.asarray(offsets_host, dtype=np.int64))
    n = ctypes.c_size_t(0)
    _check(load_library().sgdkv_decode_workspace_size_ex(ctypes.byref(desc), _np_ptr(oh), int(capacity),
                                                          ctypes.byref(n)))
    return int(n.value)


class DecodeTail(ctypes.Structure):
    _fields_ = [("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p), ("capacity", ctypes.c_int64),
                ("n_new", ctypes.c_int64)]


def decode_attention(q, k_c, v_c, offsets, offsets_host, num_kv_heads: int, *, out_dtype=None,
                     scale: float = 0.0, with_lse: bool = True, k_new=None, v_new=None, n_new: int = 0,
                     workspace=None, out=None, lse=None, stream=None, no_alloc: bool = False):
    """One decode step over the ragged cache (sgdkv_decode_attention_ex). k_new/v_new [B, Hkv, capacity, d]
    hold the rows appended since compression, of which the first n_new are attended. no_alloc: call
    sgdkv_decode_attention_noalloc instead, which takes no workspace (its split partials go to the
    library's static device scratch; pass out, and lse if wanted, to allocate nothing here either).
    Returns (out, lse)."""
    import torch
    desc = decode_desc(q, num_kv_heads, out_dtype, scale)
    oh = np.ascontiguousarray(np.asarray(offsets_host, dtype=np.int64))
    B, Hq, d = q.shape
    cap = 0 if k_new is None else int(k_new.shape[2])
    if out is None:
        out = torch.empty((B, Hq, d), dtype=torch.bfloat16 if desc.out_dtype == DTYPE_BF16 else torch.float32,
                          device=q.device)
    if with_lse and lse is None:
        lse = torch.empty((B, Hq), dtype=torch.float32, device=q.device)
    tail = DecodeTail(_ptr(k_new), _ptr(v_new), cap, int(n_new))
    if no_alloc:
        _check(load_library().sgdkv_decode_attention_noalloc(
            ctypes.byref(desc), _ptr(q), _ptr(k_c), _ptr(v_c), _ptr(offsets), _np_ptr(oh), ctypes.byref(tail),
            _ptr(out), _ptr(lse) if with_lse else None, _stream(stream)))
        return out, (lse if with_lse else None)
    if workspace is None:
        workspace = alloc_workspace(decode_workspace_size(desc, oh, cap), q.device)
    st = load_library().sgdkv_decode_attention_ex(
        ctypes.byref(desc), _ptr(q), _ptr(k_c), _ptr(v_c), _ptr(offsets), _np_ptr(oh), ctypes.byref(tail), _ptr(out),
        _ptr(lse) if with_lse else None, _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st)
    return out, (lse if with_lse else None)


def append_kv(q_like, k_step, v_step, k_new, v_new, slot: int, stream=None):
    """Write one generated token's K/V rows [B, Hkv, d] into row `slot` of k_new/v_new [B, Hkv, capacity, d]
    (sgdkv_append_kv). q_like: the decode queries [B, Hq, d] (for the descriptor)."""
    desc = decode_desc(q_like, k_step.shape[1])
    _check(load_library().sgdkv_append_kv(ctypes.byref(desc), _ptr(k_step), _ptr(v_step), _ptr(k_new), _ptr(v_new),
                                          int(k_new.shape[2]), int(slot), _stream(stream)))


# --------------------------------------------------------- paged cache
class PagePool(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("num_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class PageDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("by_segment", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("num_free", ctypes.c_int64), ("num_slots", ctypes.c_int64)]


class NormRopeDesc(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int64), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


class PagedDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("num_tokens", ctypes.c_int64), ("max_new", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_float)]


PAGES_OK, PAGES_SHORT, PAGES_ROWS, PAGES_STACK, PAGES_SLOTS = range(5)


class _on_stream:
    """Makes the tensors' device current and `stream` (None: that device's current stream) torch's current
    stream, so that what a call allocates belongs to the stream it is used on. Enters as the raw handle."""

    def __init__(self, device, stream):
        import torch
        self.guards = [torch.cuda.device(device)]
        if stream is not None:
            if not hasattr(stream, "cuda_stream"):
                stream = torch.cuda.ExternalStream(int(stream), device=device)
            if stream.device != device:
                raise SgdkvError(ERR_INVALID_ARG, f"the stream is on {stream.device}, the tensors on {device}")
            self.guards.append(torch.cuda.stream(stream))

    def __enter__(self):
        import torch
        for g in self.guards:
            g.__enter__()
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def __exit__(self, *exc):
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _need(cond: bool, message: str):
    if not cond:
        raise SgdkvError(ERR_INVALID_ARG, message)


def _need_same(device, **tensors):
    """Every given tensor is on `device` (a GPU)."""
    _need(device.type == "cuda", f"tensors must be on a GPU, not on {device}")
    for name, t in tensors.items():
        _need(t is None or t.device == device, f"{name} is on another device than {device}")


def _need_int32(shape=None, **tensors):
    import torch
    for name, t in tensors.items():
        _need(t.dtype == torch.int32, f"{name} must be int32, not {t.dtype}")
        _need(t.is_contiguous(), f"{name} must be contiguous")
        _need(shape is None or tuple(t.shape) == tuple(shape), f"{name} has shape {tuple(t.shape)}, not {shape}")


def page_pool(k_pages, v_pages) -> PagePool:
    """The descriptor of a pool k_pages, v_pages [num_pages, page_size, d]."""
    _need(k_pages.dim() == 3 and k_pages.shape == v_pages.shape and k_pages.dtype == v_pages.dtype,
          "k_pages and v_pages must be [num_pages, page_size, d] of one dtype")
    _need(k_pages.is_contiguous() and v_pages.is_contiguous(), "k_pages and v_pages must be contiguous")
    n, page, d = k_pages.shape
    return PagePool(k_pages.data_ptr(), v_pages.data_ptr(), n, page, d, _dtype_code(k_pages), 0)


def page_update(rows, add, tables, free_pages, head, *, page_size: int, n_slots: int, by_segment: bool = False,
                rows_out=None, head_out=None, slots=None, cu=None, status=None, stream=None) -> dict:
    """Pages and slots for the rows that segments gain or lose (sgdkv_page_update). rows [B * Hkv], tables
    [B * Hkv, max_pages] (updated in place), free_pages [n] (a stack, updated in place) and head [1] are int32;
    add is int32 [B], or [B * Hkv] with by_segment. Returns slots ([n_slots, Hkv] or [n_slots]), rows, head, cu,
    status and the updated tables and free_pages. rows_out and head_out may be rows and head."""
    import torch
    dev = rows.device
    _need_same(dev, add=add, tables=tables, free_pages=free_pages, head=head, rows_out=rows_out, head_out=head_out,
               slots=slots, cu=cu, status=status)
    _need(rows.dim() == 1 and add.dim() == 1 and tables.dim() == 2 and free_pages.dim() == 1,
          "rows, add and free_pages must have one dimension and tables two")
    S, n_add = rows.numel(), add.numel()
    _need(S > 0 and tables.shape[0] == S, f"tables has {tables.shape[0]} rows for {S} segments")
    _need(n_add == S if by_segment else n_add > 0 and S % n_add == 0, f"add holds {n_add} values for {S} segments")
    B = 1 if by_segment else n_add
    Hkv = S // B
    n_slots = int(n_slots)
    _need(n_slots >= 0, "n_slots must be >= 0")
    _need_int32(rows=rows, add=add, tables=tables, free_pages=free_pages)
    _need_int32((1,), head=head)
    with _on_stream(dev, stream) as s:
        new = lambda *shape: torch.empty(shape, dtype=torch.int32, device=dev)
        rows_out = new(S) if rows_out is None else rows_out
        head_out = new(1) if head_out is None else head_out
        cu = new(n_add + 1) if cu is None else cu
        status = new(1) if status is None else status
        shape = (n_slots,) if by_segment else (n_slots, Hkv)
        slots = new(*shape) if slots is None else slots
        _need_int32((S,), rows_out=rows_out)
        _need_int32((1,), head_out=head_out, status=status)
        _need_int32((n_add + 1,), cu=cu)
        _need_int32(shape, slots=slots)
        desc = PageDesc(B, Hkv, int(page_size), tables.shape[1], int(bool(by_segment)), 0, free_pages.numel(), n_slots)
        _check(load_library().sgdkv_page_update(
            ctypes.byref(desc), _ptr(rows), _ptr(add), _ptr(tables), _ptr(free_pages), _ptr(head), _ptr(rows_out),
            _ptr(head_out), _ptr(cu), _ptr(slots), _ptr(status), s))
    return dict(slots=slots, rows=rows_out, head=head_out, cu=cu, status=status, tables=tables, free_pages=free_pages)


def paged_store(k_rows, v_rows, slots, k_pages, v_pages, *, stream=None):
    """Copy rows [n, d] to their slots (sgdkv_paged_store): slots int32 [n], -1 for none."""
    dev = k_pages.device
    _need_same(dev, v_pages=v_pages, k_rows=k_rows, v_rows=v_rows, slots=slots)
    pool = page_pool(k_pages, v_pages)
    _need(k_rows.dim() == 2 and k_rows.shape == v_rows.shape and k_rows.shape[1] == pool.head_dim
          and k_rows.dtype == v_rows.dtype == k_pages.dtype, "k_rows and v_rows must be [n, d] of the pool's dtype")
    n = k_rows.shape[0]
    _need_int32((n,), slots=slots)
    with _on_stream(dev, stream) as s:
        _check(load_library().sgdkv_paged_store(ctypes.byref(pool), _ptr(k_rows), _ptr(v_rows), _ptr(slots), n, s))


def _token_stride(t, name, heads, d):
    """Elements between tokens of t [T, heads, d], whose heads must be dense."""
    _need(heads == 0 or t.shape[0] == 0 or (t.stride(2) == 1 and (heads == 1 or t.stride(1) == d)),
          f"the heads of a token of {name} must be dense")
    return t.stride(0) if t.shape[0] > 1 else heads * d


def norm_rope_store(q, k, v, positions, slots, k_pages, v_pages, *, inv_freq=None, q_weight=None, k_weight=None,
                    eps: float = 1e-6, interleaved: bool = False, q_out=None, stream=None):
    """New tokens' heads in one pass (sgdkv_norm_rope_store): queries [T, Hq, d] and keys [T, Hkv, d] normalised per
    head (with q_weight, k_weight [d]) and rotated by positions (int32 [T]) with inv_freq (fp32 [rot_dim / 2];
    None: no rotation), keys and values stored to slots (int32 [T, Hkv], -1 for none). q, k and v may be parts of
    one projection's output. q may be None. Returns q_out [T, Hq, d]."""
    import torch
    dev = k_pages.device
    _need_same(dev, v_pages=v_pages, q=q, k=k, v=v, positions=positions, slots=slots, inv_freq=inv_freq,
               q_weight=q_weight, k_weight=k_weight, q_out=q_out)
    pool = page_pool(k_pages, v_pages)
    dt, d = k_pages.dtype, pool.head_dim
    _need(k.dim() == 3 and v.shape == k.shape and k.shape[2] == d and k.dtype == v.dtype == dt,
          "k and v must be [T, Hkv, d] of the pool's dtype")
    T, Hkv = k.shape[:2]
    Hq = 0 if q is None else q.shape[1]
    _need(q is None or (q.dim() == 3 and q.shape[0] == T and q.shape[2] == d and q.dtype == dt),
          "q must be [T, Hq, d] of the pool's dtype")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        _need(w is None or (tuple(w.shape) == (d,) and w.dtype == dt and w.is_contiguous()),
              f"{name} must be [d] of the pool's dtype")
    _need(inv_freq is None or (inv_freq.dim() == 1 and inv_freq.dtype == torch.float32 and inv_freq.is_contiguous()),
          "inv_freq must be fp32 with one dimension")
    _need_int32((T,), positions=positions)
    _need_int32((T, Hkv), slots=slots)
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    with _on_stream(dev, stream) as s:
        if Hq and q_out is None:
            q_out = torch.empty((T, Hq, d), dtype=dt, device=dev)
        _need(not Hq or (tuple(q_out.shape) == (T, Hq, d) and q_out.dtype == dt and q_out.is_contiguous()),
              "q_out must be a dense [T, Hq, d] of the pool's dtype")
        desc = NormRopeDesc(T, Hq, Hkv, 0 if not Hq else _token_stride(q, "q", Hq, d), _token_stride(k, "k", Hkv, d),
                            _token_stride(v, "v", Hkv, d), rot, int(bool(interleaved)), float(eps), 0)
        _check(load_library().sgdkv_norm_rope_store(
            ctypes.byref(pool), ctypes.byref(desc), q.data_ptr() if Hq else None, k.data_ptr(), v.data_ptr(),
            _ptr(positions), _ptr(slots), _ptr(inv_freq), _ptr(q_weight), _ptr(k_weight),
            _ptr(q_out) if Hq else None, s))
    return q_out


def _paged_desc(q, num_kv_heads, batch, max_new, max_pages, out_dtype, causal, scale) -> PagedDesc:
    import torch
    T, Hq, _ = q.shape
    _need(out_dtype in (None, torch.bfloat16, torch.float32), f"out_dtype {out_dtype}")
    od = _dtype_code(q) if out_dtype is None else (DTYPE_BF16 if out_dtype == torch.bfloat16 else DTYPE_F32)
    return PagedDesc(int(batch), Hq, int(num_kv_heads), od, T, int(max_new), int(max_pages), int(bool(causal)),
                     float(scale))


def paged_attention_workspace_size(q, num_kv_heads: int, batch: int, *, max_new: int) -> int:
    """Bytes of workspace of paged_attention for queries like q [T, Hq, d] and chunks of up to max_new tokens."""
    pool = PagePool(None, None, 1, 16, q.shape[2], _dtype_code(q), 0)
    desc = _paged_desc(q, num_kv_heads, batch, max_new, 1, None, True, 0.0)
    n = ctypes.c_size_t(0)
    _check(load_library().sgdkv_paged_attention_workspace_size(ctypes.byref(pool), ctypes.byref(desc),
                                                                ctypes.byref(n)))
    return int(n.value)


def paged_attention(q, k_pages, v_pages, tables, rows, cu_new, num_kv_heads: int, *, max_new: int, causal: bool = True,
                    scale: float = 0.0, out_dtype=None, with_lse: bool = True, out=None, lse=None, workspace=None,
                    stream=None):
    """Attention of the new tokens q [T, Hq, d] over the paged rows of their segments, their own included
    (sgdkv_paged_attention): tables int32 [B * Hkv, max_pages], rows int32 [B * Hkv], cu_new int32 [B + 1], all on
    the GPU; max_new is at least the longest sequence's number of new tokens. Returns (out, lse)."""
    import torch
    dev = q.device
    _need_same(dev, k_pages=k_pages, v_pages=v_pages, tables=tables, rows=rows, cu_new=cu_new, out=out, lse=lse,
               workspace=workspace)
    pool = page_pool(k_pages, v_pages)
    _need(q.dim() == 3 and q.shape[2] == pool.head_dim and q.dtype == k_pages.dtype and q.is_contiguous(),
          "q must be a dense [T, Hq, d] of the pool's dtype")
    _need(tables.dim() == 2 and rows.dim() == 1 and cu_new.dim() == 1 and cu_new.numel() >= 2,
          "tables must be [B * Hkv, max_pages], rows [B * Hkv] and cu_new [B + 1]")
    B, (T, Hq, d) = cu_new.numel() - 1, q.shape
    _need(rows.numel() == tables.shape[0] == B * int(num_kv_heads),
          f"{rows.numel()} rows and {tables.shape[0]} tables for {B} sequences of {num_kv_heads} KV heads")
    _need_int32(tables=tables, rows=rows, cu_new=cu_new)
    desc = _paged_desc(q, num_kv_heads, B, max_new, tables.shape[1], out_dtype, causal, scale)
    with _on_stream(dev, stream) as s:
        od = torch.bfloat16 if desc.out_dtype == DTYPE_BF16 else torch.float32
        if out is None:
            out = torch.empty((T, Hq, d), dtype=od, device=dev)
        if with_lse and lse is None:
            lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
        _need(tuple(out.shape) == (T, Hq, d) and out.dtype == od and out.is_contiguous(),
              f"out must be a dense {(T, Hq, d)} of {od}")
        _need(not with_lse or (tuple(lse.shape) == (T, Hq) and lse.dtype == torch.float32 and lse.is_contiguous()),
              f"lse must be a dense fp32 {(T, Hq)}")
        if workspace is None:
            workspace = alloc_workspace(paged_attention_workspace_size(q, num_kv_heads, B, max_new=max_new), dev)
        _check(load_library().sgdkv_paged_attention(
            ctypes.byref(pool), ctypes.byref(desc), _ptr(q), _ptr(tables), _ptr(rows), _ptr(cu_new), _ptr(out),
            _ptr(lse) if with_lse else None, _ptr(workspace), workspace.numel() * workspace.element_size(), s))
    return out, (lse if with_lse else None)


# ------------------------------------------------------- kernel timing
def profile_enable(on: bool = True):
    _check(load_library().sgdkv_profile_enable(1 if on else 0))


def profile_reset():
    _check(load_library().sgdkv_profile_reset())


def profile_read(max_entries: int = 64) -> dict:
    """{kernel name: (launches, total ms)} since the last reset (waits for pending events)."""
    names = ctypes.create_string_buffer(max_entries * 64)
    counts = np.zeros(max_entries, dtype=np.int64)
    ms = np.zeros(max_entries, dtype=np.float64)
    n = ctypes.c_int32(0)
    _check(load_library().sgdkv_profile_read(max_entries, names, _np_ptr(counts), _np_ptr(ms), ctypes.byref(n)))
    out = {}
    for i in range(min(n.value, max_entries)):
        name = names.raw[i * 64:(i + 1) * 64].split(b"\0", 1)[0].decode()
        out[name] = (int(counts[i]), float(ms[i]))
    return out
