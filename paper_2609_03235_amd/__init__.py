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

A stream is a torch.cuda.Stream or a raw handle; the calls over the paged cache mark their tensors as in use on the
former, and with a raw handle the caller keeps them alive until the call is done.
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


def _raw_stream(index):
    """The raw handle of GPU `index`'s current stream where that GPU is current, else None. The handle alone:
    building a torch.cuda.Stream for it takes 2.8 us, a third of a small call."""
    import torch
    if torch.cuda.current_device() != index:
        return None
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream().cuda_stream if raw is None else raw(index)


def _switched(fn, index, stream, args, kw):
    """fn(*args, **kw) with GPU `index` current and `stream` (None: that GPU's current one) torch's current stream, so
    that what the call allocates belongs to the stream it is used on; the tensors it is given are marked as in use
    there, so that the allocator does not hand their memory to other work before the call is done. For a raw handle
    keeping them alive is the caller's: torch would use the mark, and so the handle, when a tensor is freed, and the
    caller may have destroyed the stream by then."""
    import torch
    with torch.cuda.device(index):
        if stream is None:
            return fn(*args, **kw)
        mark = hasattr(stream, "cuda_stream")
        if not mark:
            # ExternalStream takes a handle of 0 for "none given" and makes a new stream
            stream = (torch.cuda.ExternalStream(int(stream), device=torch.device("cuda", index)) if int(stream)
                      else torch.cuda.default_stream(index))
        if stream.device.index != index:
            _refuse(f"the stream is on {stream.device}, the tensors on cuda:{index}")
        with torch.cuda.stream(stream):
            result = fn(*args, **kw)
        if mark:
            for t in (*args, *kw.values()):
                if isinstance(t, torch.Tensor):
                    t.record_stream(stream)
        return result


def _refuse(message: str):
    raise SgdkvError(ERR_INVALID_ARG, message)


def _gpu_of(first, *others) -> int:
    """The index of the GPU that every given tensor is on."""
    index = first.get_device()
    if index < 0:
        _refuse(f"tensors must be on a GPU, not on {first.device}")
    for t in others:
        if t is not None and t.get_device() != index:
            _refuse(f"a tensor is on {t.device}, the others are on cuda:{index}")
    return index


def _check_int32(t, name, shape=None):
    import torch
    if t.dtype is not torch.int32 or not t.is_contiguous():
        _refuse(f"{name} must be contiguous int32, not {t.dtype}")
    if shape is not None and t.shape != shape:
        _refuse(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")


def _check_dense(t, name, shape, dtype):
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        _refuse(f"{name} must be a dense {tuple(shape)} of {dtype}, not {tuple(t.shape)} of {t.dtype}")


def _overlap(a, b) -> bool:
    """Two contiguous tensors have bytes in common."""
    a0, b0 = a.data_ptr(), b.data_ptr()
    return a0 < b0 + b.numel() * b.element_size() and b0 < a0 + a.numel() * a.element_size()


def page_pool(k_pages, v_pages) -> PagePool:
    """The descriptor of a pool k_pages, v_pages [num_pages, page_size, d]."""
    if k_pages.dim() != 3 or k_pages.shape != v_pages.shape or k_pages.dtype is not v_pages.dtype:
        _refuse("k_pages and v_pages must be [num_pages, page_size, d] of one dtype")
    if not (k_pages.is_contiguous() and v_pages.is_contiguous()):
        _refuse("k_pages and v_pages must be contiguous")
    n, page, d = k_pages.shape
    return PagePool(k_pages.data_ptr(), v_pages.data_ptr(), n, page, d, _dtype_code(k_pages), 0)


def page_update(rows, add, tables, free_pages, head, *, page_size: int, n_slots: int, by_segment: bool = False,
                rows_out=None, head_out=None, slots=None, cu=None, status=None, stream=None) -> dict:
    """Pages and slots for the rows that segments gain or lose (sgdkv_page_update). rows [B * Hkv], tables
    [B * Hkv, max_pages] (updated in place), free_pages [n] (a stack, updated in place) and head [1] are int32;
    add is int32 [B], or [B * Hkv] with by_segment. Returns slots ([n_slots, Hkv] or [n_slots]), rows, head, cu,
    status and the updated tables and free_pages. rows_out may be rows and head_out head; no other two arguments that
    share memory. Results that the caller does not bring share one allocation."""
    import torch
    index = _gpu_of(rows, add, tables, free_pages, head, rows_out, head_out, slots, cu, status)
    if rows.dim() != 1 or add.dim() != 1 or tables.dim() != 2 or free_pages.dim() != 1:
        _refuse("rows, add and free_pages must have one dimension and tables two")
    S, n_add, n_slots = rows.shape[0], add.shape[0], int(n_slots)
    if S == 0 or tables.shape[0] != S:
        _refuse(f"tables has {tables.shape[0]} rows for {S} segments")
    if n_add != S if by_segment else n_add == 0 or S % n_add:
        _refuse(f"add holds {n_add} values for {S} segments")
    if n_slots < 0:
        _refuse("n_slots must be >= 0")
    B = 1 if by_segment else n_add
    Hkv = S // B
    shape = (n_slots,) if by_segment else (n_slots, Hkv)
    for t, name, want in ((rows, "rows", None), (add, "add", None), (tables, "tables", None),
                          (free_pages, "free_pages", None), (head, "head", (1,)), (rows_out, "rows_out", (S,)),
                          (head_out, "head_out", (1,)), (cu, "cu", (n_add + 1,)), (status, "status", (1,)),
                          (slots, "slots", shape)):
        if t is not None:
            _check_int32(t, name, want)
    for t, name, own in ((rows_out, "rows_out", rows), (head_out, "head_out", head)):
        if t is not None and t.data_ptr() != own.data_ptr():
            for other in (rows, add, tables, free_pages, head, slots, cu, status,
                          head_out if name == "rows_out" else rows_out):
                if other is not None and _overlap(t, other):
                    _refuse(f"{name} overlaps another argument: it may only be the tensor that it replaces")
    handle = _raw_stream(index) if stream is None else None
    if handle is None:
        return _switched(page_update, index, stream, (rows, add, tables, free_pages, head),
                         dict(page_size=page_size, n_slots=n_slots, by_segment=by_segment, rows_out=rows_out,
                              head_out=head_out, slots=slots, cu=cu, status=status))
    if slots is None or rows_out is None or cu is None or head_out is None or status is None:
        # each at a multiple of 16 bytes
        n = n_slots if by_segment else n_slots * Hkv
        sizes = (n, -n % 4, S, -S % 4, n_add + 1, (3 - n_add) % 4, 1, 3, 1)
        parts = torch.empty(sum(sizes), dtype=torch.int32, device=rows.device).split_with_sizes(sizes)
        if slots is None:
            slots = parts[0] if by_segment else parts[0].view(shape)
        rows_out = parts[2] if rows_out is None else rows_out
        cu = parts[4] if cu is None else cu
        head_out = parts[6] if head_out is None else head_out
        status = parts[8] if status is None else status
    desc = PageDesc(B, Hkv, page_size, tables.shape[1], 1 if by_segment else 0, 0, free_pages.shape[0], n_slots)
    st = load_library().sgdkv_page_update(
        ctypes.byref(desc), rows.data_ptr(), add.data_ptr(), tables.data_ptr(), free_pages.data_ptr(), head.data_ptr(),
        rows_out.data_ptr(), head_out.data_ptr(), cu.data_ptr(), slots.data_ptr(), status.data_ptr(), handle)
    if st:
        _check(st)
    return dict(slots=slots, rows=rows_out, head=head_out, cu=cu, status=status, tables=tables, free_pages=free_pages)


def paged_store(k_rows, v_rows, slots, k_pages, v_pages, *, stream=None):
    """Copy rows [n, d] to their slots (sgdkv_paged_store): slots int32 [n], -1 for none."""
    index = _gpu_of(k_pages, v_pages, k_rows, v_rows, slots)
    pool = page_pool(k_pages, v_pages)
    if k_rows.dim() != 2:
        _refuse("k_rows and v_rows must be [n, d]")
    shape = (k_rows.shape[0], k_pages.shape[2])
    _check_dense(k_rows, "k_rows", shape, k_pages.dtype)
    _check_dense(v_rows, "v_rows", shape, k_pages.dtype)
    _check_int32(slots, "slots", shape[:1])
    handle = _raw_stream(index) if stream is None else None
    if handle is None:
        return _switched(paged_store, index, stream, (k_rows, v_rows, slots, k_pages, v_pages), {})
    st = load_library().sgdkv_paged_store(ctypes.byref(pool), k_rows.data_ptr(), v_rows.data_ptr(), slots.data_ptr(),
                                          shape[0], handle)
    if st:
        _check(st)


def _token_stride(t, name, d):
    """Elements between tokens of t [T, heads, d], whose heads must be dense."""
    T, heads, _ = t.shape
    if T and heads and (t.stride(2) != 1 or (heads > 1 and t.stride(1) != d)):
        _refuse(f"the heads of a token of {name} must be dense")
    return t.stride(0) if T > 1 else heads * d


def norm_rope_store(q, k, v, positions, slots, k_pages, v_pages, *, inv_freq=None, q_weight=None, k_weight=None,
                    eps: float = 1e-6, interleaved: bool = False, q_out=None, stream=None):
    """New tokens' heads in one pass (sgdkv_norm_rope_store): queries [T, Hq, d] and keys [T, Hkv, d] normalised per
    head (with q_weight, k_weight [d]) and rotated by positions (int32 [T]) with inv_freq (fp32 [rot_dim / 2];
    None: no rotation), keys and values stored to slots (int32 [T, Hkv], -1 for none). q, k and v may be parts of
    one projection's output. q may be None. Returns q_out [T, Hq, d]."""
    import torch
    index = _gpu_of(k_pages, v_pages, q, k, v, positions, slots, inv_freq, q_weight, k_weight, q_out)
    pool = page_pool(k_pages, v_pages)
    dt, d = k_pages.dtype, k_pages.shape[2]
    if k.dim() != 3 or v.shape != k.shape or k.shape[2] != d or k.dtype is not dt or v.dtype is not dt:
        _refuse("k and v must be [T, Hkv, d] of the pool's dtype")
    T, Hkv, _ = k.shape
    Hq = q_stride = 0
    if q is not None:
        if q.dim() != 3 or q.shape[0] != T or q.shape[2] != d or q.dtype is not dt:
            _refuse("q must be [T, Hq, d] of the pool's dtype")
        Hq = q.shape[1]
        q_stride = _token_stride(q, "q", d)
        if q_out is not None:
            _check_dense(q_out, "q_out", (T, Hq, d), dt)
    if q_weight is not None:
        _check_dense(q_weight, "q_weight", (d,), dt)
    if k_weight is not None:
        _check_dense(k_weight, "k_weight", (d,), dt)
    if inv_freq is not None:
        _check_dense(inv_freq, "inv_freq", (inv_freq.numel(),), torch.float32)
    _check_int32(positions, "positions", (T,))
    _check_int32(slots, "slots", (T, Hkv))
    desc = NormRopeDesc(T, Hq, Hkv, q_stride, _token_stride(k, "k", d), _token_stride(v, "v", d),
                        0 if inv_freq is None else 2 * inv_freq.shape[0], 1 if interleaved else 0, eps, 0)
    handle = _raw_stream(index) if stream is None else None
    if handle is None:
        return _switched(norm_rope_store, index, stream, (q, k, v, positions, slots, k_pages, v_pages),
                         dict(inv_freq=inv_freq, q_weight=q_weight, k_weight=k_weight, eps=eps,
                              interleaved=interleaved, q_out=q_out))
    if Hq and q_out is None:
        q_out = torch.empty((T, Hq, d), dtype=dt, device=q.device)
    st = load_library().sgdkv_norm_rope_store(
        ctypes.byref(pool), ctypes.byref(desc), q.data_ptr() if Hq else None, k.data_ptr(), v.data_ptr(),
        positions.data_ptr(), slots.data_ptr(), None if inv_freq is None else inv_freq.data_ptr(),
        None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
        q_out.data_ptr() if Hq else None, handle)
    if st:
        _check(st)
    return q_out


def _paged_desc(q, num_kv_heads, batch, max_new, max_pages, out_dtype, causal, scale) -> PagedDesc:
    import torch
    if out_dtype is not None and out_dtype is not torch.bfloat16 and out_dtype is not torch.float32:
        _refuse(f"out_dtype {out_dtype}")
    od = _dtype_code(q) if out_dtype is None else (DTYPE_BF16 if out_dtype is torch.bfloat16 else DTYPE_F32)
    return PagedDesc(batch, q.shape[1], num_kv_heads, od, q.shape[0], max_new, max_pages, 1 if causal else 0, scale)


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
    index = _gpu_of(q, k_pages, v_pages, tables, rows, cu_new, out, lse, workspace)
    pool = page_pool(k_pages, v_pages)
    if q.dim() != 3 or q.shape[2] != k_pages.shape[2] or q.dtype is not k_pages.dtype or not q.is_contiguous():
        _refuse("q must be a dense [T, Hq, d] of the pool's dtype")
    if tables.dim() != 2 or rows.dim() != 1 or cu_new.dim() != 1 or cu_new.shape[0] < 2:
        _refuse("tables must be [B * Hkv, max_pages], rows [B * Hkv] and cu_new [B + 1]")
    B, shape = cu_new.shape[0] - 1, q.shape
    if not rows.shape[0] == tables.shape[0] == B * num_kv_heads:
        _refuse(f"{rows.shape[0]} rows and {tables.shape[0]} tables for {B} sequences of {num_kv_heads} KV heads")
    _check_int32(tables, "tables")
    _check_int32(rows, "rows")
    _check_int32(cu_new, "cu_new")
    desc = _paged_desc(q, num_kv_heads, B, max_new, tables.shape[1], out_dtype, causal, scale)
    od = torch.bfloat16 if desc.out_dtype == DTYPE_BF16 else torch.float32
    if out is not None:
        _check_dense(out, "out", shape, od)
    if workspace is not None and not workspace.is_contiguous():
        _refuse("workspace must be contiguous")
    if with_lse and lse is not None:
        _check_dense(lse, "lse", shape[:2], torch.float32)
    handle = _raw_stream(index) if stream is None else None
    if handle is None:
        return _switched(paged_attention, index, stream, (q, k_pages, v_pages, tables, rows, cu_new, num_kv_heads),
                         dict(max_new=max_new, causal=causal, scale=scale, out_dtype=out_dtype, with_lse=with_lse,
                              out=out, lse=lse, workspace=workspace))
    if out is None:
        out = torch.empty(shape, dtype=od, device=q.device)
    if with_lse and lse is None:
        lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(paged_attention_workspace_size(q, num_kv_heads, B, max_new=max_new), q.device)
    st = load_library().sgdkv_paged_attention(
        ctypes.byref(pool), ctypes.byref(desc), q.data_ptr(), tables.data_ptr(), rows.data_ptr(), cu_new.data_ptr(),
        out.data_ptr(), lse.data_ptr() if with_lse else None, workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), handle)
    if st:
        _check(st)
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
