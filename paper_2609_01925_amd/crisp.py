"""Python binding of libcrisp (include/crisp.h): argument marshalling only.

Every function takes torch tensors that already live on the GPU, passes their
device pointers and the current HIP stream to the C entry point of the same
name, and returns the output tensors it allocated.  All computation happens in
the HIP kernels of libcrisp.so; if the library is missing, importing this
module raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Tuple

import torch

# CRISP_DEBUG=1 in the environment loads the debug build, which also checks the inputs on
# the device (non-finite values, malformed caller lists) and waits for the stream to do so.
_LIB_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_LIB_DIR, "libcrisp_debug.so" if os.environ.get("CRISP_DEBUG") == "1" else "libcrisp.so")
DEBUG_LIB_PATH = os.path.join(_LIB_DIR, "libcrisp_debug.so")

CRISP_OK, CRISP_EINVAL, CRISP_EUNSUPPORTED, CRISP_EHIP = 0, 1, 2, 3
ROUTE_VS, ROUTE_PE = 0, 1


class CrispShape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32)]


class CrispParams(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("tau_proxy", ctypes.c_float), ("gamma", ctypes.c_float),
                ("w_sink", ctypes.c_int32), ("w_local", ctypes.c_int32), ("k_min_blocks", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("route_mode", ctypes.c_int32), ("vs_mode", ctypes.c_int32),
                ("tau_jsd", ctypes.c_float), ("floor_mode", ctypes.c_int32), ("dense_below_len", ctypes.c_int32)]


class CrispCacheShape(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block", ctypes.c_int32), ("format", ctypes.c_int32)]


class CrispCacheBatch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_rows", ctypes.c_int32)]


class CrispError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{msg} (status {status})")
        self.status = status


def _load(path: str = _LIB_PATH):
    if not os.path.exists(path):
        raise ImportError(f"libcrisp.so not built at {path}; run `python -m paper_2609_01925_amd.build`")
    lib = ctypes.CDLL(path)
    P, F, I32, I64, SZ = ctypes.c_void_p, ctypes.c_float, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    sh, pa = ctypes.POINTER(CrispShape), ctypes.POINTER(CrispParams)
    cs, cb = ctypes.POINTER(CrispCacheShape), ctypes.POINTER(CrispCacheBatch)
    sig = {
        "crisp_params_default": (None, [pa]),
        "crisp_col_capacity": (I64, [sh]),
        "crisp_workspace_size": (ctypes.c_int, [sh, ctypes.POINTER(SZ)]),
        "crisp_prefill_workspace_size": (ctypes.c_int, [sh, ctypes.POINTER(SZ)]),
        "crisp_estimate": (ctypes.c_int, [sh, pa, P, P, P, P, P, P, SZ, P]),
        "crisp_jsd": (ctypes.c_int, [sh, pa, P, P, P, P, P, SZ, P]),
        "crisp_route_select": (ctypes.c_int, [sh, pa, P, P, P, P, P, P, P, P, I64, P, P, SZ, P]),
        "crisp_sparse_workspace_size": (ctypes.c_int, [sh, ctypes.POINTER(SZ)]),
        "crisp_sparse_attn": (ctypes.c_int, [sh, F, P, P, P, P, P, I64, P, P, SZ, P]),
        "crisp_sparse_attn_noalloc": (ctypes.c_int, [sh, F, P, P, P, P, P, I64, P, P]),
        "crisp_prefill_attn": (ctypes.c_int, [sh, pa, P, P, P, P, P, P, P, P, SZ, P]),
        "crisp_dense_attn": (ctypes.c_int, [sh, F, P, P, P, P, P]),
        "crisp_cache_bytes": (ctypes.c_int, [cs, ctypes.POINTER(SZ), ctypes.POINTER(SZ)]),
        "crisp_cache_append": (ctypes.c_int, [cs, cb, P, P, P, P, P, P, I64, I64, P, I64, I64, P]),
        "crisp_cache_attn_workspace_size": (ctypes.c_int, [cs, cb, I32, ctypes.POINTER(SZ)]),
        "crisp_cache_attn": (ctypes.c_int, [cs, cb, I32, F, P, P, P, P, P, P, I64, I64, P, I64, I64, P, SZ, P]),
        "crisp_cache_copy": (ctypes.c_int, [cs, P, P, P, I32, P, P]),
        "crisp_pool_words": (I64, [I32]),
        "crisp_pool_init": (ctypes.c_int, [I32, P, P]),
        "crisp_pool_reserve": (ctypes.c_int, [I32, I32, I32, I32, P, P, P, P, P, P]),
        "crisp_pool_fork": (ctypes.c_int, [I32, I32, I32, I32, P, P, P, P, P, I32, P, P]),
        "crisp_pool_free": (ctypes.c_int, [I32, I32, I32, P, P, P, P, I32, P]),
        "crisp_pool_compact": (ctypes.c_int, [I32, I32, I32, P, P, P, P, P]),
        "crisp_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "crisp_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()
EXPORTED = ("crisp_params_default", "crisp_col_capacity", "crisp_workspace_size", "crisp_prefill_workspace_size",
            "crisp_sparse_workspace_size", "crisp_estimate", "crisp_jsd", "crisp_route_select", "crisp_sparse_attn",
            "crisp_sparse_attn_noalloc", "crisp_prefill_attn", "crisp_dense_attn", "crisp_status_string", "crisp_last_error",
            "crisp_cache_bytes", "crisp_cache_append", "crisp_cache_attn_workspace_size", "crisp_cache_attn",
            "crisp_cache_copy", "crisp_pool_words", "crisp_pool_init", "crisp_pool_reserve", "crisp_pool_fork",
            "crisp_pool_free", "crisp_pool_compact")

# route_mode / vs_mode values (include/crisp.h)
ROUTE_BY_CSTRUCT, ROUTE_BY_JSD = 0, 1
VS_FLOOR, VS_GAMMA = 0, 1
FLOOR_MEAN, FLOOR_MEDIAN = 0, 1
# cache formats
CACHE_E4M3, CACHE_INT8 = 0, 1


def _check(status: int, what: str):
    if status != CRISP_OK:
        msg = lib.crisp_last_error().decode()
        raise CrispError(status, f"{what}: {lib.crisp_status_string(status).decode()}: {msg}")


def make_params(alpha=1.0, tau_proxy=0.2, gamma=0.95, w_sink=128, w_local=128, k_min_blocks=0,
                softmax_scale=0.0, route_mode=ROUTE_BY_CSTRUCT, vs_mode=VS_FLOOR, tau_jsd=0.1,
                floor_mode=FLOOR_MEAN, dense_below_len=0) -> CrispParams:
    return CrispParams(alpha, tau_proxy, gamma, w_sink, w_local, k_min_blocks, softmax_scale, route_mode, vs_mode,
                       tau_jsd, floor_mode, dense_below_len)


def flexprefill_params(gamma=0.95, tau_jsd=0.1, **kw) -> CrispParams:
    """The FlexPrefill comparator (App. A): JSD routing and gamma-coverage VS selection."""
    return make_params(gamma=gamma, tau_jsd=tau_jsd, route_mode=ROUTE_BY_JSD, vs_mode=VS_GAMMA, **kw)


def crisp_params_default() -> CrispParams:
    p = CrispParams()
    lib.crisp_params_default(ctypes.byref(p))
    return p


def shape_of(q: torch.Tensor, k: torch.Tensor, block: int) -> CrispShape:
    return CrispShape(q.shape[0], k.shape[0], q.shape[1], q.shape[2], block)


def n_blocks(n: int, block: int) -> int:
    return -(-n // block)


def crisp_col_capacity(shape: CrispShape) -> int:
    return int(lib.crisp_col_capacity(ctypes.byref(shape)))


def crisp_workspace_size(shape: CrispShape) -> int:
    b = ctypes.c_size_t()
    _check(lib.crisp_workspace_size(ctypes.byref(shape), ctypes.byref(b)), "crisp_workspace_size")
    return int(b.value)


def crisp_prefill_workspace_size(shape: CrispShape) -> int:
    b = ctypes.c_size_t()
    _check(lib.crisp_prefill_workspace_size(ctypes.byref(shape), ctypes.byref(b)), "crisp_prefill_workspace_size")
    return int(b.value)


def crisp_sparse_workspace_size(shape: CrispShape) -> int:
    b = ctypes.c_size_t()
    _check(lib.crisp_sparse_workspace_size(ctypes.byref(shape), ctypes.byref(b)), "crisp_sparse_workspace_size")
    return int(b.value)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device) -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _inputs(q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor] = None):
    """q [H_q, n, d], k and v [H_kv, n, d]: contiguous bf16 on one CUDA device.  The C ABI
    sees only pointers, so every size it will read is checked here."""
    ts = (q, k) if v is None else (q, k, v)
    for t in ts:
        if not (t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous() and t.dim() == 3):
            raise ValueError("q, k, v must be contiguous 3-d bf16 CUDA tensors [heads, seq, head_dim]")
        if t.device != q.device:
            raise ValueError("q, k, v must be on one device")
    if k.shape[1:] != q.shape[1:]:
        raise ValueError(f"k {tuple(k.shape)} does not match q {tuple(q.shape)} in seq_len and head_dim")
    if v is not None and v.shape != k.shape:
        raise ValueError(f"v {tuple(v.shape)} must have k's shape {tuple(k.shape)}")


def _tensor(t: torch.Tensor, name: str, dtype, shape, device):
    """A caller-given buffer: contiguous, of the given dtype and shape (None: any size in that
    dimension) on the given device."""
    ok = t.is_cuda and t.device == device and t.dtype == dtype and t.is_contiguous() and t.dim() == len(shape)
    ok = ok and all(w is None or t.shape[i] == w for i, w in enumerate(shape))
    if not ok:
        raise ValueError(f"{name} must be a contiguous {dtype} CUDA tensor of shape {shape} on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def _tensor_out(out: torch.Tensor, q: torch.Tensor) -> torch.Tensor:
    _tensor(out, "out", torch.bfloat16, tuple(q.shape), q.device)
    return out


def _ws(ws: torch.Tensor, device) -> torch.Tensor:
    _tensor(ws, "ws", torch.uint8, (None,), device)
    return ws


def workspace(shape: CrispShape, device, prefill: bool = False) -> torch.Tensor:
    nbytes = crisp_prefill_workspace_size(shape) if prefill else crisp_workspace_size(shape)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def crisp_estimate(q: torch.Tensor, k: torch.Tensor, params: CrispParams, block: int = 128,
                   ws: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Stages 1-2 -> (c_struct [H_q], p_v [H_q, N_b], p_s [H_q, N_b]) float32."""
    _inputs(q, k)
    sh = shape_of(q, k, block)
    nb = n_blocks(q.shape[1], block)
    dev = q.device
    cs = torch.empty(q.shape[0], dtype=torch.float32, device=dev)
    pv = torch.empty(q.shape[0], nb, dtype=torch.float32, device=dev)
    ps = torch.empty(q.shape[0], nb, dtype=torch.float32, device=dev)
    ws = workspace(sh, dev) if ws is None else _ws(ws, dev)
    _check(lib.crisp_estimate(ctypes.byref(sh), ctypes.byref(params), _ptr(q), _ptr(k), _ptr(cs), _ptr(pv), _ptr(ps),
                              _ptr(ws), ws.numel(), _stream(dev)), "crisp_estimate")
    return cs, pv, ps


def crisp_jsd(q: torch.Tensor, k: torch.Tensor, p_v: torch.Tensor, params: CrispParams, block: int = 128,
              ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """FlexPrefill's pattern search (App. A) -> D_JS per query head, float32 [H_q]."""
    _inputs(q, k)
    sh = shape_of(q, k, block)
    dev = q.device
    _tensor(p_v, "p_v", torch.float32, (q.shape[0], n_blocks(q.shape[1], block)), dev)
    jsd = torch.empty(q.shape[0], dtype=torch.float32, device=dev)
    ws = workspace(sh, dev) if ws is None else _ws(ws, dev)
    _check(lib.crisp_jsd(ctypes.byref(sh), ctypes.byref(params), _ptr(q), _ptr(k), _ptr(p_v), _ptr(jsd), _ptr(ws),
                         ws.numel(), _stream(dev)), "crisp_jsd")
    return jsd


def crisp_route_select(q: torch.Tensor, k: torch.Tensor, c_struct: torch.Tensor, p_v: torch.Tensor,
                       p_s: torch.Tensor, params: CrispParams, block: int = 128, want_mask: bool = True,
                       ws: Optional[torch.Tensor] = None):
    """Stage 3 -> (route int8 [H_q], row_ptr int32 [H_q, N_b+1], col_idx int32 [H_q, cap],
    dir_mask uint8 [H_q, 2, N_b] or None).  c_struct is the route score: C_struct, or D_JS
    from crisp_jsd when params.route_mode is ROUTE_BY_JSD."""
    _inputs(q, k)
    sh = shape_of(q, k, block)
    nb = n_blocks(q.shape[1], block)
    dev = q.device
    _tensor(c_struct, "c_struct", torch.float32, (q.shape[0],), dev)
    _tensor(p_v, "p_v", torch.float32, (q.shape[0], nb), dev)
    _tensor(p_s, "p_s", torch.float32, (q.shape[0], nb), dev)
    cap = max(crisp_col_capacity(sh), 1)
    route = torch.empty(q.shape[0], dtype=torch.int8, device=dev)
    row_ptr = torch.empty(q.shape[0], nb + 1, dtype=torch.int32, device=dev)
    col_idx = torch.empty(q.shape[0], cap, dtype=torch.int32, device=dev)
    dmask = torch.empty(q.shape[0], 2, nb, dtype=torch.uint8, device=dev) if want_mask else None
    ws = workspace(sh, dev) if ws is None else _ws(ws, dev)
    _check(lib.crisp_route_select(ctypes.byref(sh), ctypes.byref(params), _ptr(q), _ptr(k), _ptr(c_struct),
                                  _ptr(p_v), _ptr(p_s), _ptr(route), _ptr(row_ptr), _ptr(col_idx), cap,
                                  _ptr(dmask), _ptr(ws), ws.numel(), _stream(dev)), "crisp_route_select")
    return route, row_ptr, col_idx, dmask


def crisp_sparse_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, row_ptr: torch.Tensor,
                      col_idx: torch.Tensor, block: int = 128, softmax_scale: float = 0.0,
                      out: Optional[torch.Tensor] = None, balance: bool = True,
                      ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Stage 4 over caller-given CSR lists -> o bf16 [H_q, n, d].  balance=False passes no
    workspace (fixed row order)."""
    _inputs(q, k, v)
    sh = shape_of(q, k, block)
    _tensor(row_ptr, "row_ptr", torch.int32, (q.shape[0], n_blocks(q.shape[1], block) + 1), q.device)
    _tensor(col_idx, "col_idx", torch.int32, (q.shape[0], None), q.device)
    o = torch.empty_like(q) if out is None else _tensor_out(out, q)
    if balance and ws is not None:
        _ws(ws, q.device)
    if balance and ws is None:
        ws = torch.empty(max(crisp_sparse_workspace_size(sh), 256), dtype=torch.uint8, device=q.device)
    if not balance:
        ws = None
    _check(lib.crisp_sparse_attn(ctypes.byref(sh), softmax_scale, _ptr(q), _ptr(k), _ptr(v), _ptr(row_ptr),
                                 _ptr(col_idx), col_idx.shape[1], _ptr(o), _ptr(ws), 0 if ws is None else ws.numel(),
                                 _stream(q.device)), "crisp_sparse_attn")
    return o


def crisp_sparse_attn_noalloc(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, row_ptr: torch.Tensor,
                              col_idx: torch.Tensor, block: int = 128, softmax_scale: float = 0.0,
                              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Stage 4 over caller-given CSR lists with the library's own static schedule area (the
    C entry point allocates nothing; calls that overlap on one GPU race) -> o bf16 [H_q, n, d]."""
    _inputs(q, k, v)
    sh = shape_of(q, k, block)
    _tensor(row_ptr, "row_ptr", torch.int32, (q.shape[0], n_blocks(q.shape[1], block) + 1), q.device)
    _tensor(col_idx, "col_idx", torch.int32, (q.shape[0], None), q.device)
    o = torch.empty_like(q) if out is None else _tensor_out(out, q)
    _check(lib.crisp_sparse_attn_noalloc(ctypes.byref(sh), softmax_scale, _ptr(q), _ptr(k), _ptr(v), _ptr(row_ptr),
                                         _ptr(col_idx), col_idx.shape[1], _ptr(o), _stream(q.device)),
           "crisp_sparse_attn_noalloc")
    return o


def crisp_dense_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, block: int = 128,
                     softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Dense causal baseline with the same kernel -> o bf16 [H_q, n, d]."""
    _inputs(q, k, v)
    sh = shape_of(q, k, block)
    o = torch.empty_like(q) if out is None else _tensor_out(out, q)
    _check(lib.crisp_dense_attn(ctypes.byref(sh), softmax_scale, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                _stream(q.device)), "crisp_dense_attn")
    return o


def crisp_prefill_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, params: CrispParams, block: int = 128,
                       return_lists: bool = False, ws: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None):
    """All stages (Alg. 1) -> o, or (o, route, row_ptr, col_idx) with return_lists."""
    _inputs(q, k, v)
    sh = shape_of(q, k, block)
    dev = q.device
    o = torch.empty_like(q) if out is None else _tensor_out(out, q)
    if ws is not None:
        _ws(ws, dev)
    if return_lists:
        nb = n_blocks(q.shape[1], block)
        cap = max(crisp_col_capacity(sh), 1)
        route = torch.empty(q.shape[0], dtype=torch.int8, device=dev)
        row_ptr = torch.empty(q.shape[0], nb + 1, dtype=torch.int32, device=dev)
        col_idx = torch.empty(q.shape[0], cap, dtype=torch.int32, device=dev)
        ws = workspace(sh, dev) if ws is None else ws
    else:
        route = row_ptr = col_idx = None
        ws = workspace(sh, dev, prefill=True) if ws is None else ws
    _check(lib.crisp_prefill_attn(ctypes.byref(sh), ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                  _ptr(route), _ptr(row_ptr), _ptr(col_idx), _ptr(ws), ws.numel(), _stream(dev)),
                    "crisp_prefill_attn")
    return (o, route, row_ptr, col_idx) if return_lists else o


# ---------------------------------------------------------------- the 8-bit paged K/V cache


class Cache:
    """One layer's K and V: pages uint8 [n_pages, H_kv, block / 64, 2, 8192] and scales float32
    [n_pages, H_kv, 2] on one GPU, in the layout of include/crisp.h.  Neither needs contents."""

    def __init__(self, pages: torch.Tensor, scales: torch.Tensor, fmt: int = CACHE_E4M3):
        _tensor(pages, "pages", torch.uint8, (None, None, None, 2, 8192), pages.device)
        _tensor(scales, "scales", torch.float32, (pages.shape[0], pages.shape[1], 2), pages.device)
        self.pages, self.scales, self.fmt = pages, scales, fmt
        self.n_pages, self.n_kv_heads, self.block = pages.shape[0], pages.shape[1], 64 * pages.shape[2]
        self.shape = CrispCacheShape(self.n_pages, self.n_kv_heads, 128, self.block, fmt)
        self._ref, self._gpu = ctypes.byref(self.shape), pages.get_device()
        crisp_cache_bytes(self.shape)  # raises on a size or format that the library does not take


def make_cache(n_pages: int, n_kv_heads: int, block: int = 64, fmt: int = CACHE_E4M3, device="cuda") -> Cache:
    """A cache without contents."""
    crisp_cache_bytes(CrispCacheShape(n_pages, n_kv_heads, 128, block, fmt))
    return Cache(torch.empty(n_pages, n_kv_heads, block // 64, 2, 8192, dtype=torch.uint8, device=device),
                 torch.empty(n_pages, n_kv_heads, 2, dtype=torch.float32, device=device), fmt)


def crisp_cache_bytes(shape: CrispCacheShape) -> Tuple[int, int]:
    """Bytes of (pages, scales)."""
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib.crisp_cache_bytes(ctypes.byref(shape), ctypes.byref(a), ctypes.byref(b)), "crisp_cache_bytes")
    return int(a.value), int(b.value)


def _call(gpu: int, what: str, fn, *args) -> None:
    """fn(*args, the GPU's current stream) with that GPU as the current device.  These calls are made once
    a layer and token, so the checks before them are kept short."""
    if torch.cuda.current_device() == gpu:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(gpu))
    else:
        with torch.cuda.device(gpu):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(gpu))
    if status != CRISP_OK:
        _check(status, what)


def _i32(t: torch.Tensor, name: str, dims: int, gpu: int) -> torch.Size:
    shape = t.shape
    if t.dtype is not torch.int32 or len(shape) != dims or t.get_device() != gpu or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dims}-d int32 tensor on cuda:{gpu}, "
                         f"got {t.dtype} {tuple(shape)} on {t.device}")
    return shape


def _i32_of(t: torch.Tensor, name: str, shape, gpu: int) -> None:
    if _i32(t, name, len(shape), gpu) != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _batch(gpu: int, table, seq_len, row_ptr, n_rows: int) -> CrispCacheBatch:
    n, wide = _i32(table, "table", 2, gpu)
    _i32_of(seq_len, "seq_len", (n,), gpu)
    _i32_of(row_ptr, "row_ptr", (n + 1,), gpu)
    return CrispCacheBatch(n, wide, n_rows)


def _rows(t: torch.Tensor, name: str, heads: Optional[int], gpu: int) -> Tuple[int, int, int, int]:
    """A packed tensor [heads, n_rows, 128] of any head and row stride -> heads, n_rows and those strides, 0
    where there is no second head or row."""
    shape, stride = t.shape, t.stride()
    if (t.dtype is not torch.bfloat16 or len(shape) != 3 or t.get_device() != gpu or shape[2] != 128 or stride[2] != 1
            or (heads is not None and shape[0] != heads)):
        raise ValueError(f"{name} must be a bf16 tensor [{'heads' if heads is None else heads}, n_rows, 128] on cuda:{gpu} "
                         f"whose rows are contiguous, got {t.dtype} {tuple(shape)} strides {stride} on {t.device}")
    return shape[0], shape[1], stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0


def crisp_cache_append(cache: Cache, table: torch.Tensor, seq_len: torch.Tensor, row_ptr: torch.Tensor,
                       k: torch.Tensor, v: torch.Tensor) -> None:
    """K and V rows [H_kv, n_rows, 128] (any head and row strides that are multiples of 8) quantised into the
    pages behind each sequence's seq_len tokens."""
    gpu = cache._gpu
    heads, n, kh, kr = _rows(k, "k", cache.n_kv_heads, gpu)
    _, m, vh, vr = _rows(v, "v", heads, gpu)
    if m != n:
        raise ValueError(f"v {tuple(v.shape)} must have k's shape {tuple(k.shape)}")
    b = _batch(gpu, table, seq_len, row_ptr, n)
    _call(gpu, "crisp_cache_append", lib.crisp_cache_append, cache._ref, b, cache.pages.data_ptr(),
          cache.scales.data_ptr(), table.data_ptr(), seq_len.data_ptr(), row_ptr.data_ptr(), k.data_ptr(), kh, kr,
          v.data_ptr(), vh, vr)


def crisp_cache_attn_workspace_size(cache: Cache, n_q_heads: int, n_seqs: int, max_pages: int, n_rows: int) -> int:
    n = ctypes.c_size_t()
    b = CrispCacheBatch(n_seqs, max_pages, n_rows)
    _check(lib.crisp_cache_attn_workspace_size(ctypes.byref(cache.shape), ctypes.byref(b), n_q_heads, ctypes.byref(n)),
           "crisp_cache_attn_workspace_size")
    return int(n.value)


def cache_workspace(cache: Cache, n_q_heads: int, n_seqs: int, n_rows: int, max_pages: Optional[int] = None) -> torch.Tensor:
    """A workspace for crisp_cache_attn calls of n_seqs sequences and up to n_rows rows in a table of up to max_pages pages
    a sequence; without max_pages of any width."""
    wide = (1 << 30) // cache.block if max_pages is None else max_pages
    if max_pages is None and n_seqs:
        wide = min(wide, ((1 << 31) - 1) // n_seqs)
    nbytes = crisp_cache_attn_workspace_size(cache, n_q_heads, n_seqs, wide, n_rows)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=cache.pages.device)


def crisp_cache_attn(cache: Cache, table: torch.Tensor, seq_len: torch.Tensor, row_ptr: torch.Tensor, q: torch.Tensor,
                     softmax_scale: float = 0.0, ws: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of rows q [H_q, n_rows, 128] over the cached tokens (the rows' own appended before)
    -> o bf16 [H_q, n_rows, 128]; rows that row_ptr does not cover are left as they were in out."""
    gpu = cache._gpu
    heads, n, qh, qr = _rows(q, "q", None, gpu)
    o = torch.empty((heads, n, 128), dtype=torch.bfloat16, device=q.device) if out is None else out
    _, m, oh, orow = _rows(o, "out", heads, gpu)
    if m != n:
        raise ValueError(f"out {tuple(o.shape)} must have q's shape {tuple(q.shape)}")
    b = _batch(gpu, table, seq_len, row_ptr, n)
    if ws is None:
        ws = cache_workspace(cache, heads, b.n_seqs, n, b.max_pages)
    elif ws.dtype is not torch.uint8 or ws.get_device() != gpu or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous uint8 tensor on cuda:{gpu}, got {ws.dtype} on {ws.device}")
    _call(gpu, "crisp_cache_attn", lib.crisp_cache_attn, cache._ref, b, heads, softmax_scale, cache.pages.data_ptr(),
          cache.scales.data_ptr(), table.data_ptr(), seq_len.data_ptr(), row_ptr.data_ptr(), q.data_ptr(), qh, qr,
          o.data_ptr(), oh, orow, ws.data_ptr(), ws.numel())
    return o


def crisp_cache_copy(cache: Cache, pairs: torch.Tensor, count: Optional[torch.Tensor] = None) -> None:
    """Page copies: pairs int32 [n, 2] of (from, to), of which the first count[0] count (all without it)."""
    gpu = cache._gpu
    n, two = _i32(pairs, "pairs", 2, gpu)
    if two != 2:
        raise ValueError(f"pairs must have shape [n, 2], got {tuple(pairs.shape)}")
    if count is not None:
        _i32_of(count, "count", (1,), gpu)
    _call(gpu, "crisp_cache_copy", lib.crisp_cache_copy, cache._ref, cache.pages.data_ptr(), cache.scales.data_ptr(),
          pairs.data_ptr(), n, None if count is None else count.data_ptr())


def crisp_pool_words(n_pages: int) -> int:
    n = int(lib.crisp_pool_words(n_pages))
    if n < 0:
        raise CrispError(CRISP_EINVAL, lib.crisp_last_error().decode())
    return n


def crisp_pool_init(n_pages: int, device="cuda") -> torch.Tensor:
    """A pool of n_pages pages, none in use: int32 [crisp_pool_words(n_pages)]; pool[:n_pages] are the uses."""
    if torch.device(device).type != "cuda":
        raise ValueError(f"a pool lives on a GPU, got device {device}")
    pool = torch.empty(crisp_pool_words(n_pages), dtype=torch.int32, device=device)
    _call(pool.get_device(), "crisp_pool_init", lib.crisp_pool_init, n_pages, pool.data_ptr())
    return pool


def pool_pages(pool: torch.Tensor) -> int:
    """The number of pages that a pool tensor is for."""
    words = pool.numel()
    n = words * 32 // 33
    if n < 1 or n + (n + 31) // 32 != words:
        raise ValueError(f"{words} words are no pool")
    return n


def _pool(pool: torch.Tensor, table: torch.Tensor, seq_len: Optional[torch.Tensor]) -> Tuple[int, int, int, int]:
    """GPU, pages, sequences, slots of a sequence."""
    gpu = pool.get_device()
    if gpu < 0:
        raise ValueError(f"pool must be a CUDA tensor, got one on {pool.device}")
    _i32(pool, "pool", 1, gpu)
    n_seqs, wide = _i32(table, "table", 2, gpu)
    if seq_len is not None:
        _i32_of(seq_len, "seq_len", (n_seqs,), gpu)
    return gpu, pool_pages(pool), n_seqs, wide


def crisp_pool_reserve(pool: torch.Tensor, block: int, table: torch.Tensor, seq_len: torch.Tensor,
                       counts: torch.Tensor) -> torch.Tensor:
    """Pages for counts[s] more tokens of each sequence -> granted int32 [n_seqs] (counts[s] or 0)."""
    gpu, n, n_seqs, wide = _pool(pool, table, seq_len)
    _i32_of(counts, "counts", (n_seqs,), gpu)
    granted = torch.empty_like(counts)
    _call(gpu, "crisp_pool_reserve", lib.crisp_pool_reserve, n, block, n_seqs, wide, pool.data_ptr(), table.data_ptr(),
          seq_len.data_ptr(), counts.data_ptr(), granted.data_ptr())
    return granted


def crisp_pool_fork(pool: torch.Tensor, block: int, table: torch.Tensor, seq_len: torch.Tensor, src: torch.Tensor,
                    dst: torch.Tensor) -> torch.Tensor:
    """Sequences dst[i] become copies of src[i] -> copies int32 [n, 2], the page pairs for crisp_cache_copy."""
    gpu, n, n_seqs, wide = _pool(pool, table, seq_len)
    m, = _i32(src, "src", 1, gpu)
    _i32_of(dst, "dst", (m,), gpu)
    copies = torch.empty((m, 2), dtype=torch.int32, device=pool.device)
    _call(gpu, "crisp_pool_fork", lib.crisp_pool_fork, n, block, n_seqs, wide, pool.data_ptr(), table.data_ptr(),
          seq_len.data_ptr(), src.data_ptr(), dst.data_ptr(), m, copies.data_ptr())
    return copies


def crisp_pool_free(pool: torch.Tensor, table: torch.Tensor, seq_len: torch.Tensor, ids: torch.Tensor) -> None:
    """Sequences ids[i] end: their pages lose a use, their rows become -1, their lengths 0."""
    gpu, n, n_seqs, wide = _pool(pool, table, seq_len)
    m, = _i32(ids, "ids", 1, gpu)
    _call(gpu, "crisp_pool_free", lib.crisp_pool_free, n, n_seqs, wide, pool.data_ptr(), table.data_ptr(),
          seq_len.data_ptr(), ids.data_ptr(), m)


def crisp_pool_compact(pool: torch.Tensor, table: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """The pages in use gathered at the front -> (moves int32 [max(1, n_pages // 2), 2], count int32 [1]) for
    crisp_cache_copy; pool and table follow."""
    gpu, n, n_seqs, wide = _pool(pool, table, None)
    moves = torch.empty((max(1, n // 2), 2), dtype=torch.int32, device=pool.device)
    count = torch.empty(1, dtype=torch.int32, device=pool.device)
    _call(gpu, "crisp_pool_compact", lib.crisp_pool_compact, n, n_seqs, wide, pool.data_ptr(), table.data_ptr(),
          moves.data_ptr(), count.data_ptr())
    return moves, count
