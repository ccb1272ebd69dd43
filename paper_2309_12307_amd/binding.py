"""ctypes binding of libs2attn.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU (or raw device
pointers), passes their addresses and the current HIP stream to the C ABI of
include/s2attn.h, and raises on a non-zero return code.  There is no fallback of
any kind: if the shared library has not been built, the first call raises.
"""
from __future__ import annotations

import ctypes
import os
import weakref

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("S2ATTN_LIB", os.path.join(_HERE, "libs2attn.so"))

BF16, F32, E4M3 = 0, 1, 2
SHIFT_SECOND_HALF, SHIFT_NONE, SHIFT_ALL = 0, 1, 2
WRAP_JOINT, WRAP_SPLIT = 0, 2
BWD_AUTO, BWD_RECOMPUTE, BWD_STORED_DS = 0, 1, 2
PAGED_WRITE, PAGED_READ, PAGED_FWD = 0, 1, 2

EXPORTS = [
    "s2attn_check_args", "s2attn_bwd_workspace_bytes", "s2attn_fwd", "s2attn_bwd",
    "s2attn_fwd_f32", "s2attn_bwd_f32", "s2attn_fwd_ex", "s2attn_bwd_ex",
    "s2attn_strerror", "s2attn_effective_flops", "s2attn_bwd_ex_marked",
    "s2attn_bwd_workspace_bytes_ex", "s2attn_bwd_ex_static",
    "s2attn_check_window_args", "s2attn_window_workspace_bytes", "s2attn_window_fwd", "s2attn_window_bwd",
    "s2attn_check_paged_args", "s2attn_paged_workspace_bytes", "s2attn_cache_write", "s2attn_cache_read",
    "s2attn_paged_fwd",
]


class S2AttnParams(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("o", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("dout", ctypes.c_void_p),
        ("dq", ctypes.c_void_p), ("dk", ctypes.c_void_p), ("dv", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("B", ctypes.c_int), ("N", ctypes.c_int), ("H", ctypes.c_int),
        ("Hkv", ctypes.c_int), ("D", ctypes.c_int), ("G", ctypes.c_int),
        ("dtype", ctypes.c_int), ("shift", ctypes.c_int), ("shift_rule", ctypes.c_int),
        ("wrap_variant", ctypes.c_int), ("scale", ctypes.c_float),
        ("q_strides", ctypes.c_longlong * 3), ("k_strides", ctypes.c_longlong * 3),
        ("v_strides", ctypes.c_longlong * 3), ("dq_strides", ctypes.c_longlong * 3),
        ("dk_strides", ctypes.c_longlong * 3), ("dv_strides", ctypes.c_longlong * 3),
        ("heads_total", ctypes.c_int), ("head_offset", ctypes.c_int), ("bwd_algo", ctypes.c_int),
    ]
    # what the window calls go by: the device of the tensors, what is wrong with them, and those not looked at yet
    device = problem = tensors = None


class S2AttnPagedParams(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("o", ctypes.c_void_p), ("lse", ctypes.c_void_p),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
        ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p), ("row_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("T", ctypes.c_int), ("B", ctypes.c_int), ("H", ctypes.c_int), ("Hkv", ctypes.c_int), ("D", ctypes.c_int),
        ("pages", ctypes.c_int), ("page_size", ctypes.c_int), ("table_cols", ctypes.c_int),
        ("dtype", ctypes.c_int), ("cache_dtype", ctypes.c_int), ("window", ctypes.c_int), ("sinks", ctypes.c_int),
        ("max_kv", ctypes.c_int), ("scale", ctypes.c_float),
        ("q_strides", ctypes.c_longlong * 2), ("k_strides", ctypes.c_longlong * 2), ("v_strides", ctypes.c_longlong * 2),
        ("k_cache_strides", ctypes.c_longlong * 3), ("v_cache_strides", ctypes.c_longlong * 3),
        ("k_exp_strides", ctypes.c_longlong * 3), ("v_exp_strides", ctypes.c_longlong * 3),
        ("table_stride", ctypes.c_longlong),
    ]


class S2AttnError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"s2attn error {code}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Opens libs2attn.so (built in-tree by build.py).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2309_12307_amd.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.s2attn_check_args.argtypes = [ctypes.POINTER(S2AttnParams), i]
        L.s2attn_check_args.restype = i
        L.s2attn_bwd_workspace_bytes.argtypes = [i] * 7
        L.s2attn_bwd_workspace_bytes.restype = sz
        L.s2attn_bwd_workspace_bytes_ex.argtypes = [ctypes.POINTER(S2AttnParams)]
        L.s2attn_bwd_workspace_bytes_ex.restype = sz
        for name in ("s2attn_fwd", "s2attn_fwd_f32"):
            f = getattr(L, name)
            f.argtypes = [vp] * 5 + [i] * 6 + [vp]
            f.restype = i
        for name in ("s2attn_bwd", "s2attn_bwd_f32"):
            f = getattr(L, name)
            f.argtypes = [vp] * 9 + [vp, sz] + [i] * 6 + [vp]
            f.restype = i
        for name in ("s2attn_fwd_ex", "s2attn_bwd_ex", "s2attn_bwd_ex_static"):
            f = getattr(L, name)
            f.argtypes = [ctypes.POINTER(S2AttnParams), vp]
            f.restype = i
        L.s2attn_bwd_ex_marked.argtypes = [ctypes.POINTER(S2AttnParams), vp, ctypes.POINTER(vp)]
        L.s2attn_bwd_ex_marked.restype = i
        L.s2attn_check_window_args.argtypes = [ctypes.POINTER(S2AttnParams), i, i, i]
        L.s2attn_check_window_args.restype = i
        L.s2attn_window_workspace_bytes.argtypes = [ctypes.POINTER(S2AttnParams), i, i]
        L.s2attn_window_workspace_bytes.restype = sz
        for name in ("s2attn_window_fwd", "s2attn_window_bwd"):
            f = getattr(L, name)
            f.argtypes = [ctypes.POINTER(S2AttnParams), i, i, vp]
            f.restype = i
        L.s2attn_check_paged_args.argtypes = [ctypes.POINTER(S2AttnPagedParams), i]
        L.s2attn_check_paged_args.restype = i
        L.s2attn_paged_workspace_bytes.argtypes = [ctypes.POINTER(S2AttnPagedParams)]
        L.s2attn_paged_workspace_bytes.restype = sz
        for name in ("s2attn_cache_write", "s2attn_cache_read", "s2attn_paged_fwd"):
            f = getattr(L, name)
            f.argtypes = [ctypes.POINTER(S2AttnPagedParams), vp]
            f.restype = i
        L.s2attn_strerror.argtypes = [i]
        L.s2attn_strerror.restype = ctypes.c_char_p
        L.s2attn_effective_flops.argtypes = [i] * 6
        L.s2attn_effective_flops.restype = ctypes.c_double
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().s2attn_strerror(code).decode()


def _check(code: int) -> None:
    if code != 0:
        raise S2AttnError(code, strerror(code))


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _ptrs(*ts):
    """Addresses of contiguous tensors (None for None)."""
    out = []
    for t in ts:
        if t is None:
            out.append(None)
        elif t.is_contiguous():
            out.append(t.data_ptr())
        else:
            raise ValueError("s2attn tensors must be contiguous")
    return out


_torch = None   # torch, imported at the first call that needs it


def _import_torch():
    global _torch
    import torch
    _torch = torch
    return torch


def _current_device() -> int:
    torch = _torch or _import_torch()
    try:
        if torch.cuda.is_initialized():
            return torch._C._cuda_getDevice()
    except AttributeError:
        pass
    return torch.cuda.current_device()


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    torch = _torch or _import_torch()
    try:   # the handle itself: no Stream object for a call of a few microseconds
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:
        pass
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t) -> int:
    torch = _torch or _import_torch()
    dtype = t.dtype
    if dtype == torch.bfloat16:
        return BF16
    if dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {dtype}")


def _dims(q, k):
    B, N, H, D = q.shape
    Hkv = k.shape[2]
    return B, N, H, Hkv, D


def bwd_workspace_bytes(B, N, H, Hkv, D, G, dtype=BF16) -> int:
    return int(lib().s2attn_bwd_workspace_bytes(B, N, H, Hkv, D, G, dtype))


def bwd_workspace_bytes_ex(p: "S2AttnParams") -> int:
    """Workspace size for a parameter block (accounts for its shift rule and head sharding)."""
    return int(lib().s2attn_bwd_workspace_bytes_ex(ctypes.byref(p)))


def effective_flops(B, N, H, D, G, which: int = 2) -> float:
    return float(lib().s2attn_effective_flops(B, N, H, D, G, which))


def _device_of(t) -> int:
    return t.device.index if t.is_cuda else -1


def make_params(q, k, v, o, lse, G, dout=None, dq=None, dk=None, dv=None, workspace=None,
                shift=-1, shift_rule=SHIFT_SECOND_HALF, wrap_variant=WRAP_JOINT, scale=0.0,
                dtype=None, dims=None, strided=False, heads_total=0, head_offset=0,
                bwd_algo=BWD_AUTO) -> S2AttnParams:
    """strided=True takes the {batch, token, head} strides of q, k, v (and dq, dk, dv) from
    the tensors themselves, so views into a packed (B, N, 3, H, D) tensor can be passed."""
    if dims is None:
        B, N, H, Hkv, D = _dims(q, k)
    else:
        B, N, H, Hkv, D = dims
    p = S2AttnParams()
    if q is not None and not isinstance(q, int):   # (a block for a size alone may have neither)
        tensors = (q, k, v, o, lse, dout, dq, dk, dv, workspace)
        if G == 0:   # for the window calls
            p.device, p.problem = _device_of(q), _problem_of(*tensors, (B, N, H, Hkv, D), strided)
        else:        # they may get any block: a look at the tensors that are still there then, none for the others' calls
            try:
                p.tensors = list(map(weakref.ref, tensors[:5] if dout is None else tensors)), strided
            except TypeError:   # addresses among them
                p.tensors = [x if x is None or isinstance(x, int) else weakref.ref(x) for x in tensors], strided
    p.q, p.k, p.v, p.o, p.lse = _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse)
    p.dout, p.dq, p.dk, p.dv = _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv)
    p.workspace = _ptr(workspace)
    p.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    p.B, p.N, p.H, p.Hkv, p.D, p.G = B, N, H, Hkv, D, G
    p.dtype = _dtype_code(q) if dtype is None else dtype
    p.shift, p.shift_rule, p.wrap_variant, p.scale = shift, shift_rule, wrap_variant, scale
    p.heads_total, p.head_offset, p.bwd_algo = heads_total, head_offset, bwd_algo
    if strided:
        for name, t in (("q", q), ("k", k), ("v", v), ("dq", dq), ("dk", dk), ("dv", dv)):
            if t is None or isinstance(t, int):
                continue
            if t.stride(3) != 1:
                raise ValueError("the head-dim axis must be contiguous")
            setattr(p, name + "_strides", (ctypes.c_longlong * 3)(t.stride(0), t.stride(1), t.stride(2)))
    return p


def _problem_of(q, k, v, o, lse, dout, dq, dk, dv, workspace, dims, strided):
    """What is wrong with a block's tensors (None: nothing): s2attn_window_fwd and s2attn_window_bwd refuse it."""
    B, N, H, Hkv, D = dims
    for shape, tensors in (((B, N, Hkv, D), dict(k=k, v=v, dk=dk, dv=dv)), ((B, N, H, D), dict(o=o, dout=dout, dq=dq, q=q))):
        for name, t in tensors.items():
            if t is None or isinstance(t, int):
                continue
            if t.shape != shape or t.dtype != q.dtype or t.device != q.device:
                return f"{name} must be {shape} of q's type on q's device"
            if name in ("o", "dout") or not strided:
                if not t.is_contiguous():
                    return f"{name} must be contiguous" + ("" if strided else " (or strided=True given)")
            elif not any(t.stride()[:3]) and max(shape[:3]) > 1:   # all zero stands for contiguous
                return f"{name} is one row, expanded"
    if not (lse is None or isinstance(lse, int)):
        if lse.shape != (B, H, N) or lse.element_size() != 4 or not lse.is_floating_point() or not lse.is_contiguous() or lse.device != q.device:
            return f"lse must be a contiguous float32 {(B, H, N)} on q's device"
    if not (workspace is None or isinstance(workspace, int)) and not (workspace.is_contiguous() and workspace.device == q.device):
        return "workspace must be contiguous on q's device"
    return None


def check_args(p: S2AttnParams, backward: bool) -> int:
    return int(lib().s2attn_check_args(ctypes.byref(p), 1 if backward else 0))


def s2attn_fwd(q, k, v, o, lse, G, stream=None) -> None:
    """o, lse <- S2-Attn(q, k, v) with the published defaults.  bf16 or fp32 tensors."""
    ptrs = _ptrs(q, k, v, o, lse)
    B, N, H, D = q.shape
    L = _lib or lib()
    f = L.s2attn_fwd if _dtype_code(q) == BF16 else L.s2attn_fwd_f32
    code = f(*ptrs, B, N, H, k.shape[2], D, G, _stream(stream))
    if code:
        _check(code)


def s2attn_bwd(q, k, v, o, dout, lse, dq, dk, dv, workspace, G, stream=None) -> None:
    """dq, dk, dv <- gradients of sum(o * dout); workspace is a uint8 device tensor."""
    ptrs = _ptrs(q, k, v, o, dout, lse, dq, dk, dv, workspace)
    B, N, H, D = q.shape
    L = _lib or lib()
    f = L.s2attn_bwd if _dtype_code(q) == BF16 else L.s2attn_bwd_f32
    code = f(*ptrs, workspace.numel() * workspace.element_size(), B, N, H, k.shape[2], D, G, _stream(stream))
    if code:
        _check(code)


def s2attn_fwd_ex(p: S2AttnParams, stream=None) -> None:
    _check(lib().s2attn_fwd_ex(ctypes.byref(p), _stream(stream)))


def s2attn_bwd_ex(p: S2AttnParams, stream=None) -> None:
    _check(lib().s2attn_bwd_ex(ctypes.byref(p), _stream(stream)))


STATIC_SCRATCH_BYTES = 16 << 20


def s2attn_bwd_ex_static(p: S2AttnParams, stream=None) -> None:
    """s2attn_bwd_ex on the library's static scratch array: no workspace, no allocation."""
    _check(lib().s2attn_bwd_ex_static(ctypes.byref(p), _stream(stream)))


def s2attn_bwd_ex_marked(p: S2AttnParams, events, stream=None) -> None:
    """events: sequence of four raw hipEvent_t handles (ints) or None entries."""
    arr = (ctypes.c_void_p * 4)(*[e if e else None for e in events])
    _check(lib().s2attn_bwd_ex_marked(ctypes.byref(p), _stream(stream), arr))


# ---- attention with a sliding window and sinks ----------------------------------------------------------------------

def _on_device(p):
    """The tensors of a parameter block lie on the current device, whose stream the call goes to."""
    device = getattr(p, "device", None)
    if device is None:       # a block of raw addresses
        return
    if device < 0:
        raise ValueError("the tensors are not on a GPU")
    current = _current_device()
    if current != device:
        raise ValueError(f"the tensors are on cuda:{device}, the current device is cuda:{current}")


def _whole(p):
    if p.tensors is not None:
        refs, strided = p.tensors
        tensors = [x() if isinstance(x, weakref.ref) else x for x in refs]
        tensors += [None] * (10 - len(tensors))   # (a forward's has no gradients)
        if tensors[0] is not None:
            p.device, p.problem = _device_of(tensors[0]), _problem_of(*tensors, (p.B, p.N, p.H, p.Hkv, p.D), strided)
        p.tensors = None
    if p.problem:
        raise ValueError(p.problem)
    _on_device(p)


def check_window_args(p: S2AttnParams, window: int, sinks: int, backward: bool) -> int:
    return int(lib().s2attn_check_window_args(ctypes.byref(p), window, sinks, 1 if backward else 0))


def window_workspace_bytes(p: S2AttnParams, window: int, sinks: int = 0) -> int:
    """Workspace of s2attn_window_bwd for a parameter block."""
    return int(lib().s2attn_window_workspace_bytes(ctypes.byref(p), window, sinks))


def s2attn_window_fwd(p: S2AttnParams, window: int, sinks: int = 0, stream=None) -> None:
    """o, lse <- causal attention over the last `window` tokens and the first `sinks`; p from make_params, whose G and
    shift options are not read (pass G = 0)."""
    _whole(p)
    code = (_lib or lib()).s2attn_window_fwd(ctypes.byref(p), window, sinks, _stream(stream))
    if code:
        _check(code)


def s2attn_window_bwd(p: S2AttnParams, window: int, sinks: int = 0, stream=None) -> None:
    """dq, dk, dv <- gradients of sum(o * dout) of s2attn_window_fwd."""
    _whole(p)
    code = (_lib or lib()).s2attn_window_bwd(ctypes.byref(p), window, sinks, _stream(stream))
    if code:
        _check(code)


# ---- paged cache ----------------------------------------------------------------------------------------------------

def _strided(t, n, name):
    """Address and strides of the first n axes; the last axis is contiguous."""
    if t.dim() != n + 1:
        raise ValueError(f"{name} must have {n + 1} axes")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    if not any(t.stride()[:n]) and max(t.shape[:n]) > 1:   # all zero stands for contiguous
        raise ValueError(f"{name} is one row, expanded")
    return t.data_ptr(), (ctypes.c_longlong * n)(*t.stride()[:n])


def _cache_dtype_code(t) -> int:
    torch = _torch or _import_torch()
    return E4M3 if t.dtype == torch.float8_e4m3fn else _dtype_code(t)


def make_paged_params(row_start, kv_len, page_table, k_cache, v_cache, k_exp=None, v_exp=None, q=None, o=None, lse=None,
                      k=None, v=None, workspace=None, window=0, sinks=0, max_kv=0, scale=0.0) -> S2AttnPagedParams:
    """Parameter block of the paged cache's calls: q, o (and lse) for s2attn_paged_fwd, k, v for s2attn_cache_write and
    s2attn_cache_read, or all of them where their rows are the same.

    row_start (B + 1), kv_len (B), page_table (B, columns): int32.  k_cache, v_cache: (pages, page_size, Hkv, D) views of any
    strides with a contiguous last axis; torch.float8_e4m3fn takes k_exp and v_exp, uint8 (pages, page_size, Hkv).  q (T, H, D)
    and k, v (T, Hkv, D) may be strided views, o (T, H, D) and lse (H, T) are contiguous.  The tensors must outlive the block."""
    torch = _torch or _import_torch()
    p = S2AttnPagedParams()
    if q is None and k is None:
        raise ValueError("q and o, or k and v, are needed")
    tensors = [t for t in (row_start, kv_len, page_table, k_cache, v_cache, k_exp, v_exp, q, o, lse, k, v, workspace) if t is not None]
    p.device = _device_of(k_cache)
    if any(t.device != k_cache.device for t in tensors):
        raise ValueError("all tensors must be on one device")
    for name, t, n in (("row_start", row_start, 1), ("kv_len", kv_len, 1), ("page_table", page_table, 2)):
        if t.dtype != torch.int32 or t.dim() != n or (t.shape[-1] > 1 and t.stride(-1) != 1):
            raise ValueError(f"{name} must be int32 with {n} axes, the last contiguous")
    p.B = kv_len.shape[0]
    if row_start.shape[0] != p.B + 1 or page_table.shape[0] != p.B:
        raise ValueError("row_start must have B + 1 entries, page_table B rows")
    if p.B > 1 and page_table.stride(0) == 0:    # zero stands for contiguous
        raise ValueError("page_table is one row, expanded")
    p.pages, p.page_size, p.Hkv, p.D = k_cache.shape
    if v_cache.shape != k_cache.shape or v_cache.dtype != k_cache.dtype:
        raise ValueError("k_cache and v_cache must have one shape and type")
    p.cache_dtype = _cache_dtype_code(k_cache)
    p.page_table, p.row_start, p.kv_len = page_table.data_ptr(), row_start.data_ptr(), kv_len.data_ptr()
    p.table_cols, p.table_stride = page_table.shape[1], max(page_table.stride(0), 1)
    p.k_cache, p.k_cache_strides = _strided(k_cache, 3, "k_cache")
    p.v_cache, p.v_cache_strides = _strided(v_cache, 3, "v_cache")
    if p.cache_dtype == E4M3:
        for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
            if t is None or t.dtype != torch.uint8 or t.shape != k_cache.shape[:3] or (not any(t.stride()) and t.numel() > 1):
                raise ValueError(f"{name} must be uint8 (pages, page_size, Hkv) for an e4m3 cache")
        p.k_exp, p.v_exp = k_exp.data_ptr(), v_exp.data_ptr()
        p.k_exp_strides = (ctypes.c_longlong * 3)(*k_exp.stride())
        p.v_exp_strides = (ctypes.c_longlong * 3)(*v_exp.stride())
    elif k_exp is not None or v_exp is not None:
        raise ValueError("exponents belong to an e4m3 cache")
    rows = q if q is not None else k
    p.T, p.dtype = rows.shape[0], _dtype_code(rows)
    if (k is None) != (v is None) or (q is None) != (o is None):
        raise ValueError("k and v, q and o go together")
    p.H = p.Hkv if q is None else q.shape[1]
    if q is not None:
        p.q, p.q_strides = _strided(q, 2, "q")
        if q.shape[2] != p.D or o.shape != q.shape or o.dtype != q.dtype or not o.is_contiguous():
            raise ValueError("q and o must be (T, H, D) of one type, o contiguous")
        p.o = o.data_ptr()
        if lse is not None:
            if lse.dtype != torch.float32 or lse.shape != (p.H, p.T) or not lse.is_contiguous():
                raise ValueError("lse must be a contiguous float32 (H, T)")
            p.lse = lse.data_ptr()
    if k is not None:
        for name, t in (("k", k), ("v", v)):
            if t.shape != (p.T, p.Hkv, p.D) or t.dtype != rows.dtype:
                raise ValueError("k and v must be (T, Hkv, D) of the rows' type")
            at, strides = _strided(t, 2, name)
            setattr(p, name, at)
            setattr(p, name + "_strides", strides)
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        p.workspace, p.workspace_bytes = workspace.data_ptr() or None, workspace.numel() * workspace.element_size()
    p.window, p.sinks, p.max_kv, p.scale = window, sinks, max_kv, scale
    return p


def check_paged_args(p: S2AttnPagedParams, call: int) -> int:
    return int(lib().s2attn_check_paged_args(ctypes.byref(p), call))


def paged_workspace_bytes(p: S2AttnPagedParams) -> int:
    """Workspace s2attn_paged_fwd wants for a parameter block (0: none); it runs with less."""
    return int(lib().s2attn_paged_workspace_bytes(ctypes.byref(p)))


def s2attn_cache_write(p: S2AttnPagedParams, stream=None) -> None:
    """k, v of the rows -> the cache."""
    _on_device(p)
    code = (_lib or lib()).s2attn_cache_write(ctypes.byref(p), _stream(stream))
    if code:
        _check(code)


def s2attn_cache_read(p: S2AttnPagedParams, stream=None) -> None:
    """The rows' positions of the cache -> k, v."""
    _on_device(p)
    code = (_lib or lib()).s2attn_cache_read(ctypes.byref(p), _stream(stream))
    if code:
        _check(code)


def s2attn_paged_fwd(p: S2AttnPagedParams, stream=None) -> None:
    """o (and lse) of the rows <- attention over the cache."""
    _on_device(p)
    code = (_lib or lib()).s2attn_paged_fwd(ctypes.byref(p), _stream(stream))
    if code:
        _check(code)
