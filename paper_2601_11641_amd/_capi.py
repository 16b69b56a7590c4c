"""ctypes binding of libmoddit.so with the C names (argument marshalling only).

Tensors are passed as device pointers (``tensor.data_ptr()``); every step of
the path runs in the HIP kernels of the library.  The stream defaults to
torch's current stream on the current device.  A non-zero status raises
ModError with the library's message.  Importing fails loudly when the
library has not been built.
"""
from __future__ import annotations

import ctypes
import math
import os
from ctypes import POINTER, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoddit.so")

MOD_OK = 0
MOD_ERR_INVALID_ARG = 1
MOD_ERR_UNSUPPORTED = 2
MOD_ERR_BAD_STATE = 3
MOD_ERR_HIP = 4
MOD_ERR_NOMEM = 5
MOD_BUDGET_TOPK = 0
MOD_BUDGET_MASS = 1
MOD_BUDGET_PATTERN = 2
MOD_ROPE_ADJACENT = 0
MOD_ROPE_HALVES = 1
MOD_CACHE_E4M3 = 0
MOD_CACHE_INT8 = 1


class ModError(RuntimeError):
    def __init__(self, status: int, func: str, msg: str):
        super().__init__(f"{func}: {_status_name(status)}: {msg}")
        self.status = status


class mod_shape(ctypes.Structure):
    _fields_ = [("B", c_int), ("H", c_int), ("L", c_int), ("d", c_int), ("block", c_int),
                ("frame_tokens", c_int), ("text_tokens", c_int)]


class mod_params(ctypes.Structure):
    _fields_ = [("warmup_m", c_int), ("delta_t", c_int), ("tau_e", c_float),
                ("anchor_rule", c_int), ("statistic", c_int), ("eta", c_float)]


class mod_budget(ctypes.Structure):
    _fields_ = [("mode", c_int), ("density", c_float), ("mass", c_float), ("patterns", c_int)]


class mod_strides(ctypes.Structure):
    _fields_ = [("b", c_int64), ("h", c_int64), ("l", c_int64)]


class mod_rope_params(ctypes.Structure):
    _fields_ = [("d", c_int), ("dims", c_int * 3), ("frames", c_int), ("height", c_int), ("width", c_int),
                ("theta", c_double), ("pairing", c_int)]


class mod_cache_shape(ctypes.Structure):
    _fields_ = [("B", c_int), ("H", c_int), ("capacity", c_int), ("d", c_int), ("block", c_int),
                ("format", c_int)]


class mod_cache(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("k_scale", c_void_p), ("v_scale", c_void_p)]
    made = None   # of tensors: their device, shapes and addresses (make_cache),
    fits = None   # and the cache shape that they were found to have (0.4 us instead of 1.4)


# torch bundles its own HIP runtime (SONAME libamdhip64.so.7).  Loading torch
# first makes the dynamic loader bind this library to that same runtime
# instead of mapping a second one from /opt/rocm into the process.
try:
    import torch  # noqa: F401
except ImportError:  # pragma: no cover - torch is optional for the ABI itself
    torch = None

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                      "(or python paper_2601_11641_amd/build_lib.py)")
_lib = ctypes.CDLL(LIB_PATH)

_SIGS = {
    "mod_num_blocks": (c_int, [POINTER(mod_shape)]),
    "mod_num_coeffs": (c_int, [POINTER(mod_shape)]),
    "mod_stats_create": (c_int, [POINTER(mod_shape), POINTER(mod_params), POINTER(c_void_p)]),
    "mod_stats_destroy": (c_int, [c_void_p]),
    "mod_collect_stats": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p]),
    "mod_update_stats": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int,
                                 c_void_p]),
    "mod_predict_block_mask": (c_int, [c_void_p, c_void_p, c_void_p, c_int, POINTER(mod_budget),
                                       c_void_p, c_void_p, c_void_p]),
    "mod_attn_workspace_bytes": (c_size_t, [POINTER(mod_shape)]),
    "mod_attn_plan_bytes": (c_size_t, [POINTER(mod_shape)]),
    "mod_block_sparse_attn_fwd": (c_int, [POINTER(mod_shape), c_void_p, c_void_p, c_void_p,
                                          c_void_p, c_void_p, c_float, c_void_p, c_void_p,
                                          c_void_p, c_size_t, c_void_p]),
    "mod_block_sparse_attn_fwd_noalloc": (c_int, [POINTER(mod_shape), c_void_p, c_void_p, c_void_p,
                                                  c_void_p, c_void_p, c_float, c_void_p, c_void_p,
                                                  c_void_p]),
    "mod_rope_create": (c_int, [POINTER(mod_rope_params), POINTER(c_void_p)]),
    "mod_rope_destroy": (c_int, [c_void_p]),
    "mod_rope_fwd": (c_int, [c_void_p, POINTER(mod_shape), c_void_p, POINTER(mod_strides), c_void_p,
                             POINTER(mod_strides), c_int, c_void_p, c_void_p]),
    "mod_rope_bwd": (c_int, [c_void_p, POINTER(mod_shape), c_void_p, POINTER(mod_strides), c_void_p,
                             POINTER(mod_strides), c_int, c_void_p, c_void_p]),
    "mod_cache_blocks": (c_int, [POINTER(mod_cache_shape)]),
    "mod_cache_write": (c_int, [POINTER(mod_cache_shape), POINTER(mod_cache), c_void_p, POINTER(mod_strides),
                                c_void_p, POINTER(mod_strides), c_int, c_int, c_void_p, c_void_p, c_void_p]),
    "mod_cache_read": (c_int, [POINTER(mod_cache_shape), POINTER(mod_cache), c_void_p, POINTER(mod_strides),
                               c_void_p, POINTER(mod_strides), c_int, c_int, c_void_p, c_void_p, c_void_p]),
    "mod_cache_attn_workspace_bytes": (c_size_t, [POINTER(mod_cache_shape), c_int, c_int, c_int]),
    "mod_cache_attn_plan": (c_int, [POINTER(mod_cache_shape), c_int, c_int, c_int, c_int, POINTER(c_int),
                                    POINTER(c_int)]),
    "mod_cache_attn_fwd": (c_int, [POINTER(mod_cache_shape), POINTER(mod_cache), c_void_p, c_int, c_int, c_int,
                                   c_void_p, c_void_p, c_void_p, c_float, c_void_p, c_void_p, c_void_p, c_size_t,
                                   c_void_p]),
    "mod_stats_get_anchor": (c_int, [c_void_p, c_int, POINTER(c_double), POINTER(c_int)]),
    "mod_stats_get_pooled": (c_int, [c_void_p, POINTER(c_double), POINTER(c_double)]),
    "mod_stats_get_block_mass": (c_int, [c_void_p, POINTER(c_double)]),
    "mod_stats_get_prediction": (c_int, [c_void_p, POINTER(c_double)]),
    "mod_stats_get_gate": (c_int, [c_void_p, POINTER(c_int32)]),
    "mod_status_string": (ctypes.c_char_p, [c_int]),
    "mod_last_error": (ctypes.c_char_p, []),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTED = tuple(_SIGS)


# the current stream's address without a stream object (0.1 us instead of 2.7)
_current_raw_stream = getattr(getattr(torch, "_C", None), "_cuda_getCurrentRawStream", None)
# the current device once a device tensor exists (0.07 us instead of 0.23)
_current_device = getattr(getattr(torch, "_C", None), "_cuda_getDevice", None) or (lambda: torch.cuda.current_device())


def _status_name(st: int) -> str:
    return _lib.mod_status_string(st).decode()


def _check(st: int, func: str):
    if st != MOD_OK:
        raise ModError(st, func, _lib.mod_last_error().decode())


def _ptr(x, what: str, dtype=None):
    """Device pointer of a tensor (checked contiguous / dtype), an int, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        if not x.is_contiguous():
            raise ValueError(f"{what} must be contiguous")
        if dtype is not None and str(x.dtype) != dtype:
            raise ValueError(f"{what} must be {dtype}, got {x.dtype}")
        if not x.is_cuda:
            raise ValueError(f"{what} must be a device tensor")
        return x.data_ptr()
    raise TypeError(f"{what}: unsupported argument type {type(x)}")


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    if _current_raw_stream is not None:
        return _current_raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _stream_beside(x, stream):
    """_stream in a call whose tensor x has passed _device (0.16 us less)."""
    if stream is None and _current_raw_stream is not None and not isinstance(x, int):
        return _current_raw_stream(_current_device())
    return _stream(stream)


def make_shape(B, H, L, d, block, frame_tokens=0, text_tokens=0) -> mod_shape:
    return mod_shape(B, H, L, d, block, frame_tokens, text_tokens)


def num_video_blocks(shape: mod_shape) -> int:
    """nv: the blocks of the video tokens, over which the MOD model and the
    introspection arrays are sized."""
    return -(-(shape.L - shape.text_tokens) // shape.block)


def make_params(warmup_m=1, delta_t=0, tau_e=0.0, anchor_rule=0, statistic=0, eta=1e-4) -> mod_params:
    s = {"pooled": 0, "attention": 1}.get(statistic, statistic)
    return mod_params(warmup_m, delta_t, tau_e, anchor_rule, int(s), eta)


def make_budget(mode="topk", density=1.0, mass=1.0, patterns=1) -> mod_budget:
    m = {"topk": MOD_BUDGET_TOPK, "mass": MOD_BUDGET_MASS, "pattern": MOD_BUDGET_PATTERN}.get(mode, mode)
    return mod_budget(int(m), density, mass, int(patterns))


# ---------------------------------------------------------------- entry points

def _ref(x):
    return None if x is None else ctypes.byref(x)


def mod_num_blocks(shape: mod_shape) -> int:
    return _lib.mod_num_blocks(_ref(shape))


def mod_num_coeffs(shape: mod_shape) -> int:
    return _lib.mod_num_coeffs(_ref(shape))


def mod_stats_create(shape: mod_shape, params: mod_params) -> int:
    h = c_void_p()
    _check(_lib.mod_stats_create(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(h)),
           "mod_stats_create")
    return h.value


def mod_stats_destroy(stats) -> None:
    _check(_lib.mod_stats_destroy(stats), "mod_stats_destroy")


def mod_collect_stats(stats, q, k, step: int, stream=None) -> None:
    _check(_lib.mod_collect_stats(stats, _ptr(q, "q", "torch.bfloat16"),
                                  _ptr(k, "k", "torch.bfloat16"), step, _stream(stream)),
           "mod_collect_stats")


def mod_update_stats(stats, q, k, lse, kv_idx, kv_cnt, step: int, stream=None) -> None:
    _check(_lib.mod_update_stats(stats, _ptr(q, "q", "torch.bfloat16"), _ptr(k, "k", "torch.bfloat16"),
                                 _ptr(lse, "lse", "torch.float32"), _ptr(kv_idx, "kv_idx", "torch.int32"),
                                 _ptr(kv_cnt, "kv_cnt", "torch.int32"), step, _stream(stream)),
           "mod_update_stats")


def mod_predict_block_mask(stats, q, k, step: int, budget: mod_budget, kv_idx, kv_cnt,
                           stream=None) -> None:
    _check(_lib.mod_predict_block_mask(stats, _ptr(q, "q", "torch.bfloat16"),
                                       _ptr(k, "k", "torch.bfloat16"), step,
                                       ctypes.byref(budget), _ptr(kv_idx, "kv_idx", "torch.int32"),
                                       _ptr(kv_cnt, "kv_cnt", "torch.int32"), _stream(stream)),
           "mod_predict_block_mask")


def mod_attn_workspace_bytes(shape: mod_shape) -> int:
    return int(_lib.mod_attn_workspace_bytes(_ref(shape)))


def mod_attn_plan_bytes(shape: mod_shape) -> int:
    return int(_lib.mod_attn_plan_bytes(_ref(shape)))


def mod_block_sparse_attn_fwd(shape: mod_shape, q, k, v, kv_idx, kv_cnt, scale: float, o,
                              lse=None, workspace=None, ws_bytes: int = 0, stream=None) -> None:
    """workspace=None: a device buffer of mod_attn_workspace_bytes(shape)
    bytes is allocated for the call (pass one to keep allocations out of a
    loop)."""
    if workspace is None and hasattr(q, "device"):
        ws_bytes = mod_attn_workspace_bytes(shape)
        workspace = torch.empty(max(ws_bytes, 1), dtype=torch.uint8, device=q.device)
    _check(_lib.mod_block_sparse_attn_fwd(
        ctypes.byref(shape), _ptr(q, "q", "torch.bfloat16"), _ptr(k, "k", "torch.bfloat16"),
        _ptr(v, "v", "torch.bfloat16"), _ptr(kv_idx, "kv_idx", "torch.int32"),
        _ptr(kv_cnt, "kv_cnt", "torch.int32"), float(scale), _ptr(o, "o", "torch.bfloat16"),
        _ptr(lse, "lse", "torch.float32"), _ptr(workspace, "workspace"), ws_bytes,
        _stream(stream)), "mod_block_sparse_attn_fwd")


MOD_ATTN_NOALLOC_MAX_BYTES = 2 << 20


def mod_block_sparse_attn_fwd_noalloc(shape: mod_shape, q, k, v, kv_idx, kv_cnt, scale: float, o,
                                      lse=None, stream=None) -> None:
    """The attention forward with its work plan in the library's own device
    array (no workspace, no allocation in the library or here)."""
    _check(_lib.mod_block_sparse_attn_fwd_noalloc(
        ctypes.byref(shape), _ptr(q, "q", "torch.bfloat16"), _ptr(k, "k", "torch.bfloat16"),
        _ptr(v, "v", "torch.bfloat16"), _ptr(kv_idx, "kv_idx", "torch.int32"),
        _ptr(kv_cnt, "kv_cnt", "torch.int32"), float(scale), _ptr(o, "o", "torch.bfloat16"),
        _ptr(lse, "lse", "torch.float32"), _stream(stream)), "mod_block_sparse_attn_fwd_noalloc")


# ---------------------------------------------------------------- the cached layer

def _device(x, what: str):
    """The library launches on the current device: any other tensor is refused."""
    d = x.get_device()
    if d < 0:
        raise ValueError(f"{what} must be a device tensor")
    if d != _current_device():
        raise ValueError(f"{what} is on {x.device}, but the current device is cuda:{_current_device()}")


def _array(x, dims, dtype, what: str):
    """Address of a contiguous device tensor of that shape (None: any) and
    type, an int, or None."""
    if x is None or isinstance(x, int):
        return x
    if not hasattr(x, "data_ptr"):
        raise TypeError(f"{what}: unsupported argument type {type(x)}")
    if dims is not None and x.shape != dims:
        raise ValueError(f"{what} must have shape {tuple(dims)}, got {tuple(x.shape)}")
    if dtype is not None and x.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, got {x.dtype}")
    if not x.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    _device(x, what)
    return x.data_ptr()


def _strided(x, dims, what: str):
    """Pointer and strides of a [B, H, L, d] bf16 tensor whose channels are
    contiguous (an int: the address of a contiguous one)."""
    if x is None or isinstance(x, int):
        return x, None
    if not hasattr(x, "data_ptr"):
        raise TypeError(f"{what}: unsupported argument type {type(x)}")
    if x.shape != dims:
        raise ValueError(f"{what} must have shape {tuple(dims)}, got {tuple(x.shape)}")
    if x.dtype is not torch.bfloat16:
        raise ValueError(f"{what} must be torch.bfloat16, got {x.dtype}")
    _device(x, what)
    if x.is_contiguous():
        return x.data_ptr(), None
    b, h, t, c = x.stride()
    if c != 1:
        raise ValueError(f"{what} must have contiguous channels")
    # the stride of an axis of one entry is of no account
    return x.data_ptr(), ctypes.byref(mod_strides(b if dims[0] > 1 else 0, h if dims[1] > 1 else 0,
                                                  t if dims[2] > 1 else 0))


def make_rope_params(d, dims, grid, theta=10000.0, pairing="adjacent") -> mod_rope_params:
    """dims: channels per axis, grid: positions per axis (time, height, width)."""
    m = {"adjacent": MOD_ROPE_ADJACENT, "halves": MOD_ROPE_HALVES}.get(pairing, pairing)
    return mod_rope_params(d, (c_int * 3)(*dims), *grid, theta, int(m))


def make_cache_shape(B, H, capacity, d, block, format="e4m3") -> mod_cache_shape:
    f = {"e4m3": MOD_CACHE_E4M3, "int8": MOD_CACHE_INT8}.get(format, format)
    return mod_cache_shape(B, H, capacity, d, block, int(f))


def make_cache(k, v, k_scale, v_scale) -> mod_cache:
    """The cache in these tensors (codes [B, H, capacity, d] of one byte, fp32
    scales [B, H, n]; with other numbers of axes as many elements, with one axis
    at least as many), which the caller keeps alive: the struct holds their
    addresses.  The calls refuse a cache shape that its tensors do not have."""
    for x, what in ((k, "k"), (v, "v")):
        if hasattr(x, "element_size") and x.element_size() != 1:
            raise ValueError(f"{what} must have one byte per code, got {x.dtype}")
    tensors = (k, v, k_scale, v_scale)
    at = [_array(x, None, t, what) for x, t, what in zip(tensors, (None, None, torch.float32, torch.float32),
                                                         ("k", "v", "k_scale", "v_scale"))]
    c = mod_cache(*at)
    shapes = [tuple(x.shape) if hasattr(x, "shape") else None for x in tensors]
    devices = {x.get_device() for x in tensors if hasattr(x, "get_device")}
    if devices:
        c.made = (devices.pop(), shapes, at)
    return c


def _check_cache(shape, cache):
    """Refuse a cache of other sizes than the shape says, or of another device
    (addresses are taken as they are)."""
    made = cache.made
    if made is None:
        return
    device, shapes, at = made
    if device != _current_device():
        raise ValueError(f"the cache is on cuda:{device}, but the current device is cuda:{_current_device()}")
    if cache.fits == bytes(shape):
        return
    codes = (shape.B, shape.H, shape.capacity, shape.d)
    scales = (shape.B, shape.H, -(-shape.capacity // max(1, shape.block)))
    for name, got, address, want in zip(("k", "v", "k_scale", "v_scale"), shapes, at, (codes, codes, scales, scales)):
        if got is None or got == want or getattr(cache, name) != address:
            continue
        held, needed = math.prod(got), math.prod(want)
        if len(got) == len(want) or held < needed or (held > needed and len(got) > 1):
            raise ValueError(f"the cache's {name} has shape {got}, the cache shape says {want}")
    cache.fits = bytes(shape)


def mod_rope_create(params: mod_rope_params) -> int:
    h = c_void_p()
    _check(_lib.mod_rope_create(_ref(params), ctypes.byref(h)), "mod_rope_create")
    return h.value


def mod_rope_destroy(rope) -> None:
    _check(_lib.mod_rope_destroy(rope), "mod_rope_destroy")


def _rope_call(name, rope, shape, x, y, first, starts, stream):
    dims = (shape.B, shape.H, shape.L, shape.d)
    src, dst = ("x", "y") if name == "mod_rope_fwd" else ("dy", "dx")
    xp, xs = _strided(x, dims, src)
    yp, ys = _strided(y, dims, dst)
    _check(getattr(_lib, name)(rope, ctypes.byref(shape), xp, xs, yp, ys, first,
                               _array(starts, (shape.B,), torch.int32, "starts"), _stream(stream)), name)


def mod_rope_fwd(rope, shape: mod_shape, x, y, first: int = 0, starts=None, stream=None) -> None:
    """y = R x.  x and y: [B, H, L, d] tensors with any strides over the first
    three axes (a transposed view of a projection's output, say)."""
    _rope_call("mod_rope_fwd", rope, shape, x, y, first, starts, stream)


def mod_rope_bwd(rope, shape: mod_shape, dy, dx, first: int = 0, starts=None, stream=None) -> None:
    """dx = R^T dy, the gradient of mod_rope_fwd."""
    _rope_call("mod_rope_bwd", rope, shape, dy, dx, first, starts, stream)


def mod_cache_blocks(shape: mod_cache_shape) -> int:
    return _lib.mod_cache_blocks(_ref(shape))


def _store_call(name, shape, cache, k, v, first, starts, counts, L, stream):
    x = k if k is not None else v
    if L is None:
        size = getattr(x, "shape", None)
        if x is not None and size is None:
            raise TypeError("L is needed where k and v are addresses")
        L = size[2] if size is not None and len(size) == 4 else 1
    dims = (shape.B, shape.H, L, shape.d)
    _check_cache(shape, cache)
    kp, ks = _strided(k, dims, "k")
    vp, vs = _strided(v, dims, "v")
    if starts is not None:
        starts = _array(starts, (shape.B,), torch.int32, "starts")
    if counts is not None:
        counts = _array(counts, (shape.B,), torch.int32, "counts")
    _check(getattr(_lib, name)(ctypes.byref(shape), ctypes.byref(cache), kp, ks, vp, vs, L, first, starts, counts,
                               _stream(stream) if x is None else _stream_beside(x, stream)), name)


def mod_cache_write(shape: mod_cache_shape, cache: mod_cache, k, v, first: int = 0, starts=None, counts=None, L=None,
                    stream=None) -> None:
    """Quantise k and v ([B, H, L, d] bf16, any strides over the first three
    axes; L is needed only with addresses) into the cache."""
    _store_call("mod_cache_write", shape, cache, k, v, first, starts, counts, L, stream)


def mod_cache_read(shape: mod_cache_shape, cache: mod_cache, k, v, first: int = 0, starts=None, counts=None, L=None,
                   stream=None) -> None:
    """What the cache holds at those positions into k and v (either may be None)."""
    _store_call("mod_cache_read", shape, cache, k, v, first, starts, counts, L, stream)


def mod_cache_attn_workspace_bytes(shape: mod_cache_shape, Hq: int, Lq: int, max_len: int) -> int:
    return int(_lib.mod_cache_attn_workspace_bytes(_ref(shape), Hq, Lq, max_len))


def mod_cache_attn_plan(shape: mod_cache_shape, Hq: int, Lq: int, max_len: int, lists: bool = False):
    """(rows of a tile, parts of a walk) of such a call."""
    rows, parts = c_int(), c_int()
    _check(_lib.mod_cache_attn_plan(_ref(shape), Hq, Lq, max_len, int(bool(lists)), ctypes.byref(rows),
                                    ctypes.byref(parts)), "mod_cache_attn_plan")
    return rows.value, parts.value


def mod_cache_attn_fwd(shape: mod_cache_shape, cache: mod_cache, q, max_len: int, kv_len, kv_idx, kv_cnt,
                       scale: float, o, lse=None, workspace=None, ws_bytes: int = 0, stream=None, Hq=None,
                       Lq=None) -> None:
    """q, o: contiguous [B, Hq, Lq, d] (with addresses, pass Hq and Lq).
    workspace=None: a device buffer is allocated for the call (pass one to
    keep allocations out of a loop)."""
    if hasattr(q, "shape"):
        if q.dim() != 4 or q.shape[0] != shape.B or q.shape[3] != shape.d:
            raise ValueError(f"q must have shape ({shape.B}, Hq, Lq, {shape.d}), got {tuple(q.shape)}")
        Hq, Lq = q.shape[1], q.shape[2]
    elif Hq is None or Lq is None:
        raise TypeError("Hq and Lq are needed where q is an address")
    _check_cache(shape, cache)
    B, bf16, i32 = shape.B, torch.bfloat16, torch.int32
    if kv_idx is not None or kv_cnt is not None:
        block = max(1, shape.block)
        n, nq = -(-max_len // block), -(-Lq // block)
        kv_idx, kv_cnt = _array(kv_idx, (B, Hq, nq, n), i32, "kv_idx"), _array(kv_cnt, (B, Hq, nq), i32, "kv_cnt")
    if kv_len is not None:
        kv_len = _array(kv_len, (B,), i32, "kv_len")
    args = (_array(q, None, bf16, "q"), Hq, Lq, max_len, kv_len, kv_idx, kv_cnt, float(scale),
            _array(o, (B, Hq, Lq, shape.d), bf16, "o"), _array(lse, (B, Hq, Lq), torch.float32, "lse"))
    st = _stream_beside(q, stream)
    if workspace is None and hasattr(q, "device"):
        ws_bytes = mod_cache_attn_workspace_bytes(shape, Hq, Lq, max_len)
        if ws_bytes > 0:
            if st == _stream(None):
                workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device)
            else:   # of the stream that uses it: nothing else does before or after in another order
                # (address 0, the default stream, would make an ExternalStream some other one)
                with torch.cuda.stream(torch.cuda.ExternalStream(st) if st else torch.cuda.default_stream()):
                    workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device)
    elif hasattr(workspace, "nbytes") and workspace.nbytes < ws_bytes:
        raise ValueError(f"workspace has {workspace.nbytes} bytes, ws_bytes says {ws_bytes}")
    _check(_lib.mod_cache_attn_fwd(ctypes.byref(shape), ctypes.byref(cache), *args,
                                   _array(workspace, None, None, "workspace"), ws_bytes, st), "mod_cache_attn_fwd")


def _dbl(n):
    a = np.empty(n, dtype=np.float64)
    return a, a.ctypes.data_as(POINTER(c_double))


def mod_stats_get_anchor(stats, slot: int, B: int, H: int, p: int):
    a, ptr = _dbl(B * H * p)
    step = c_int()
    _check(_lib.mod_stats_get_anchor(stats, slot, ptr, ctypes.byref(step)), "mod_stats_get_anchor")
    return a.reshape(B, H, p), step.value


def mod_stats_get_pooled(stats, B: int, H: int, n: int, d: int):
    qa, qp = _dbl(B * H * n * d)
    ka, kp = _dbl(B * H * n * d)
    _check(_lib.mod_stats_get_pooled(stats, qp, kp), "mod_stats_get_pooled")
    return qa.reshape(B, H, n, d), ka.reshape(B, H, n, d)


def mod_stats_get_block_mass(stats, B: int, H: int, n: int):
    a, ptr = _dbl(B * H * n * n)
    _check(_lib.mod_stats_get_block_mass(stats, ptr), "mod_stats_get_block_mass")
    return a.reshape(B, H, n, n)


def mod_stats_get_prediction(stats, B: int, H: int, n: int):
    a, ptr = _dbl(B * H * (3 * n - 1))
    _check(_lib.mod_stats_get_prediction(stats, ptr), "mod_stats_get_prediction")
    return a.reshape(B, H, 3 * n - 1)


def mod_stats_get_gate(stats, B: int, H: int):
    a = np.empty(B * H, dtype=np.int32)
    _check(_lib.mod_stats_get_gate(stats, a.ctypes.data_as(POINTER(c_int32))),
           "mod_stats_get_gate")
    return a.reshape(B, H)


def mod_status_string(status: int) -> str:
    return _status_name(status)


def mod_last_error() -> str:
    return _lib.mod_last_error().decode()


def raw_lib():
    """The loaded ctypes library (for status-code tests)."""
    return _lib


class Stats:
    """Owner of a mod_stats handle (destroyed on close / garbage collection)."""

    def __init__(self, shape: mod_shape, params: mod_params):
        self.shape, self.params = shape, params
        self.handle = mod_stats_create(shape, params)
        self.n = mod_num_blocks(shape)
        self.n_video = num_video_blocks(shape)
        self.p = mod_num_coeffs(shape)

    def close(self):
        if self.handle:
            mod_stats_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class Rope:
    """Owner of a mod_rope handle (destroyed on close / garbage collection)."""

    def __init__(self, params: mod_rope_params):
        self.handle = None
        self.params = params
        self.handle = mod_rope_create(params)

    def close(self):
        if self.handle:
            mod_rope_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class Cache:
    """The tensors of a cache and its descriptors: k, v [B, H, capacity, d]
    uint8, k_scale, v_scale [B, H, n] fp32, `ref` for the calls."""

    def __init__(self, shape: mod_cache_shape, device="cuda"):
        n = mod_cache_blocks(shape)
        if n == 0:
            raise ModError(MOD_ERR_INVALID_ARG, "mod_cache_blocks", mod_last_error())
        self.shape, self.n = shape, n
        codes = (shape.B, shape.H, shape.capacity, shape.d)
        self.k = torch.empty(codes, dtype=torch.uint8, device=device)
        self.v = torch.empty(codes, dtype=torch.uint8, device=device)
        self.k_scale = torch.empty((shape.B, shape.H, n), dtype=torch.float32, device=device)
        self.v_scale = torch.empty((shape.B, shape.H, n), dtype=torch.float32, device=device)
        self.ref = make_cache(self.k, self.v, self.k_scale, self.v_scale)
