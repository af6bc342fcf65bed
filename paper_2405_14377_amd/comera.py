"""Python binding of ``libcomera.so`` (the C ABI declared in include/comera.h).

Argument marshalling only: every function here has the name of the C entry
point it calls and passes device pointers, sizes and the stream straight
through.  Tensors (anything with ``data_ptr()``) are passed by pointer; plain
ints are taken as raw addresses.  The library must have been built (see
``build.py``); loading fails loudly otherwise -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcomera.so")

MAX_CORES = 8
F32, BF16 = 0, 1
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_INTERNAL = 0, -1, -2, -3, -4, -5
ORDER_DENSE, ORDER_SWEEP_RL, ORDER_SWEEP_LR, ORDER_ZERO, ORDER_FUSED_RL = 0, 1, 2, 3, 4

# every function declared in include/comera.h
EXPORTS = (
    "comera_ttm_plan", "comera_ttm_plan_num_orders", "comera_ttm_plan_chosen",
    "comera_ttm_plan_order_info", "comera_ttm_workspace_bytes", "comera_ttm_forward",
    "comera_ttm_backward", "comera_ttm_plan_destroy", "comera_tt_embed_workspace_bytes",
    "comera_tt_embed_forward", "comera_tt_embed_backward", "comera_status_string", "comera_last_hip_error",
    "comera_ttm_plan_set_timing", "comera_ttm_plan_kernel_time", "comera_ttm_plan_set_reuse_forward",
    "comera_ttm_backward_masks", "comera_tt_embed_backward_ex", "comera_ttm_plan_set_fp8", "comera_fp8_quantize",
    "comera_ttm_regularizer_grads", "comera_debug_launch_check", "comera_debug_launch_count",
    "comera_debug_launch_info", "comera_ttm_forward_noalloc",
    "comera_dense_embed_workspace_bytes", "comera_dense_embed_forward", "comera_dense_embed_backward",
    "comera_block_norm_workspace_bytes", "comera_block_norm_forward", "comera_block_norm_backward",
    "comera_grad_plan", "comera_grad_plan_destroy", "comera_grad_workspace_bytes", "comera_grad_norm",
    "comera_grad_clip", "comera_grad_table_bytes", "comera_grad_plan_set_table",
)
FP8_QUANTIZE_WS_BYTES = 2048
KERNEL_FWD, KERNEL_DX, KERNEL_DW = 0, 1, 2
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_NONE, GATE_CHANNEL, GATE_TOKEN = 0, 1, 2


class ComeraError(RuntimeError):
    def __init__(self, status: int, where: str):
        extra = f": {comera_last_hip_error()}" if status == ERR_HIP else ""
        super().__init__(f"{where}: status {status} ({comera_status_string(status)}){extra}")
        self.status = status


class comera_ttm_shape(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("act", ctypes.c_int32),
                ("n", ctypes.c_int64 * MAX_CORES), ("m", ctypes.c_int64 * MAX_CORES),
                ("r", ctypes.c_int64 * (MAX_CORES + 1))]


class comera_tt_embed_shape(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("pad_", ctypes.c_int32),
                ("v", ctypes.c_int64 * MAX_CORES), ("e", ctypes.c_int64 * MAX_CORES),
                ("r", ctypes.c_int64 * (MAX_CORES + 1))]


class comera_dense_embed_shape(ctypes.Structure):
    _fields_ = [("V", ctypes.c_int64), ("E", ctypes.c_int64), ("table", ctypes.c_int32), ("act", ctypes.c_int32)]


class comera_block_norm_shape(ctypes.Structure):
    _fields_ = [("width", ctypes.c_int64), ("stream", ctypes.c_int32), ("act", ctypes.c_int32),
                ("post", ctypes.c_int32), ("pre", ctypes.c_int32), ("gate", ctypes.c_int32), ("eps", ctypes.c_float),
                ("res_scale", ctypes.c_float), ("branch_scale", ctypes.c_float)]


class comera_grad_tensor(ctypes.Structure):
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("pad_", ctypes.c_int32)]


_lib = None
_torch = None          # torch, once load() has imported it (it may be missing: no tensors then, only addresses)
_f32 = _bf16 = _i32 = _i64 = None      # its types


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the library once; raise if it has not been built."""
    global _lib, _torch, _f32, _bf16, _i32, _i64
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with paper_2405_14377_amd/build.py "
                          "(the HIP library is required; there is no CPU fallback)")
    # One HIP runtime per process: torch ships its own libamdhip64 under a
    # different file name, so if this library were opened first the process
    # would end up with two runtimes and the second one finds no device.
    # Loading torch first makes this library bind to torch's runtime.
    try:
        import torch
        _torch = torch
        _f32, _bf16, _i32, _i64 = torch.float32, torch.bfloat16, torch.int32, torch.int64
    except ImportError:
        pass
    lib = ctypes.CDLL(path)
    vp, i32, i64, sz, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_double
    P = ctypes.POINTER
    lib.comera_ttm_plan.argtypes = [P(comera_ttm_shape), i64, vp, i32, P(vp)]
    lib.comera_ttm_plan.restype = i32
    lib.comera_ttm_plan_num_orders.argtypes = [vp]
    lib.comera_ttm_plan_num_orders.restype = i32
    lib.comera_ttm_plan_chosen.argtypes = [vp]
    lib.comera_ttm_plan_chosen.restype = i32
    lib.comera_ttm_plan_order_info.argtypes = [vp, i32, ctypes.c_char_p, sz, P(i32), P(dbl), P(dbl), P(dbl), P(i32)]
    lib.comera_ttm_plan_order_info.restype = i32
    lib.comera_ttm_workspace_bytes.argtypes = [vp]
    lib.comera_ttm_workspace_bytes.restype = sz
    lib.comera_ttm_forward.argtypes = [vp, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.comera_ttm_forward.restype = i32
    lib.comera_ttm_forward_noalloc.argtypes = [vp, i64, vp, vp, vp, vp, vp]
    lib.comera_ttm_forward_noalloc.restype = i32
    lib.comera_ttm_backward.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.comera_ttm_backward.restype = i32
    lib.comera_ttm_backward_masks.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.comera_ttm_backward_masks.restype = i32
    lib.comera_ttm_regularizer_grads.argtypes = [P(comera_ttm_shape), ctypes.c_float, ctypes.c_float, vp, vp, vp, vp,
                                                 vp]
    lib.comera_ttm_regularizer_grads.restype = i32
    lib.comera_ttm_plan_destroy.argtypes = [vp]
    lib.comera_ttm_plan_destroy.restype = None
    lib.comera_tt_embed_workspace_bytes.argtypes = [P(comera_tt_embed_shape), i64]
    lib.comera_tt_embed_workspace_bytes.restype = sz
    lib.comera_tt_embed_forward.argtypes = [P(comera_tt_embed_shape), vp, i64, vp, vp, vp, vp, sz, vp, vp]
    lib.comera_tt_embed_forward.restype = i32
    lib.comera_tt_embed_backward.argtypes = [P(comera_tt_embed_shape), vp, i64, vp, vp, vp, vp, i32, vp, sz, vp, vp]
    lib.comera_tt_embed_backward.restype = i32
    lib.comera_tt_embed_backward_ex.argtypes = [P(comera_tt_embed_shape), vp, i64, vp, vp, vp, vp, i32, vp, sz, vp,
                                                vp]
    lib.comera_tt_embed_backward_ex.restype = i32
    lib.comera_ttm_plan_set_timing.argtypes = [vp, i32]
    lib.comera_ttm_plan_set_reuse_forward.argtypes = [vp, i32]
    lib.comera_ttm_plan_set_reuse_forward.restype = i32
    lib.comera_ttm_plan_set_fp8.argtypes = [vp, i32]
    lib.comera_ttm_plan_set_fp8.restype = i32
    lib.comera_fp8_quantize.argtypes = [vp, i32, i64, i64, vp, i64, vp, i64, vp, vp, sz, vp]
    lib.comera_fp8_quantize.restype = i32
    lib.comera_ttm_plan_set_timing.restype = i32
    lib.comera_ttm_plan_kernel_time.argtypes = [vp, i32, P(dbl), P(i32)]
    lib.comera_ttm_plan_kernel_time.restype = i32
    f32 = ctypes.c_float
    lib.comera_dense_embed_workspace_bytes.argtypes = [P(comera_dense_embed_shape), i64]
    lib.comera_dense_embed_workspace_bytes.restype = sz
    lib.comera_dense_embed_forward.argtypes = [P(comera_dense_embed_shape), vp, i64, vp, f32, vp, vp, vp]
    lib.comera_dense_embed_forward.restype = i32
    lib.comera_dense_embed_backward.argtypes = [P(comera_dense_embed_shape), vp, i64, vp, f32, i64, vp, vp, sz, vp, vp]
    lib.comera_dense_embed_backward.restype = i32
    lib.comera_block_norm_workspace_bytes.argtypes = [P(comera_block_norm_shape), i64]
    lib.comera_block_norm_workspace_bytes.restype = sz
    lib.comera_block_norm_forward.argtypes = [P(comera_block_norm_shape), i64] + [vp] * 10
    lib.comera_block_norm_forward.restype = i32
    lib.comera_block_norm_backward.argtypes = [P(comera_block_norm_shape), i64] + [vp] * 16 + [sz, vp]
    lib.comera_block_norm_backward.restype = i32
    lib.comera_grad_plan.argtypes = [vp, i64, P(vp)]
    lib.comera_grad_plan.restype = i32
    lib.comera_grad_plan_destroy.argtypes = [vp]
    lib.comera_grad_plan_destroy.restype = None
    lib.comera_grad_table_bytes.argtypes = [vp]
    lib.comera_grad_table_bytes.restype = sz
    lib.comera_grad_plan_set_table.argtypes = [vp, vp, sz, vp]
    lib.comera_grad_plan_set_table.restype = i32
    lib.comera_grad_workspace_bytes.argtypes = [vp]
    lib.comera_grad_workspace_bytes.restype = sz
    lib.comera_grad_norm.argtypes = [vp, f32, vp, vp, vp, sz, vp]
    lib.comera_grad_norm.restype = i32
    lib.comera_grad_clip.argtypes = [vp, f32, f32, vp, vp, vp, sz, vp]
    lib.comera_grad_clip.restype = i32
    lib.comera_status_string.argtypes = [i32]
    lib.comera_status_string.restype = ctypes.c_char_p
    lib.comera_last_hip_error.argtypes = []
    lib.comera_last_hip_error.restype = ctypes.c_char_p
    lib.comera_debug_launch_check.argtypes = [i32]
    lib.comera_debug_launch_check.restype = i32
    lib.comera_debug_launch_count.argtypes = []
    lib.comera_debug_launch_count.restype = i32
    u32, u64 = ctypes.c_uint32, ctypes.c_uint64
    lib.comera_debug_launch_info.argtypes = [i32, ctypes.c_char_p, sz, P(u32), P(u32), P(u64), P(i32)]
    lib.comera_debug_launch_info.restype = i32
    _lib = lib
    return lib


# ------------------------------------------------------------------ marshalling helpers
def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return int(x.data_ptr())


def _ptr_array(xs: Optional[Sequence]):
    """Host array of device pointers (NULL entries allowed), or NULL."""
    if xs is None:
        return None
    arr = (ctypes.c_void_p * max(1, len(xs)))()
    for i, x in enumerate(xs):
        arr[i] = _ptr(x)
    return arr


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _torch is None:
            raise ImportError("the current stream is torch's: pass a stream")
        # the handle alone: building a Stream object costs 3 us a call
        return _torch._C._cuda_getCurrentRawStream(_torch._C._cuda_getDevice())
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)


def _nbytes(ws) -> int:
    if ws is None:
        return 0
    return int(ws.numel() * ws.element_size())


def _check(status: int, where: str) -> None:
    if status != OK:
        raise ComeraError(status, where)


def ttm_shape(n: Sequence[int], m: Sequence[int], r: Sequence[int], act: int = F32) -> comera_ttm_shape:
    s = comera_ttm_shape()
    s.d = len(n)
    s.act = act
    for k in range(len(n)):
        s.n[k] = int(n[k])
        s.m[k] = int(m[k])
    for k in range(len(r)):
        s.r[k] = int(r[k])
    return s


def tt_embed_shape(v: Sequence[int], e: Sequence[int], r: Sequence[int]) -> comera_tt_embed_shape:
    s = comera_tt_embed_shape()
    s.d = len(v)
    for k in range(len(v)):
        s.v[k] = int(v[k])
        s.e[k] = int(e[k])
    for k in range(len(r)):
        s.r[k] = int(r[k])
    return s


def dense_embed_shape(V: int, E: int, table: int = F32, act: int = F32) -> comera_dense_embed_shape:
    return comera_dense_embed_shape(int(V), int(E), int(table), int(act))


def block_norm_shape(width: int, stream: int = F32, act: int = F32, post: int = NORM_NONE, pre: int = NORM_RMS,
                     gate: int = GATE_NONE, eps: float = 1e-6, res_scale: float = 1.0,
                     branch_scale: float = 1.0) -> comera_block_norm_shape:
    return comera_block_norm_shape(int(width), int(stream), int(act), int(post), int(pre), int(gate), float(eps),
                                   float(res_scale), float(branch_scale))


# ------------------------------------------------------------------ tensor checks
# The calls around the compressed layers check the tensors that they are
# given (raw addresses are taken as they are, a workspace's or a table's with
# its bytes behind it: (address, bytes)): a tensor of another type, a
# strided view, one that is too short or lies on another device than the
# current one would be read wrongly or out of its bounds.
def _dtype_of(code: int):
    return _bf16 if code == BF16 else _f32


def _taken(where: str, *args) -> list:
    """Addresses of (tensor, torch dtype or None for any, entries) triples; None and raw addresses pass."""
    dev, out = None, []
    for t, dtype, n in args:
        if t is None or t.__class__ is int:
            out.append(t)
            continue
        at = t.get_device()
        if at != dev:
            if at < 0:
                raise ComeraError(ERR_INVALID_ARG, f"{where}: a tensor in host memory")
            dev = _torch.cuda.current_device()
            if at != dev:
                raise ComeraError(ERR_INVALID_ARG, f"{where}: a tensor on device {at}, the current device is {dev}")
        if t.dtype is not dtype and dtype is not None:
            raise ComeraError(ERR_INVALID_ARG, f"{where}: {t.dtype} where {dtype} is expected")
        if not t.is_contiguous():
            raise ComeraError(ERR_INVALID_ARG, f"{where}: a tensor that is not contiguous")
        if t.numel() < n:
            raise ComeraError(ERR_INVALID_ARG, f"{where}: {t.numel()} entries where {n} are expected")
        out.append(t.data_ptr())
    return out


def _workspace(where: str, ws):
    """(what _taken checks, bytes) of a workspace or a table: a tensor, an (address, bytes) pair or None."""
    if ws.__class__ is tuple:
        return ws[0], int(ws[1])
    if ws.__class__ is int:
        raise ComeraError(ERR_WORKSPACE, f"{where}: a workspace at a raw address is given as (address, bytes)")
    return ws, _nbytes(ws)


# ------------------------------------------------------------------ entry points
def comera_status_string(status: int) -> str:
    return load().comera_status_string(int(status)).decode()


def comera_last_hip_error() -> str:
    return load().comera_last_hip_error().decode()


def comera_ttm_plan(shape: comera_ttm_shape, batch: int, mask_active=None, force_order: int = -1,
                    raise_on_error: bool = True):
    """Returns a plan handle (int) or, with raise_on_error=False, (status, handle)."""
    lib = load()
    h = ctypes.c_void_p()
    buf = None
    if mask_active is not None:
        data = bytes(int(bool(x)) for x in mask_active)
        buf = ctypes.create_string_buffer(data, max(1, len(data)))
    st = lib.comera_ttm_plan(ctypes.byref(shape), int(batch), buf, int(force_order), ctypes.byref(h))
    if not raise_on_error:
        return st, h.value
    _check(st, "comera_ttm_plan")
    return h.value


def comera_ttm_plan_num_orders(plan) -> int:
    return int(load().comera_ttm_plan_num_orders(plan))


def comera_ttm_plan_chosen(plan) -> int:
    return int(load().comera_ttm_plan_chosen(plan))


def comera_ttm_plan_order_info(plan, i: int) -> dict:
    buf = ctypes.create_string_buffer(160)
    kind = ctypes.c_int32()
    ff, fb, by = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    ex = ctypes.c_int32()
    st = load().comera_ttm_plan_order_info(plan, int(i), buf, 160, ctypes.byref(kind), ctypes.byref(ff),
                                           ctypes.byref(fb), ctypes.byref(by), ctypes.byref(ex))
    _check(st, "comera_ttm_plan_order_info")
    return {"desc": buf.value.decode(), "kind": kind.value, "flops_fwd": ff.value, "flops_bwd": fb.value,
            "bytes": by.value, "executable": bool(ex.value)}


def comera_ttm_workspace_bytes(plan) -> int:
    return int(load().comera_ttm_workspace_bytes(plan))


def comera_ttm_forward(plan, b: int, X, G, D, Y, ws, stream=None) -> int:
    st = load().comera_ttm_forward(plan, int(b), _ptr(X), _ptr_array(G), _ptr_array(D), _ptr(Y), _ptr(ws),
                                   _nbytes(ws), _stream(stream))
    _check(st, "comera_ttm_forward")
    return st


def comera_ttm_forward_noalloc(plan, b: int, X, G, D, Y, stream=None, raise_on_error: bool = True) -> int:
    st = load().comera_ttm_forward_noalloc(plan, int(b), _ptr(X), _ptr_array(G), _ptr_array(D), _ptr(Y),
                                           _stream(stream))
    if raise_on_error:
        _check(st, "comera_ttm_forward_noalloc")
    return st


def comera_ttm_backward(plan, b: int, X, dY, G, D, dX, dG, ws, stream=None) -> int:
    st = load().comera_ttm_backward(plan, int(b), _ptr(X), _ptr(dY), _ptr_array(G), _ptr_array(D), _ptr(dX),
                                    _ptr_array(dG), _ptr(ws), _nbytes(ws), _stream(stream))
    _check(st, "comera_ttm_backward")
    return st


def comera_ttm_regularizer_grads(shape, gamma: float, beta: float, G, D, dG, dD, stream=None) -> int:
    """Add the early-stage regulariser gradients in place (eq. pretrain-rank):
    dG_k += 2 beta G_k, dD_k += gamma dS^/dD_k.  `shape` is a comera_ttm_shape;
    G, dG, D, dD are lists of device tensors (or None)."""
    st = load().comera_ttm_regularizer_grads(ctypes.byref(shape), float(gamma), float(beta), _ptr_array(G),
                                             _ptr_array(D), _ptr_array(dG), _ptr_array(dD), _stream(stream))
    _check(st, "comera_ttm_regularizer_grads")
    return st


def comera_ttm_backward_masks(plan, b: int, X, dY, G, D, dX, dG, dD, ws, stream=None) -> int:
    st = load().comera_ttm_backward_masks(plan, int(b), _ptr(X), _ptr(dY), _ptr_array(G), _ptr_array(D), _ptr(dX),
                                          _ptr_array(dG), _ptr_array(dD), _ptr(ws), _nbytes(ws), _stream(stream))
    _check(st, "comera_ttm_backward_masks")
    return st


def comera_ttm_plan_destroy(plan) -> None:
    if plan:
        load().comera_ttm_plan_destroy(plan)


def comera_ttm_plan_set_timing(plan, enable: bool) -> None:
    _check(load().comera_ttm_plan_set_timing(plan, int(bool(enable))), "comera_ttm_plan_set_timing")


def comera_ttm_plan_set_reuse_forward(plan, enable: bool) -> None:
    _check(load().comera_ttm_plan_set_reuse_forward(plan, int(bool(enable))), "comera_ttm_plan_set_reuse_forward")


def comera_ttm_plan_set_fp8(plan, enable: bool) -> None:
    _check(load().comera_ttm_plan_set_fp8(plan, int(bool(enable))), "comera_ttm_plan_set_fp8")


def comera_fp8_quantize(x, dtype: int, rows: int, cols: int, q, ldq: int, qt, ldt: int, scale, ws,
                        stream=None) -> int:
    st = load().comera_fp8_quantize(_ptr(x), int(dtype), int(rows), int(cols), _ptr(q), int(ldq), _ptr(qt), int(ldt),
                                    _ptr(scale), _ptr(ws), _nbytes(ws), _stream(stream))
    _check(st, "comera_fp8_quantize")
    return st


def comera_ttm_plan_kernel_time(plan, kernel: int):
    """(mean ms, launches) of one kernel since the last query; clears the record."""
    ms, cnt = ctypes.c_double(), ctypes.c_int32()
    _check(load().comera_ttm_plan_kernel_time(plan, int(kernel), ctypes.byref(ms), ctypes.byref(cnt)),
           "comera_ttm_plan_kernel_time")
    return ms.value, cnt.value


def comera_tt_embed_workspace_bytes(shape: comera_tt_embed_shape, n_tokens: int) -> int:
    return int(load().comera_tt_embed_workspace_bytes(ctypes.byref(shape), int(n_tokens)))


def comera_tt_embed_forward(shape, ids, n_tokens: int, G, D, Y, ws, err_flag=None, stream=None) -> int:
    st = load().comera_tt_embed_forward(ctypes.byref(shape), _ptr(ids), int(n_tokens), _ptr_array(G), _ptr_array(D),
                                        _ptr(Y), _ptr(ws), _nbytes(ws), _ptr(err_flag), _stream(stream))
    _check(st, "comera_tt_embed_forward")
    return st


def comera_tt_embed_backward(shape, ids, n_tokens: int, dY, G, D, dG, deterministic: int, ws, err_flag=None,
                             stream=None) -> int:
    st = load().comera_tt_embed_backward(ctypes.byref(shape), _ptr(ids), int(n_tokens), _ptr(dY), _ptr_array(G),
                                         _ptr_array(D), _ptr_array(dG), int(deterministic), _ptr(ws), _nbytes(ws),
                                         _ptr(err_flag), _stream(stream))
    _check(st, "comera_tt_embed_backward")
    return st


EMBED_REUSE_FORWARD = 1


def comera_debug_launch_check(enable: bool) -> None:
    _check(load().comera_debug_launch_check(int(bool(enable))), "comera_debug_launch_check")


def comera_debug_launch_log() -> list:
    """Every launch recorded since launch check mode was switched on:
    dicts with the kernel expression, grid, block, LDS bytes and whether the
    configuration is within the limits."""
    lib = load()
    out = []
    name = ctypes.create_string_buffer(256)
    g3, b3 = (ctypes.c_uint32 * 3)(), (ctypes.c_uint32 * 3)()
    lds, ok = ctypes.c_uint64(), ctypes.c_int32()
    for i in range(int(lib.comera_debug_launch_count())):
        _check(lib.comera_debug_launch_info(i, name, 256, g3, b3, ctypes.byref(lds), ctypes.byref(ok)),
               "comera_debug_launch_info")
        out.append({"kernel": name.value.decode(), "grid": tuple(g3), "block": tuple(b3), "lds": lds.value,
                    "ok": bool(ok.value)})
    return out


def comera_tt_embed_backward_ex(shape, ids, n_tokens: int, dY, G, D, dG, flags: int, ws, err_flag=None,
                                stream=None) -> int:
    st = load().comera_tt_embed_backward_ex(ctypes.byref(shape), _ptr(ids), int(n_tokens), _ptr(dY), _ptr_array(G),
                                            _ptr_array(D), _ptr_array(dG), int(flags), _ptr(ws), _nbytes(ws),
                                            _ptr(err_flag), _stream(stream))
    _check(st, "comera_tt_embed_backward_ex")
    return st


def comera_dense_embed_workspace_bytes(shape: comera_dense_embed_shape, n_tokens: int) -> int:
    return int(load().comera_dense_embed_workspace_bytes(ctypes.byref(shape), int(n_tokens)))


def comera_dense_embed_forward(shape, ids, n_tokens: int, T, scale: float, Y, err_flag=None, stream=None) -> int:
    """Y[t, :] = scale * T[ids[t], :]."""
    lib = load()
    where = "comera_dense_embed_forward"
    ids, T, Y, err_flag = _taken(where, (ids, _i64, n_tokens), (T, _dtype_of(shape.table), shape.V * shape.E),
                                 (Y, _dtype_of(shape.act), n_tokens * shape.E), (err_flag, _i32, 1))
    st = lib.comera_dense_embed_forward(shape, ids, int(n_tokens), T, float(scale), Y, err_flag, _stream(stream))
    _check(st, where)
    return st


def comera_dense_embed_backward(shape, ids, n_tokens: int, dY, scale: float, pad_id: int, dT, ws, err_flag=None,
                                stream=None) -> int:
    """dT[v, :] = scale * the sum of dY's rows of the tokens v; pad_id = -1 for none."""
    lib = load()
    where = "comera_dense_embed_backward"
    ws, nbytes = _workspace(where, ws)
    ids, dY, dT, ws, err_flag = _taken(where, (ids, _i64, n_tokens),
                                       (dY, _dtype_of(shape.act), n_tokens * shape.E),
                                       (dT, _dtype_of(shape.table), shape.V * shape.E), (ws, None, 0),
                                       (err_flag, _i32, 1))
    st = lib.comera_dense_embed_backward(shape, ids, int(n_tokens), dY, float(scale), int(pad_id), dT, ws, nbytes,
                                         err_flag, _stream(stream))
    _check(st, where)
    return st


def comera_block_norm_workspace_bytes(shape: comera_block_norm_shape, b: int) -> int:
    return int(load().comera_block_norm_workspace_bytes(ctypes.byref(shape), int(b)))


def comera_block_norm_forward(shape, b: int, X, F, post_w, post_b, gate, pre_w, pre_b, Xn, H, stream=None) -> int:
    """Xn = res_scale X + branch_scale gate Npost(F), H = Npre(Xn)."""
    lib = load()
    where = "comera_block_norm_forward"
    w, f32 = shape.width, _f32
    st, act, e = _dtype_of(shape.stream), _dtype_of(shape.act), b * w
    p = _taken(where, (X, st, e), (F, act, e), (post_w, f32, w), (post_b, f32, w),
               (gate, act, e) if shape.gate == GATE_TOKEN else (gate, f32, w), (pre_w, f32, w), (pre_b, f32, w),
               (Xn, st, e), (H, act, e))
    rc = lib.comera_block_norm_forward(shape, int(b), *p, _stream(stream))
    _check(rc, where)
    return rc


def comera_block_norm_backward(shape, b: int, Xn, F, post_w, post_b, gate, pre_w, dXn, dH, dX, dF, dgate, dpost_w,
                               dpost_b, dpre_w, dpre_b, ws, stream=None) -> int:
    """Gradients of comera_block_norm_forward; None for an output that is not wanted."""
    lib = load()
    where = "comera_block_norm_backward"
    w, f32 = shape.width, _f32
    st, act, e = _dtype_of(shape.stream), _dtype_of(shape.act), b * w
    gk = (act, e) if shape.gate == GATE_TOKEN else (f32, w)
    ws, nbytes = _workspace(where, ws)
    p = _taken(where, (Xn, st, e), (F, act, e), (post_w, f32, w), (post_b, f32, w), (gate,) + gk, (pre_w, f32, w),
               (dXn, st, e), (dH, act, e), (dX, st, e), (dF, act, e), (dgate,) + gk, (dpost_w, f32, w),
               (dpost_b, f32, w), (dpre_w, f32, w), (dpre_b, f32, w), (ws, None, 0))
    rc = lib.comera_block_norm_backward(shape, int(b), *p, nbytes, _stream(stream))
    _check(rc, where)
    return rc


def comera_grad_plan(tensors, count: int, raise_on_error: bool = True):
    """Plan handle (int) for a host array of comera_grad_tensor or, with
    raise_on_error=False, (status, handle)."""
    h = ctypes.c_void_p()
    st = load().comera_grad_plan(tensors, int(count), ctypes.byref(h))
    if not raise_on_error:
        return st, h.value
    _check(st, "comera_grad_plan")
    return h.value


def comera_grad_plan_destroy(plan) -> None:
    if plan:
        load().comera_grad_plan_destroy(plan)


def comera_grad_table_bytes(plan) -> int:
    return int(load().comera_grad_table_bytes(plan))


def comera_grad_plan_set_table(plan, table, stream=None) -> int:
    """Write a long list's table to `table` (None: work without one); later calls have to be ordered behind it."""
    lib = load()
    where = "comera_grad_plan_set_table"
    table, nbytes = _workspace(where, table)
    st = lib.comera_grad_plan_set_table(plan, *_taken(where, (table, None, 0)), nbytes, _stream(stream))
    _check(st, where)
    return st


def comera_grad_workspace_bytes(plan) -> int:
    return int(load().comera_grad_workspace_bytes(plan))


# GradPlan's tables in device memory: plan handle -> (table, handles of the streams that its memory waits for)
_tables: dict = {}


def _keep_table(plan, stream: int) -> int:
    """Before a call on `stream`: the table's memory, once released, is given
    to nobody else until the work on that stream is done.  Returns the stream."""
    held = _tables.get(plan)
    if held is not None and stream not in held[1]:
        held[0].record_stream(_torch.cuda.ExternalStream(stream) if stream else _torch.cuda.default_stream())
        held[1].add(stream)
    return stream


def comera_grad_norm(plan, scale: float, norm, flag, ws, stream=None) -> int:
    """norm = scale * sqrt(sum of all squares); flag = 1 if it is not finite."""
    lib = load()
    where = "comera_grad_norm"
    ws, nbytes = _workspace(where, ws)
    p = _taken(where, (norm, _f32, 1), (flag, _i32, 1), (ws, None, 0))
    st = lib.comera_grad_norm(plan, float(scale), *p, nbytes, _keep_table(plan, _stream(stream)))
    _check(st, where)
    return st


def comera_grad_clip(plan, scale: float, max_norm: float, norm, flag, ws, stream=None) -> int:
    """The norm, and out = scale * min(1, max_norm / norm) * g for every tensor of the plan."""
    lib = load()
    where = "comera_grad_clip"
    ws, nbytes = _workspace(where, ws)
    p = _taken(where, (norm, _f32, 1), (flag, _i32, 1), (ws, None, 0))
    st = lib.comera_grad_clip(plan, float(scale), float(max_norm), *p, nbytes, _keep_table(plan, _stream(stream)))
    _check(st, where)
    return st


class GradPlan:
    """Owns the plan of a list of gradient tensors and a long list's table,
    and keeps the tensors alive.  outs: where the clipped gradients go (None,
    or a None entry: in place).  Made once, for gradients that keep their
    buffers: 361 tensors take 0.5 to 0.6 ms of the host.  Made outside a graph
    capture: a table is waited for, so that calls on any stream find it.

    The plan may be dropped while calls through this module are pending: its
    table is kept until they are done (streams of one's own have to exist until
    the plan is dropped).  A captured graph holds the table's address: keep the
    plan as long as the graph is replayed.  The gradients and outs are the
    caller's tensors, whose use on other streams than their own is the caller's
    to record, as for every call here."""

    def __init__(self, grads, outs=None):
        self.handle = None
        self.grads = list(grads)
        self.outs = [None] * len(self.grads) if outs is None else list(outs)
        if len(self.outs) != len(self.grads):
            raise ComeraError(ERR_INVALID_ARG, "GradPlan: as many outs as grads are expected")
        load()
        codes = {_f32: F32, _bf16: BF16}
        rows = []
        for g, o in zip(self.grads, self.outs):
            code, n = codes.get(g.dtype), g.numel()
            if code is None:
                raise ComeraError(ERR_INVALID_ARG, f"GradPlan: {g.dtype} gradients are not taken")
            if o is not None and o.numel() != n:
                raise ComeraError(ERR_INVALID_ARG, "GradPlan: an out of another size than its gradient")
            at = _taken("GradPlan", (g, g.dtype, 0), (o, g.dtype, 0))
            rows.append((at[0], at[1], n, code, 0))
        arr = (comera_grad_tensor * max(1, len(rows)))(*rows)
        self.handle = comera_grad_plan(arr, len(self.grads))
        self.table = None
        nbytes = comera_grad_table_bytes(self.handle)
        if nbytes:
            self.table = _torch.empty(nbytes, dtype=_torch.uint8, device=self.grads[0].device)
            comera_grad_plan_set_table(self.handle, self.table)
            _torch.cuda.current_stream().synchronize()
            _tables[self.handle] = self.table, {_stream(None)}     # whose memory it is

    @property
    def workspace_bytes(self) -> int:
        return comera_grad_workspace_bytes(self.handle)

    def __del__(self):
        try:
            _tables.pop(self.handle, None)
            comera_grad_plan_destroy(self.handle)
        except Exception:
            pass
        self.handle = None


class TTMPlan:
    """Owns a plan handle (destroyed with the object)."""

    def __init__(self, n, m, r, act: int = F32, batch: int = 0, mask_active=None, force_order: int = -1):
        self.shape = ttm_shape(n, m, r, act)
        self.n, self.m, self.r, self.act, self.batch = tuple(n), tuple(m), tuple(r), act, batch
        self.handle = comera_ttm_plan(self.shape, batch, mask_active, force_order)

    @property
    def workspace_bytes(self) -> int:
        return comera_ttm_workspace_bytes(self.handle)

    @property
    def num_orders(self) -> int:
        return comera_ttm_plan_num_orders(self.handle)

    @property
    def chosen(self) -> int:
        return comera_ttm_plan_chosen(self.handle)

    def order_info(self, i: int) -> dict:
        return comera_ttm_plan_order_info(self.handle, i)

    def set_reuse_forward(self, enable: bool = True) -> None:
        comera_ttm_plan_set_reuse_forward(self.handle, enable)

    def set_fp8(self, enable: bool = True) -> None:
        comera_ttm_plan_set_fp8(self.handle, enable)

    def __del__(self):
        try:
            comera_ttm_plan_destroy(self.handle)
        except Exception:
            pass
        self.handle = None
