"""Python binding of the DTST spectral-layer library (libdtst.so).

Argument marshalling only: every function here forwards to the C ABI of the
same name declared in ``include/dtst.h``.  Device arrays are torch tensors
(PyTorch provides device memory and streams); their data pointers and the
current HIP stream are passed straight through.  The library must be built
(``python paper_2607_14394_amd/build.py``); importing this module fails
loudly when it is missing -- there is no fallback implementation.
"""

from __future__ import annotations

import array
import ctypes
import functools
import operator
import os
import struct

# torch ships its own HIP runtime under the same soname (libamdhip64.so.7).
# Loading torch first makes libdtst.so bind to that one copy; loading
# libdtst.so first would bring a second HIP/HSA runtime into the process,
# and one of the two then finds no device.
import torch

__all__ = [
    "DtstError", "Desc", "lib", "make_desc", "dtst_desc_validate", "dtst_desc_workspace_bytes",
    "dtst_basis_host", "dtst_plan", "dtst_plan_destroy", "dtst_plan_info", "dtst_forward", "dtst_mix",
    "dtst_inverse", "dtst_forward_adj", "dtst_inverse_adj", "dtst_mix_wgrad", "dtst_block_epilogue",
    "dtst_inverse_block", "dtst_pointwise", "dtst_forward_noalloc", "dtst_profile_enable",
    "dtst_profile_collect", "dtst_plan_block_info", "Schedule", "dtst_desc_schedule", "Plan", "LIB_PATH",
    "PLAN_SPLIT_SCHEDULE", "PLAN_UNFUSED_BLOCK", "SCRATCH_BYTES", "torch_stream",
    "RECURRENCE_SPAN", "code_columns", "scale_columns", "empty_codes", "recurrence_states_shape", "dtst_rms_norm",
    "dtst_rms_norm_adj", "dtst_rms_norm_adj_workspace", "dtst_quantise", "dtst_product",
    "dtst_recurrence", "dtst_recurrence_adj", "dtst_recurrence_workspace",
    "dtst_layer_norm", "dtst_layer_norm_adj", "dtst_layer_norm_adj_workspace", "dtst_global_norm", "dtst_clip",
    "dtst_conv", "dtst_conv_adj", "dtst_conv_adj_workspace", "SCAN_SPAN", "scan_states_shape", "dtst_scan", "dtst_scan_workspace", "dtst_scan_adj",
    "dtst_scan_adj_workspace",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdtst.so")

DTST_OK = 0
PLAN_SPLIT_SCHEDULE = 1      # DTST_PLAN_SPLIT_SCHEDULE of include/dtst.h
PLAN_UNFUSED_BLOCK = 2       # DTST_PLAN_UNFUSED_BLOCK of include/dtst.h
SCRATCH_BYTES = 64 << 20     # DTST_SCRATCH_BYTES of include/dtst.h
STATUS_NAMES = {0: "DTST_OK", 1: "DTST_ERR_INVALID_ARG", 2: "DTST_ERR_UNSUPPORTED",
                3: "DTST_ERR_OUT_OF_MEMORY", 4: "DTST_ERR_DEVICE"}


class DtstError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class KernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 40), ("launches", ctypes.c_int64), ("total_ms", ctypes.c_double)]


class Desc(ctypes.Structure):
    _fields_ = [
        ("n_global", ctypes.c_int64 * 4),
        ("n_local", ctypes.c_int64 * 4),
        ("offset", ctypes.c_int64 * 4),
        ("kmax", ctypes.c_int32 * 3),
        ("kt", ctypes.c_int32),
        ("batch", ctypes.c_int64),
        ("c_in", ctypes.c_int64),
        ("c_out", ctypes.c_int64),
    ]


class Schedule(ctypes.Structure):
    """dtst_schedule: the kernels a plan takes."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("forward", "inverse", "block", "z_classes", "t_folded", "block_z_classes", "block_t_folded",
                 "z_mirrored", "y_parts")]


# The descriptors of the latent-sequence operators, packed in the layout of
# include/dtst.h (a ctypes.Structure takes three times as long to fill).
NORM_DESC = struct.Struct("@7q3if")
NORM_ADJ_DESC = struct.Struct("@7q3i4x")
QUANTISE_DESC = struct.Struct("@7qi4x")
PRODUCT_DESC = struct.Struct("@8q3i4x")
RECURRENCE_DESC = struct.Struct("@17qi4x")
CONV_DESC = struct.Struct("@10q3i4x")
SCAN_DESC = struct.Struct("@26q2i")

# DTST_F32 .. DTST_E4M3 of include/dtst.h
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.float8_e4m3fn: 3}
RECURRENCE_SPAN = 128        # DTST_RECURRENCE_SPAN of include/dtst.h
SCAN_SPAN = 16               # DTST_SCAN_SPAN of include/dtst.h

# DTST_ROWS_* and DTST_BLOCK_* of include/dtst.h
ROWS_T_FIRST, ROWS_T_FIRST_Y, ROWS_Z_FIRST, ROWS_Z_FIRST_Y = range(4)
BLOCK_SEPARATE, BLOCK_CHUNKS, BLOCK_ROW_TASKS = range(3)


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libdtst.so not found at {LIB_PATH}; build it with "
                          "`python paper_2607_14394_amd/build.py` (no fallback path exists)")
    L = ctypes.CDLL(LIB_PATH)
    P, I64, SZ, I, VP = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int, ctypes.c_void_p
    sig = {
        "dtst_desc_validate": [ctypes.POINTER(Desc)],
        "dtst_desc_workspace_bytes": [ctypes.POINTER(Desc), ctypes.POINTER(SZ)],
        "dtst_desc_workspace_bytes_ex": [ctypes.POINTER(Desc), ctypes.c_uint32, ctypes.POINTER(SZ)],
        "dtst_desc_schedule": [ctypes.POINTER(Desc), ctypes.c_uint32, ctypes.POINTER(Schedule)],
        "dtst_basis_host": [ctypes.POINTER(Desc), I, I, ctypes.POINTER(ctypes.c_float), SZ],
        "dtst_plan": [ctypes.POINTER(Desc), ctypes.POINTER(P)],
        "dtst_plan_ex": [ctypes.POINTER(Desc), ctypes.c_uint32, ctypes.POINTER(P)],
        "dtst_plan_destroy": [P],
        "dtst_plan_info": [P, ctypes.POINTER(I64), ctypes.POINTER(SZ)],
        "dtst_plan_block_info": [P, ctypes.POINTER(SZ), ctypes.POINTER(I)],
        "dtst_forward": [P, VP, VP, I, VP, SZ, VP],
        "dtst_mix": [P, VP, VP, VP, I64, I64, I, VP],
        "dtst_inverse": [P, VP, VP, VP, SZ, VP],
        "dtst_forward_adj": [P, VP, VP, VP, SZ, VP],
        "dtst_inverse_adj": [P, VP, VP, I, VP, SZ, VP],
        "dtst_mix_wgrad": [P, VP, VP, VP, I64, I64, I, VP],
        "dtst_block_epilogue": [P, VP, VP, VP, VP],
        "dtst_inverse_block": [P, VP, VP, VP, VP, VP, SZ, VP],
        "dtst_pointwise": [VP, VP, VP, VP, I64, I64, I64, I64, I, VP],
        "dtst_forward_noalloc": [P, VP, VP, I, VP],
        "dtst_rms_norm": [VP] * 9,
        "dtst_rms_norm_adj_workspace": [I64, I64, ctypes.POINTER(SZ)],
        "dtst_rms_norm_adj": [VP] * 10 + [SZ, VP],
        "dtst_layer_norm": [VP] * 11,
        "dtst_layer_norm_adj_workspace": [I64, I64, ctypes.POINTER(SZ)],
        "dtst_layer_norm_adj": [VP] * 12 + [SZ, VP],
        "dtst_quantise": [VP] * 7,
        "dtst_product": [VP] * 8,
        "dtst_recurrence_workspace": [I64, I64, I64, I, ctypes.POINTER(SZ)],
        "dtst_recurrence": [VP] * 10 + [SZ, VP],
        "dtst_recurrence_adj": [VP] * 13 + [SZ, VP],
        "dtst_conv": [VP] * 9,
        "dtst_conv_adj_workspace": [I64, I64, I64, I64, ctypes.POINTER(SZ)],
        "dtst_conv_adj": [VP] * 13 + [SZ, VP],
        "dtst_scan_workspace": [I64, I64, I64, I64, ctypes.POINTER(SZ)],
        "dtst_scan": [VP] * 14 + [SZ, VP],
        "dtst_scan_adj_workspace": [I64, I64, I64, I64, ctypes.POINTER(SZ)],
        "dtst_scan_adj": [VP] * 21 + [SZ, VP],
        "dtst_global_norm_workspace": [I64, VP, ctypes.POINTER(SZ)],
        "dtst_global_norm": [I64] + [VP] * 5 + [SZ, VP],
        "dtst_clip": [I64] + [VP] * 4 + [ctypes.c_float, VP, VP],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    L.dtst_profile_enable.argtypes = [I]
    L.dtst_profile_enable.restype = ctypes.c_int
    L.dtst_profile_collect.argtypes = [ctypes.POINTER(KernelTime), I, ctypes.POINTER(I)]
    L.dtst_profile_collect.restype = ctypes.c_int
    L.dtst_status_string.argtypes = [ctypes.c_int]
    L.dtst_status_string.restype = ctypes.c_char_p
    L.dtst_last_error.argtypes = []
    L.dtst_last_error.restype = ctypes.c_char_p
    return L


lib = _load()


def _check(status):
    if status != DTST_OK:
        raise DtstError(status, lib.dtst_last_error().decode())


def make_desc(n_global, n_local, offset, kmax, kt, batch, c_in, c_out) -> Desc:
    d = Desc()
    for i in range(4):
        d.n_global[i] = int(n_global[i])
        d.n_local[i] = int(n_local[i])
        d.offset[i] = int(offset[i])
    for i in range(3):
        d.kmax[i] = int(kmax[i])
    d.kt = int(kt)
    d.batch, d.c_in, d.c_out = int(batch), int(c_in), int(c_out)
    return d


def _desc(d):
    if isinstance(d, Desc):
        return d
    return make_desc(d["n_global"], d["n_local"], d["offset"], d["kmax"], d["kt"], d["batch"], d["c_in"], d["c_out"])


# ---- host-only helpers -----------------------------------------------------
def dtst_desc_validate(desc):
    _check(lib.dtst_desc_validate(ctypes.byref(_desc(desc))))


def dtst_desc_workspace_bytes(desc, flags=0) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.dtst_desc_workspace_bytes_ex(ctypes.byref(_desc(desc)), int(flags), ctypes.byref(n)))
    return n.value


def dtst_desc_schedule(desc, flags=0) -> Schedule:
    s = Schedule()
    _check(lib.dtst_desc_schedule(ctypes.byref(_desc(desc)), int(flags), ctypes.byref(s)))
    return s


def dtst_basis_host(desc, dim, kind):
    """fp32 basis of one dimension as a complex64 numpy array (K, N_loc)."""
    import numpy as np
    d = _desc(desc)
    if 0 <= dim <= 3:
        k = 2 * d.kmax[dim] if dim < 3 else d.kt
        n = d.n_local[dim]
    else:
        k = n = 1  # the library rejects the request
    buf = np.zeros(max(2 * k * n, 2), dtype=np.float32)
    _check(lib.dtst_basis_host(ctypes.byref(d), int(dim), int(kind),
                               buf.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), buf.size))
    return buf.view(np.complex64).reshape(k, n)


# ---- plans and execute calls (device tensors) ------------------------------
def _ptr(t):
    # (an integer: the c_void_p argument types convert it)
    return None if t is None else t.data_ptr()


def torch_stream():
    """The current torch stream as the integer value of its hipStream_t."""
    # torch.cuda.current_stream() builds a Stream object (3 us a call, as much
    # as a launch); the raw getter returns its handle alone.
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) if hasattr(torch._C, "_cuda_getDevice") else None


def _stream(stream):
    return torch_stream() if stream is None else int(stream)


def dtst_plan(desc, flags=0):
    """dtst_plan_ex; flags 0 or a combination of PLAN_SPLIT_SCHEDULE and
    PLAN_UNFUSED_BLOCK."""
    h = ctypes.c_void_p()
    _check(lib.dtst_plan_ex(ctypes.byref(_desc(desc)), int(flags), ctypes.byref(h)))
    return h


def dtst_plan_destroy(plan):
    _check(lib.dtst_plan_destroy(plan))


def dtst_plan_info(plan):
    m = ctypes.c_int64(0)
    ws = ctypes.c_size_t(0)
    _check(lib.dtst_plan_info(plan, ctypes.byref(m), ctypes.byref(ws)))
    return m.value, ws.value


def dtst_plan_block_info(plan):
    """(workspace bytes of dtst_inverse_block, 1 if it runs the fused kernel)."""
    ws = ctypes.c_size_t(0)
    fused = ctypes.c_int(0)
    _check(lib.dtst_plan_block_info(plan, ctypes.byref(ws), ctypes.byref(fused)))
    return ws.value, fused.value


def _wsargs(ws):
    if ws is None:
        return None, 0
    return ws.data_ptr(), ws.nbytes


def dtst_forward(plan, x, xhat, accumulate, ws, stream=None):
    p, n = _wsargs(ws)
    _check(lib.dtst_forward(plan, _ptr(x), _ptr(xhat), int(accumulate), p, n, _stream(stream)))


def dtst_forward_noalloc(plan, x, xhat, accumulate, stream=None):
    _check(lib.dtst_forward_noalloc(plan, _ptr(x), _ptr(xhat), int(accumulate), _stream(stream)))


def dtst_mix(plan, xhat, w_shard, yhat, m0, m1, op=0, stream=None):
    _check(lib.dtst_mix(plan, _ptr(xhat), _ptr(w_shard), _ptr(yhat), int(m0), int(m1), int(op), _stream(stream)))


def dtst_inverse(plan, yhat, y, ws, stream=None):
    p, n = _wsargs(ws)
    _check(lib.dtst_inverse(plan, _ptr(yhat), _ptr(y), p, n, _stream(stream)))


def dtst_forward_adj(plan, g_xhat, g_x, ws, stream=None):
    p, n = _wsargs(ws)
    _check(lib.dtst_forward_adj(plan, _ptr(g_xhat), _ptr(g_x), p, n, _stream(stream)))


def dtst_inverse_adj(plan, g_y, g_yhat, accumulate, ws, stream=None):
    p, n = _wsargs(ws)
    _check(lib.dtst_inverse_adj(plan, _ptr(g_y), _ptr(g_yhat), int(accumulate), p, n, _stream(stream)))


def dtst_block_epilogue(plan, x, w_bypass, y, stream=None):
    _check(lib.dtst_block_epilogue(plan, _ptr(x), _ptr(w_bypass), _ptr(y), _stream(stream)))


def dtst_inverse_block(plan, yhat, x, w_bypass, y, ws, stream=None):
    _check(lib.dtst_inverse_block(plan, _ptr(yhat), _ptr(x), _ptr(w_bypass), _ptr(y), *_wsargs(ws),
                                  _stream(stream)))


def dtst_pointwise(x, w, bias, y, act=0, stream=None):
    """y = act(w x + bias) over the points of x (batch, c_in, ...) into y
    (batch, c_out, ...); bias may be None.  Shape checks here, arithmetic in
    the library."""
    if x.dim() < 2 or y.dim() != x.dim() or x.shape[0] != y.shape[0] or x.shape[2:] != y.shape[2:]:
        raise ValueError(f"x {tuple(x.shape)} and y {tuple(y.shape)} must be (batch, channels, points...)")
    for t, name in ((x, "x"), (w, "w"), (y, "y")) + (((bias, "bias"),) if bias is not None else ()):
        if t.device.type != "cuda" or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 device tensor")
    B, ci, co = x.shape[0], x.shape[1], y.shape[1]
    if tuple(w.shape) != (co, ci) or (bias is not None and tuple(bias.shape) != (co,)):
        raise ValueError(f"w must be ({co}, {ci}) and bias ({co},)")
    points = x[0, 0].numel()
    _check(lib.dtst_pointwise(_ptr(x), _ptr(w), _ptr(bias), _ptr(y), int(B), int(ci), int(co), int(points), int(act),
                              _stream(stream)))


def dtst_mix_wgrad(plan, xhat, g_yhat, g_w_shard, m0, m1, accumulate, stream=None):
    _check(lib.dtst_mix_wgrad(plan, _ptr(xhat), _ptr(g_yhat), _ptr(g_w_shard), int(m0), int(m1), int(accumulate),
                              _stream(stream)))


# ---- operators on latent sequences (device tensors) --------------------------
# Shape, type and device checks here, arithmetic in the library.  A workspace
# that is not given is allocated for the call.

def code_columns(k):
    """Columns of the codes of rows of k values."""
    return (k + 127) // 128 * 128


def scale_columns(k):
    """Columns of the scales of rows of k values."""
    return ((k + 127) // 128 + 3) // 4 * 4


def empty_codes(rows, k, device="cuda"):
    """Codes (float8_e4m3fn) and scales (float8_e8m0fnu) for rows of k values."""
    return (torch.empty((rows, code_columns(k)), dtype=torch.float8_e4m3fn, device=device),
            torch.empty((rows, scale_columns(k)), dtype=torch.float8_e8m0fnu, device=device))


def recurrence_states_shape(batch, steps, features):
    return (batch, -(-steps // RECURRENCE_SPAN), features)


def _device():
    """The current device (-2 without one: no tensor is there)."""
    try:
        return torch._C._cuda_getDevice()
    except (RuntimeError, AttributeError):
        return -2


# The current stream of a device.
_current = _raw_stream if _raw_stream is not None else lambda dev: torch_stream()


def _refuse(t, shape, name, dtypes):
    raise ValueError(f"{name}: need {' or '.join(str(d) for d in dtypes)} of shape {tuple(shape)} with contiguous rows on "
                     f"the current device, got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


# (The checks of a call are a third of its time on the host: each reads a tensor's properties once.)
def _rows(t, shape, name, dtypes, dev):
    """Row stride of a 2-D tensor on device dev with contiguous rows."""
    if t.shape == shape and t.dtype in dtypes and t.get_device() == dev:
        rows, cols = shape
        if rows > 1 and t.is_contiguous():
            return cols
        s0, s1 = t.stride()
        if s1 == 1 or cols == 1 or rows == 0:
            return s0 if rows > 1 else cols + 15 & -16  # (that of a single row is any; one that suits every type)
    _refuse(t, shape, name, dtypes)


def _vector(t, n, name, dev, dtype=torch.float32):
    if t.shape != (n,) or t.dtype != dtype or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: need contiguous {dtype} of shape ({n},) on the current device")


_FLOATS = (torch.float32, torch.bfloat16, torch.float16)
_CODE, _SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _codes(q, s, rows, k, name, dev):
    """Row strides of codes and scales."""
    kq = k + 127 & -128
    ks = (kq >> 7) + 3 & -4
    if (q.shape == (rows, kq) and s.shape == (rows, ks) and q.dtype is _CODE and s.dtype is _SCALE
            and q.get_device() == dev and s.get_device() == dev):
        if q.is_contiguous() and s.is_contiguous():
            return kq, ks
        (q0, q1), (s0, s1) = q.stride(), s.stride()
        if q1 == 1 and s1 == 1:
            return q0, s0
    _refuse(q, (rows, kq), name, (_CODE,)) if q.shape != (rows, kq) or q.dtype is not _CODE or q.stride(-1) != 1 or (
        q.get_device() != dev) else _refuse(s, (rows, ks), name + " scale", (_SCALE,))


def _scratch(ws, need, device, stream):
    """Pointer and bytes of the workspace, and what keeps it until the launch."""
    if ws is None:
        if not need:
            return None, 0, None
        if stream is None or int(stream) == torch_stream():
            ws = torch.empty(need, dtype=torch.uint8, device=device)
        else:
            # From the memory of the stream that the call runs on: a block that the
            # current stream has freed may still be in use by what is queued there.
            with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=device)):
                ws = torch.empty(need, dtype=torch.uint8, device=device)
    elif ws.device != device or not ws.is_contiguous():
        raise ValueError(f"ws: need a contiguous tensor on {device}, got strides {ws.stride()} on {ws.device}")
    return ws.data_ptr(), ws.nbytes, ws


def dtst_rms_norm(x, weight, y, res=None, sum_out=None, scale=None, rstd=None, eps=1e-6, stream=None):
    """u = x + res into sum_out, y = u / rms(u) * weight; y in x's type, or
    codes with their scales.  x, res, sum_out: (rows, cols)."""
    if x.dim() != 2:
        raise ValueError("x must be (rows, cols)")
    shape = rows, cols = x.shape
    dev, tx = _device(), x.dtype
    rt = res.dtype if res is not None else tx if sum_out is None else sum_out.dtype
    ld_x = _rows(x, shape, "x", _FLOATS, dev)
    ld_res = 0 if res is None else _rows(res, shape, "res", (tx, torch.float32), dev)
    ld_sum = 0 if sum_out is None else _rows(sum_out, shape, "sum_out", (rt,), dev)
    if scale is not None:
        ld_y, ld_scale = _codes(y, scale, rows, cols, "y", dev)
    else:
        ld_y, ld_scale = _rows(y, shape, "y", (tx,), dev), 0
    _vector(weight, cols, "weight", dev)
    if rstd is not None:
        _vector(rstd, rows, "rstd", dev)
    if not rows:  # (the library knows y's scales by their address, which an empty tensor has not)
        return
    status = lib.dtst_rms_norm(
        NORM_DESC.pack(rows, cols, ld_x, ld_res, ld_sum, ld_y, ld_scale, _TYPES[tx], _TYPES[rt], _TYPES[y.dtype], eps),
        x.data_ptr(), None if res is None else res.data_ptr(), weight.data_ptr(),
        None if sum_out is None else sum_out.data_ptr(), y.data_ptr(), None if scale is None else scale.data_ptr(),
        None if rstd is None else rstd.data_ptr(), _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


@functools.lru_cache(maxsize=1024)
def dtst_rms_norm_adj_workspace(rows, cols) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.dtst_rms_norm_adj_workspace(int(rows), int(cols), ctypes.byref(n)))
    return n.value


def dtst_rms_norm_adj(g_y, u, weight, rstd, g_u, g_weight, g_sum=None, g_x=None, accumulate=False, ws=None,
                      stream=None):
    """Backward of dtst_rms_norm from its stored sum u and rstd: g_u (of x and
    res alike; g_x the same in g_y's type) and g_weight."""
    if g_y.dim() != 2:
        raise ValueError("g_y must be (rows, cols)")
    shape = rows, cols = g_y.shape
    dev, tx, tr = _device(), g_y.dtype, (u.dtype,)
    d = NORM_ADJ_DESC.pack(rows, cols, _rows(g_y, shape, "g_y", _FLOATS, dev),
                           _rows(u, shape, "u", (tx, torch.float32), dev),
                           0 if g_sum is None else _rows(g_sum, shape, "g_sum", tr, dev),
                           _rows(g_u, shape, "g_u", tr, dev), 0 if g_x is None else _rows(g_x, shape, "g_x", (tx,), dev),
                           _TYPES[tx], _TYPES[u.dtype], int(accumulate))
    _vector(weight, cols, "weight", dev)
    _vector(g_weight, cols, "g_weight", dev)
    _vector(rstd, rows, "rstd", dev)
    p, n, ws = _scratch(ws, dtst_rms_norm_adj_workspace(rows, cols), g_y.device, stream)
    status = lib.dtst_rms_norm_adj(d, g_y.data_ptr(), u.data_ptr(), weight.data_ptr(), rstd.data_ptr(),
                                   None if g_sum is None else g_sum.data_ptr(), g_u.data_ptr(),
                                   None if g_x is None else g_x.data_ptr(), g_weight.data_ptr(), p, n,
                                   _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def dtst_layer_norm(x, weight, bias, y, res=None, sum_out=None, scale=None, mean=None, rstd=None, eps=1e-5,
                    stream=None):
    """u = x + res into sum_out, y = (u - mean(u)) / std(u) * weight + bias (or
    None); y in x's type, or codes with their scales.  x, res, sum_out: (rows,
    cols); mean, rstd: what the backward needs, (rows,) float32."""
    if x.dim() != 2:
        raise ValueError("x must be (rows, cols)")
    shape = rows, cols = x.shape
    dev, tx = _device(), x.dtype
    rt = res.dtype if res is not None else tx if sum_out is None else sum_out.dtype
    ld_x = _rows(x, shape, "x", _FLOATS, dev)
    ld_res = 0 if res is None else _rows(res, shape, "res", (tx, torch.float32), dev)
    ld_sum = 0 if sum_out is None else _rows(sum_out, shape, "sum_out", (rt,), dev)
    if scale is not None:
        ld_y, ld_scale = _codes(y, scale, rows, cols, "y", dev)
    else:
        ld_y, ld_scale = _rows(y, shape, "y", (tx,), dev), 0
    _vector(weight, cols, "weight", dev)
    if bias is not None:
        _vector(bias, cols, "bias", dev)
    if mean is not None:
        _vector(mean, rows, "mean", dev)
    if rstd is not None:
        _vector(rstd, rows, "rstd", dev)
    if not rows:  # (as in dtst_rms_norm)
        return
    status = lib.dtst_layer_norm(
        NORM_DESC.pack(rows, cols, ld_x, ld_res, ld_sum, ld_y, ld_scale, _TYPES[tx], _TYPES[rt], _TYPES[y.dtype], eps),
        x.data_ptr(), None if res is None else res.data_ptr(), weight.data_ptr(),
        None if bias is None else bias.data_ptr(), None if sum_out is None else sum_out.data_ptr(), y.data_ptr(),
        None if scale is None else scale.data_ptr(), None if mean is None else mean.data_ptr(),
        None if rstd is None else rstd.data_ptr(), _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


@functools.lru_cache(maxsize=1024)
def dtst_layer_norm_adj_workspace(rows, cols) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.dtst_layer_norm_adj_workspace(int(rows), int(cols), ctypes.byref(n)))
    return n.value


def dtst_layer_norm_adj(g_y, u, weight, mean, rstd, g_u, g_weight, g_bias, g_sum=None, g_x=None, accumulate=False,
                        ws=None, stream=None):
    """Backward of dtst_layer_norm from its stored sum u, mean and rstd: g_u (of
    x and res alike; g_x the same in g_y's type), g_weight and g_bias."""
    if g_y.dim() != 2:
        raise ValueError("g_y must be (rows, cols)")
    shape = rows, cols = g_y.shape
    dev, tx, tr = _device(), g_y.dtype, (u.dtype,)
    d = NORM_ADJ_DESC.pack(rows, cols, _rows(g_y, shape, "g_y", _FLOATS, dev),
                           _rows(u, shape, "u", (tx, torch.float32), dev),
                           0 if g_sum is None else _rows(g_sum, shape, "g_sum", tr, dev),
                           _rows(g_u, shape, "g_u", tr, dev), 0 if g_x is None else _rows(g_x, shape, "g_x", (tx,), dev),
                           _TYPES[tx], _TYPES[u.dtype], int(accumulate))
    _vector(weight, cols, "weight", dev)
    _vector(g_weight, cols, "g_weight", dev)
    _vector(g_bias, cols, "g_bias", dev)
    _vector(mean, rows, "mean", dev)
    _vector(rstd, rows, "rstd", dev)
    p, n, ws = _scratch(ws, dtst_layer_norm_adj_workspace(rows, cols), g_y.device, stream)
    status = lib.dtst_layer_norm_adj(d, g_y.data_ptr(), u.data_ptr(), weight.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                     None if g_sum is None else g_sum.data_ptr(), g_u.data_ptr(),
                                     None if g_x is None else g_x.data_ptr(), g_weight.data_ptr(), g_bias.data_ptr(), p, n,
                                     _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def dtst_quantise(x, q=None, scale=None, qt=None, scale_t=None, stream=None):
    """Rows of x (rows, cols) as codes and scales into q and scale, and (or)
    its transpose's rows into qt and scale_t."""
    if x.dim() != 2:
        raise ValueError("x must be (rows, cols)")
    if (q is None) != (scale is None) or (qt is None) != (scale_t is None) or (q is None and qt is None):
        raise ValueError("need q with scale, or qt with scale_t, or all four")
    rows, cols = x.shape
    dev = _device()
    ld_x = _rows(x, (rows, cols), "x", _FLOATS, dev)
    ld_q, ld_s = (0, 0) if q is None else _codes(q, scale, rows, cols, "q", dev)
    ld_qt, ld_st = (0, 0) if qt is None else _codes(qt, scale_t, cols, rows, "qt", dev)
    if not rows:  # (as in dtst_rms_norm)
        return
    status = lib.dtst_quantise(QUANTISE_DESC.pack(rows, cols, ld_x, ld_q, ld_s, ld_qt, ld_st, _TYPES[x.dtype]),
                               x.data_ptr(), None if q is None else q.data_ptr(),
                               None if scale is None else scale.data_ptr(), None if qt is None else qt.data_ptr(),
                               None if scale_t is None else scale_t.data_ptr(),
                               _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def dtst_product(a, a_scale, b, b_scale, c, bias=None, accumulate=False, short_sums=False, stream=None):
    """c = a b^T + bias (+ c): codes a (m, k) and b (n, k) with their scales
    into c (m, n).  short_sums: sums of fewer bits would do (they are exact all
    the same)."""
    if c.dim() != 2 or a.dim() != 2:
        raise ValueError("a and c must be (m, k) and (m, n)")
    m, n = c.shape
    k = a.shape[1]
    dev = _device()
    ld_a, ld_sa = _codes(a, a_scale, m, k, "a", dev)
    ld_b, ld_sb = _codes(b, b_scale, n, k, "b", dev)
    d = PRODUCT_DESC.pack(m, n, k, ld_a, ld_sa, ld_b, ld_sb, _rows(c, (m, n), "c", _FLOATS, dev), _TYPES[c.dtype],
                          int(accumulate), int(short_sums))
    if bias is not None:
        _vector(bias, n, "bias", dev)
    status = lib.dtst_product(d, a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(),
                              None if bias is None else bias.data_ptr(), c.data_ptr(),
                              _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


@functools.lru_cache(maxsize=1024)
def dtst_recurrence_workspace(batch, steps, features, dtype) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.dtst_recurrence_workspace(int(batch), int(steps), int(features), _TYPES[dtype], ctypes.byref(n)))
    return n.value


def _sequence(t, shape, name, dtype, dev):
    """Strides of batch entries and steps of a (batch, steps, features) tensor."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev:
        sb, st, sf = t.stride()
        if sf == 1 or shape[2] == 1 or t.numel() == 0:
            return sb, st
    _refuse(t, shape, name, (dtype,))


def _state(t, shape, name, dev):
    if t.shape != shape or t.dtype != torch.float32 or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: need contiguous torch.float32 of shape {tuple(shape)} on the current device")


def dtst_recurrence(z, v, y, o=None, h0=None, h_out=None, lengths=None, states=None, ws=None, stream=None):
    """h_t = s(z_t) h_{t-1} + (1 - s(z_t)) v_t, y_t = h_t o_t s(o_t) along the
    steps of (batch, steps, features); h0, h_out: (batch, features) float32,
    lengths: (batch,) int32, states: recurrence_states_shape float32."""
    if z.dim() != 3:
        raise ValueError("z must be (batch, steps, features)")
    shape = B, T, F = z.shape
    e, dev = z.dtype, _device()
    if e not in _FLOATS:
        raise ValueError(f"z: need {' or '.join(str(d) for d in _FLOATS)}")
    d = RECURRENCE_DESC.pack(B, T, F, *_sequence(z, shape, "z", e, dev), *_sequence(v, shape, "v", e, dev),
                             *((0, 0) if o is None else _sequence(o, shape, "o", e, dev)),
                             *_sequence(y, shape, "y", e, dev), 0, 0, 0, 0, 0, 0, _TYPES[e])
    if h0 is not None:
        _state(h0, (B, F), "h0", dev)
    if h_out is not None:
        _state(h_out, (B, F), "h_out", dev)
    if states is not None:
        _state(states, recurrence_states_shape(B, T, F), "states", dev)
    if lengths is not None:
        _vector(lengths, B, "lengths", dev, torch.int32)
    if T <= RECURRENCE_SPAN and ws is None:  # (none is needed)
        p, n = None, 0
    else:
        p, n, ws = _scratch(ws, dtst_recurrence_workspace(B, T, F, e), z.device, stream)
    status = lib.dtst_recurrence(d, z.data_ptr(), v.data_ptr(), None if o is None else o.data_ptr(),
                                 None if h0 is None else h0.data_ptr(), None if lengths is None else lengths.data_ptr(),
                                 y.data_ptr(), None if h_out is None else h_out.data_ptr(),
                                 None if states is None else states.data_ptr(), p, n,
                                 _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def dtst_recurrence_adj(z, v, g_y, states, g_z, g_v, o=None, g_o=None, g_h=None, g_hzero=None, lengths=None, ws=None,
                        stream=None):
    """Backward of dtst_recurrence from its inputs and states: g_z, g_v, g_o
    and, from the gradient g_h of the last state, g_hzero of the first."""
    if z.dim() != 3:
        raise ValueError("z must be (batch, steps, features)")
    shape = B, T, F = z.shape
    e, dev = z.dtype, _device()
    if e not in _FLOATS:
        raise ValueError(f"z: need {' or '.join(str(d) for d in _FLOATS)}")
    if (o is None) != (g_o is None):
        raise ValueError("g_o goes with o")
    none = (0, 0)
    d = RECURRENCE_DESC.pack(B, T, F, *_sequence(z, shape, "z", e, dev), *_sequence(v, shape, "v", e, dev),
                             *(none if o is None else _sequence(o, shape, "o", e, dev)),
                             *_sequence(g_y, shape, "g_y", e, dev), *_sequence(g_z, shape, "g_z", e, dev),
                             *_sequence(g_v, shape, "g_v", e, dev),
                             *(none if g_o is None else _sequence(g_o, shape, "g_o", e, dev)), _TYPES[e])
    if g_h is not None:
        _state(g_h, (B, F), "g_h", dev)
    if g_hzero is not None:
        _state(g_hzero, (B, F), "g_hzero", dev)
    _state(states, recurrence_states_shape(B, T, F), "states", dev)
    if lengths is not None:
        _vector(lengths, B, "lengths", dev, torch.int32)
    p, n, ws = _scratch(ws, dtst_recurrence_workspace(B, T, F, e), z.device, stream)
    status = lib.dtst_recurrence_adj(d, z.data_ptr(), v.data_ptr(), _ptr(o), _ptr(lengths), states.data_ptr(),
                                     g_y.data_ptr(), _ptr(g_h), g_z.data_ptr(), g_v.data_ptr(), _ptr(g_o),
                                     _ptr(g_hzero), p, n, _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def _typed_state(t, shape, name, dtype, dev):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: need contiguous {dtype} of shape {tuple(shape)} on the current device")


def dtst_conv(x, weight, y, bias=None, state=None, state_out=None, lengths=None, silu=True, stream=None):
    """y_t = act(bias + sum_k weight_k x_{t-K+1+k}) along the steps of (batch, steps,
    features), act(v) = v s(v) (silu) or v.  weight: (taps, features) float32, bias:
    (features,) float32, state, state_out: the taps - 1 inputs before the first and
    after the last step, (batch, taps - 1, features) of x's type, lengths: (batch,)
    int32."""
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x must be (batch, steps, features), weight (taps, features)")
    shape = B, T, F = x.shape
    K = weight.shape[0]
    e, dev = x.dtype, _device()
    if e not in _FLOATS:
        raise ValueError(f"x: need {' or '.join(str(t) for t in _FLOATS)}")
    d = CONV_DESC.pack(B, T, F, K, *_sequence(x, shape, "x", e, dev), *_sequence(y, shape, "y", e, dev), 0, 0, _TYPES[e],
                       int(silu), 0)
    _array(weight, (K, F), "weight", dev)
    if bias is not None:
        _vector(bias, F, "bias", dev)
    if state is not None:
        _typed_state(state, (B, K - 1, F), "state", e, dev)
    if state_out is not None:
        _typed_state(state_out, (B, K - 1, F), "state_out", e, dev)
    if lengths is not None:
        _vector(lengths, B, "lengths", dev, torch.int32)
    status = lib.dtst_conv(d, x.data_ptr(), weight.data_ptr(), None if bias is None else bias.data_ptr(),
                           None if state is None else state.data_ptr(), None if lengths is None else lengths.data_ptr(),
                           y.data_ptr(), None if state_out is None else state_out.data_ptr(),
                           _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


@functools.lru_cache(maxsize=1024)
def dtst_conv_adj_workspace(batch, steps, features, taps) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.dtst_conv_adj_workspace(int(batch), int(steps), int(features), int(taps), ctypes.byref(n)))
    return n.value


def dtst_conv_adj(x, weight, g_y, g_x, g_weight, bias=None, g_bias=None, state=None, g_state_out=None, g_state=None,
                  lengths=None, silu=True, accumulate=False, ws=None, stream=None):
    """Backward of dtst_conv from its inputs: g_x, g_weight, g_bias and, with the
    gradient g_state_out of the inputs after the last step, g_state of those before
    the first.  accumulate: g_weight and g_bias are added to."""
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x must be (batch, steps, features), weight (taps, features)")
    shape = B, T, F = x.shape
    K = weight.shape[0]
    e, dev = x.dtype, _device()
    if e not in _FLOATS:
        raise ValueError(f"x: need {' or '.join(str(t) for t in _FLOATS)}")
    d = CONV_DESC.pack(B, T, F, K, *_sequence(x, shape, "x", e, dev), *_sequence(g_y, shape, "g_y", e, dev),
                       *_sequence(g_x, shape, "g_x", e, dev), _TYPES[e], int(silu), int(accumulate))
    _array(weight, (K, F), "weight", dev)
    _array(g_weight, (K, F), "g_weight", dev)
    for t, name in ((bias, "bias"), (g_bias, "g_bias")):
        if t is not None:
            _vector(t, F, name, dev)
    for t, name in ((state, "state"), (g_state_out, "g_state_out"), (g_state, "g_state")):
        if t is not None:
            _typed_state(t, (B, K - 1, F), name, e, dev)
    if lengths is not None:
        _vector(lengths, B, "lengths", dev, torch.int32)
    p, n, ws = _scratch(ws, dtst_conv_adj_workspace(B, T, F, K), x.device, stream)
    status = lib.dtst_conv_adj(d, x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(state), _ptr(lengths), g_y.data_ptr(),
                               _ptr(g_state_out), g_x.data_ptr(), g_weight.data_ptr(), _ptr(g_bias), _ptr(g_state), p, n,
                               _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def scan_states_shape(batch, steps, features, states):
    return (batch, -(-steps // SCAN_SPAN), states, features)


@functools.lru_cache(maxsize=1024)
def dtst_scan_workspace(batch, steps, features, states) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.dtst_scan_workspace(int(batch), int(steps), int(features), int(states), ctypes.byref(n)))
    return n.value


def _array(t, shape, name, dev):
    if t.shape != shape or t.dtype != torch.float32 or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: need contiguous torch.float32 of shape {tuple(shape)} on the current device")


_NONE = (0, 0)
_NO_GRADIENTS = (0,) * 10


def dtst_scan(x, delta, a, b, c, y, d=None, o=None, h0=None, h_out=None, lengths=None, states=None, ws=None, stream=None):
    """h_t = exp(D_t a) h_{t-1} + D_t x_t b_t with D = log(1 + exp(delta)),
    y_t = (sum over the states of c_t h_t, + d x_t) o_t s(o_t).  x, delta, o, y:
    (batch, steps, features), b, c: (batch, steps, states), a: (states, features)
    float32, d: (features,) float32, h0, h_out: (batch, states, features) float32,
    lengths: (batch,) int32, states: scan_states_shape float32, for the backward."""
    if x.dim() != 3 or a.dim() != 2:
        raise ValueError("x must be (batch, steps, features), a (states, features)")
    shape = B, T, F = x.shape
    N = a.shape[0]
    e, dev = x.dtype, _device()
    if e not in _FLOATS:
        raise ValueError(f"x: need {' or '.join(str(t) for t in _FLOATS)}")
    bc = (B, T, N)
    desc = SCAN_DESC.pack(B, T, F, N, *_sequence(x, shape, "x", e, dev), *_sequence(delta, shape, "delta", e, dev),
                          *_sequence(b, bc, "b", e, dev), *_sequence(c, bc, "c", e, dev),
                          *(_NONE if o is None else _sequence(o, shape, "o", e, dev)), *_sequence(y, shape, "y", e, dev),
                          *_NO_GRADIENTS, _TYPES[e], 0)
    _array(a, (N, F), "a", dev)
    if d is not None:
        _vector(d, F, "d", dev)
    if h0 is not None:
        _array(h0, (B, N, F), "h0", dev)
    if h_out is not None:
        _array(h_out, (B, N, F), "h_out", dev)
    if states is not None:
        _array(states, scan_states_shape(B, T, F, N), "states", dev)
    if lengths is not None:
        _vector(lengths, B, "lengths", dev, torch.int32)
    if T == 1 and ws is None:  # (none is needed)
        p, n = None, 0
    else:
        p, n, ws = _scratch(ws, dtst_scan_workspace(B, T, F, N), x.device, stream)
    status = lib.dtst_scan(desc, x.data_ptr(), delta.data_ptr(), a.data_ptr(), b.data_ptr(), c.data_ptr(),
                           None if d is None else d.data_ptr(), None if o is None else o.data_ptr(),
                           None if h0 is None else h0.data_ptr(), None if lengths is None else lengths.data_ptr(),
                           y.data_ptr(), None if h_out is None else h_out.data_ptr(),
                           None if states is None else states.data_ptr(), p, n,
                           _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


@functools.lru_cache(maxsize=1024)
def dtst_scan_adj_workspace(batch, steps, features, states) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.dtst_scan_adj_workspace(int(batch), int(steps), int(features), int(states), ctypes.byref(n)))
    return n.value


def dtst_scan_adj(x, delta, a, b, c, g_y, states, g_x, g_delta, g_a, g_b, g_c, d=None, g_d=None, o=None, g_o=None, g_h=None,
                  g_hzero=None, lengths=None, accumulate=False, ws=None, stream=None):
    """Backward of dtst_scan from its inputs and states: the gradients of each
    operand in its shape and type and, from the gradient g_h of the last states,
    g_hzero of the first.  accumulate: g_a and g_d are added to."""
    if x.dim() != 3 or a.dim() != 2:
        raise ValueError("x must be (batch, steps, features), a (states, features)")
    shape = B, T, F = x.shape
    N = a.shape[0]
    e, dev = x.dtype, _device()
    if e not in _FLOATS:
        raise ValueError(f"x: need {' or '.join(str(t) for t in _FLOATS)}")
    if (o is None) != (g_o is None):
        raise ValueError("g_o goes with o")
    bc = (B, T, N)
    desc = SCAN_DESC.pack(B, T, F, N, *_sequence(x, shape, "x", e, dev), *_sequence(delta, shape, "delta", e, dev),
                          *_sequence(b, bc, "b", e, dev), *_sequence(c, bc, "c", e, dev),
                          *(_NONE if o is None else _sequence(o, shape, "o", e, dev)),
                          *_sequence(g_y, shape, "g_y", e, dev), *_sequence(g_x, shape, "g_x", e, dev),
                          *_sequence(g_delta, shape, "g_delta", e, dev), *_sequence(g_b, bc, "g_b", e, dev),
                          *_sequence(g_c, bc, "g_c", e, dev),
                          *(_NONE if g_o is None else _sequence(g_o, shape, "g_o", e, dev)), _TYPES[e], int(accumulate))
    _array(a, (N, F), "a", dev)
    _array(g_a, (N, F), "g_a", dev)
    _array(states, scan_states_shape(B, T, F, N), "states", dev)
    for t, name in ((d, "d"), (g_d, "g_d")):
        if t is not None:
            _vector(t, F, name, dev)
    for t, name in ((g_h, "g_h"), (g_hzero, "g_hzero")):
        if t is not None:
            _array(t, (B, N, F), name, dev)
    if lengths is not None:
        _vector(lengths, B, "lengths", dev, torch.int32)
    p, n, ws = _scratch(ws, dtst_scan_adj_workspace(B, T, F, N), x.device, stream)
    status = lib.dtst_scan_adj(desc, x.data_ptr(), delta.data_ptr(), a.data_ptr(), b.data_ptr(), c.data_ptr(), _ptr(d),
                               _ptr(o), _ptr(lengths), states.data_ptr(), g_y.data_ptr(), _ptr(g_h), g_x.data_ptr(),
                               g_delta.data_ptr(), g_a.data_ptr(), g_b.data_ptr(), g_c.data_ptr(), _ptr(g_d), _ptr(g_o),
                               _ptr(g_hzero), p, n, _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


# ---- the gradients of a training step ----------------------------------------

_dtype_of = operator.attrgetter("dtype")
_COUNTED = {**_TYPES, torch.complex64: 0}  # (as twice as many real values)
del _COUNTED[torch.float8_e4m3fn]


def _tensors(tensors, name, dev):
    """Addresses, counts, types and dtypes of a list of tensors.  (Hundreds of
    them: each property is read by one pass in C.)"""
    T = torch.Tensor
    tensors = list(tensors)
    dtypes = list(map(_dtype_of, tensors))
    kinds = set(dtypes)
    if not (kinds <= _COUNTED.keys() and set(map(T.get_device, tensors)) <= {dev} and all(map(T.is_contiguous, tensors))
            and not (torch.complex64 in kinds and any(map(T.is_conj, tensors)))):
        raise ValueError(f"{name}: need contiguous tensors of {', '.join(str(d) for d in _COUNTED)} on the current device")
    counts = array.array("q", map(T.numel, tensors))
    if torch.complex64 in kinds:
        counts = array.array("q", [n * (1 + (d is torch.complex64)) for n, d in zip(counts, dtypes)])
    types = array.array("i", [_COUNTED[dtypes[0]]] * len(dtypes) if len(kinds) == 1 else map(_COUNTED.get, dtypes))
    return array.array("Q", map(T.data_ptr, tensors)), counts, types, dtypes


def _at(a):
    return a.buffer_info()[0]


def _one(t, name, dev):
    if t.numel() != 1 or t.dtype != torch.float32 or t.get_device() != dev:
        raise ValueError(f"{name}: need one torch.float32 on the current device")


def dtst_global_norm(tensors, norm, ws=None, stream=None):
    """The norm of all tensors (float32, bfloat16, float16, complex64) together
    into norm, one float32 on the device.  Over shards, the root of the sum of
    the norms' squares is the whole's."""
    dev = _device()
    p, counts, types, _ = _tensors(tensors, "tensors", dev)
    _one(norm, "norm", dev)
    need = ctypes.c_size_t(0)
    _check(lib.dtst_global_norm_workspace(len(counts), _at(counts), ctypes.byref(need)))
    q, n, ws = _scratch(ws, need.value, norm.device, stream)
    status = lib.dtst_global_norm(len(counts), _at(p), _at(counts), _at(types), norm.data_ptr(), q, n,
                                  _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def dtst_clip(tensors, norm, most, out=None, stream=None):
    """tensors min(1, most / norm), in place or into the tensors `out` of the same
    shapes and types; norm: one float32 on the device."""
    dev = _device()
    p, counts, types, dtypes = _tensors(tensors, "tensors", dev)
    _one(norm, "norm", dev)
    po = None
    if out is not None:
        po, n_out, _, d_out = _tensors(out, "out", dev)
        if n_out != counts or d_out != dtypes:
            raise ValueError("out: need the tensors' sizes and types")
    status = lib.dtst_clip(len(counts), _at(p), _at(counts), _at(types), norm.data_ptr(), float(most),
                           None if po is None else _at(po), _current(dev) if stream is None else int(stream))
    if status:
        _check(status)


def dtst_profile_enable(on=True):
    _check(lib.dtst_profile_enable(1 if on else 0))


def dtst_profile_collect():
    """{kernel role: (launches, total_ms)} since the last collect."""
    cap = 32
    arr = (KernelTime * cap)()
    n = ctypes.c_int(0)
    _check(lib.dtst_profile_collect(arr, cap, ctypes.byref(n)))
    return {arr[i].name.decode(): (arr[i].launches, arr[i].total_ms) for i in range(n.value)}


class Plan:
    """Owns one library plan and a torch-allocated workspace; shape and dtype
    checks on the tensors happen here, the arithmetic in the library."""

    def __init__(self, desc, device="cuda", flags=0):
        self.desc = _desc(desc)
        self.handle = dtst_plan(self.desc, flags)
        self.n_modes, self.ws_bytes = dtst_plan_info(self.handle)
        self.ws = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device=device)
        self.block_ws_bytes, self.block_fused = dtst_plan_block_info(self.handle)
        self.ws_block = None   # allocated by the first inverse_block when larger than ws
        self.device = device
        d = self.desc
        self.K = (2 * d.kmax[0], 2 * d.kmax[1], 2 * d.kmax[2], d.kt)
        self.n_local = tuple(d.n_local)
        # tensor shapes of the calls (a tuple per call and tensor otherwise)
        self._x, self._y = self.spatial_shape(d.c_in), self.spatial_shape(d.c_out)
        self._xhat, self._yhat = self.spectral_shape(d.c_in), self.spectral_shape(d.c_out)
        self._channels = (d.c_in, d.c_out)

    def close(self):
        if self.handle is not None:
            dtst_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- shape helpers --
    def spatial_shape(self, channels):
        return (self.desc.batch, channels) + self.n_local

    def spectral_shape(self, channels):
        return (self.desc.batch, channels) + self.K

    def _need(self, t, shape, dtype, name):
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(f"{name}: need contiguous {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")

    def forward(self, x, xhat, accumulate=False, stream=None):
        self._need(x, self._x, torch.float32, "x")
        self._need(xhat, self._xhat, torch.complex64, "xhat")
        dtst_forward(self.handle, x, xhat, accumulate, self.ws, stream)

    def inverse(self, yhat, y, stream=None):
        self._need(yhat, self._yhat, torch.complex64, "yhat")
        self._need(y, self._y, torch.float32, "y")
        dtst_inverse(self.handle, yhat, y, self.ws, stream)

    def forward_adj(self, g_xhat, g_x, stream=None):
        self._need(g_xhat, self._xhat, torch.complex64, "g_xhat")
        self._need(g_x, self._x, torch.float32, "g_x")
        dtst_forward_adj(self.handle, g_xhat, g_x, self.ws, stream)

    def inverse_adj(self, g_y, g_yhat, accumulate=False, stream=None):
        self._need(g_y, self._y, torch.float32, "g_y")
        self._need(g_yhat, self._yhat, torch.complex64, "g_yhat")
        dtst_inverse_adj(self.handle, g_y, g_yhat, accumulate, self.ws, stream)

    def mix(self, xhat, w, yhat, m0=0, m1=None, op=0, stream=None):
        m1 = self.n_modes if m1 is None else m1
        a, b = (self._xhat, self._yhat) if op == 0 else (self._yhat, self._xhat)
        self._need(xhat, a, torch.complex64, "xhat")
        self._need(yhat, b, torch.complex64, "yhat")
        self._need(w, (m1 - m0,) + self._channels, torch.complex64, "w")
        dtst_mix(self.handle, xhat, w, yhat, m0, m1, op, stream)

    def wgrad(self, xhat, g_yhat, g_w, m0=0, m1=None, accumulate=False, stream=None):
        m1 = self.n_modes if m1 is None else m1
        self._need(xhat, self._xhat, torch.complex64, "xhat")
        self._need(g_yhat, self._yhat, torch.complex64, "g_yhat")
        self._need(g_w, (m1 - m0,) + self._channels, torch.complex64, "g_w")
        dtst_mix_wgrad(self.handle, xhat, g_yhat, g_w, m0, m1, accumulate, stream)

    def inverse_block(self, yhat, x, w_bypass, y, stream=None):
        """y = GELU(w_bypass x + inverse(yhat)) (the block's last step)."""
        self._need(yhat, self._yhat, torch.complex64, "yhat")
        self._need(x, self._x, torch.float32, "x")
        self._need(w_bypass, self._channels[::-1], torch.float32, "w_bypass")
        self._need(y, self._y, torch.float32, "y")
        ws = self.ws
        if self.block_ws_bytes > self.ws_bytes:
            if self.ws_block is None:
                self.ws_block = torch.empty(self.block_ws_bytes, dtype=torch.uint8, device=self.device)
            ws = self.ws_block
        dtst_inverse_block(self.handle, yhat, x, w_bypass, y, ws, stream)

    def block_epilogue(self, x, w_bypass, y, stream=None):
        """y <- GELU(w_bypass x + y) in place (the block's bypass and activation)."""
        self._need(x, self._x, torch.float32, "x")
        self._need(w_bypass, self._channels[::-1], torch.float32, "w_bypass")
        self._need(y, self._y, torch.float32, "y")
        dtst_block_epilogue(self.handle, x, w_bypass, y, stream)
