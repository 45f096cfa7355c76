"""ctypes binding over libgi.so (declared in include/gi.h).

Argument marshalling only: every step of the inference path runs inside the library.
PyTorch is used for device memory and streams.  There is no fallback: if the library
has not been built, or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Any, List, NamedTuple, Optional, Sequence

import numpy as np

from . import workloads as wl

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgi.so")

GI_OK = 0
GI_E_INVALID, GI_E_UNSUPPORTED, GI_E_NOMEM, GI_E_CUDA, GI_E_STATE, GI_E_ARENA = -1, -2, -3, -4, -5, -6
GI_F16, GI_F32, GI_BF16, GI_Q4 = 1, 2, 3, 4  # GI_BF16: operators on rows, scales; GI_Q4: weights of a 1x1 convolution
GI_NHWC, GI_PHWC4 = 0, 1
GI_OP_CONV2D, GI_OP_DEPTHWISE_CONV2D, GI_OP_ADD, GI_OP_ACTIVATION, GI_OP_GLOBAL_AVG_POOL, GI_OP_RESIZE_BILINEAR = 1, 2, 3, 4, 5, 6
GI_OP_CONCAT = 7
GI_EXEC_PACK, GI_EXEC_UNPACK = 100, 101
GI_ACT_NONE, GI_ACT_RELU, GI_ACT_RELU6 = 0, 1, 2
GI_PLAN_GREEDY_BY_SIZE, GI_PLAN_GREEDY_SHARED_OBJECTS, GI_PLAN_NAIVE, GI_PLAN_MIN_COST_FLOW = 0, 1, 2, 3
GI_PW_AUTO, GI_PW_SIMT, GI_PW_TC_PAIR, GI_PW_TC_LANE, GI_PW_TC_WIDE, GI_PW_RULE = 0, 1, 2, 3, 4, 5
GI_XOP_AUTO, GI_XOP_OFF, GI_XOP_ON, GI_XOP_CHAIN = 0, 1, 2, 3
GI_STATIC_ARENA_BYTES = 16 << 20
GI_MAX_TOP = 32
KERNEL_NAMES = {1: "pack", 2: "unpack", 3: "conv_simt", 4: "pointwise_tc", 5: "depthwise", 6: "eltwise", 7: "pool",
                8: "resize", 9: "conv3x3_tc", 10: "pointwise_ts", 11: "depthwise_pointwise", 12: "none", 13: "concat", 14: "conv_tc", 15: "inverted_residual", 16: "pointwise_mm", 17: "pointwise_chain", 18: "block_mma", 19: "pointwise_mma", 20: "conv_mma", 21: "linear_q4"}

_KIND = {wl.CONV2D: GI_OP_CONV2D, wl.DEPTHWISE: GI_OP_DEPTHWISE_CONV2D, wl.ADD: GI_OP_ADD,
         wl.ACTIVATION: GI_OP_ACTIVATION, wl.GLOBAL_AVG_POOL: GI_OP_GLOBAL_AVG_POOL,
         wl.RESIZE_BILINEAR: GI_OP_RESIZE_BILINEAR, wl.CONCAT: GI_OP_CONCAT}
_ACT = {wl.ACT_NONE: GI_ACT_NONE, wl.ACT_RELU: GI_ACT_RELU, wl.ACT_RELU6: GI_ACT_RELU6}


class gi_op_desc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("inputs", C.c_int32 * 2), ("kh", C.c_int32), ("kw", C.c_int32),
                ("stride_h", C.c_int32), ("stride_w", C.c_int32), ("dilation_h", C.c_int32), ("dilation_w", C.c_int32),
                ("pad_t", C.c_int32), ("pad_l", C.c_int32), ("pad_b", C.c_int32), ("pad_r", C.c_int32),
                ("cout", C.c_int32), ("act", C.c_int32), ("out_h", C.c_int32), ("out_w", C.c_int32),
                ("align_corners", C.c_int32), ("weight_dtype", C.c_int32), ("weights", C.c_void_p),
                ("bias", C.c_void_p)]


class gi_q4_weights(C.Structure):
    _fields_ = [("q", C.c_void_p), ("scales", C.c_void_p), ("zeros", C.c_void_p), ("scale_dtype", C.c_int32), ("group", C.c_int32)]


class gi_compile_options(C.Structure):
    _fields_ = [("planner", C.c_int32), ("fuse", C.c_int32), ("align", C.c_int32), ("pointwise", C.c_int32),
                ("cross_op", C.c_int32)]


class gi_exec_info(C.Structure):
    _fields_ = [("n_ops", C.c_int32), ("n_fused_ops", C.c_int32), ("n_tensors", C.c_int32), ("batch", C.c_int32),
                ("storage", C.c_int32), ("arena_bytes", C.c_uint64), ("naive_bytes", C.c_uint64),
                ("lower_bound_bytes", C.c_uint64), ("weight_bytes", C.c_uint64)]


class gi_tensor_info(C.Structure):
    _fields_ = [("h", C.c_int32), ("w", C.c_int32), ("c", C.c_int32), ("alive", C.c_int32), ("intermediate", C.c_int32),
                ("first_op", C.c_int32), ("last_op", C.c_int32), ("bytes", C.c_uint64), ("offset", C.c_uint64)]


class gi_op_info(C.Structure):
    _fields_ = [("kind", C.c_int32), ("graph_op", C.c_int32), ("inputs", C.c_int32 * 2), ("residual", C.c_int32),
                ("output", C.c_int32), ("act_pre", C.c_int32), ("act_post", C.c_int32), ("kernel", C.c_int32),
                ("bytes", C.c_uint64), ("flops", C.c_uint64)]


class gi_launch_info(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("n_ops", C.c_int32), ("bytes", C.c_uint64), ("flops", C.c_uint64)]


class gi_linear_q4(C.Structure):
    _fields_ = [("cin", C.c_int32), ("cout", C.c_int32), ("group", C.c_int32), ("scale_dtype", C.c_int32), ("has_zeros", C.c_int32),
                ("dtype", C.c_int32), ("act", C.c_int32)]


class gi_log_probs_desc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("classes", C.c_int32), ("ld", C.c_int64), ("dtype", C.c_int32), ("temperature", C.c_float),
                ("n_given", C.c_int32), ("top", C.c_int32)]


EXPORTS = ["gi_graph_create", "gi_graph_input", "gi_add_op", "gi_graph_output", "gi_graph_destroy", "gi_compile",
           "gi_exec_query", "gi_exec_tensor", "gi_exec_op", "gi_exec_launch", "gi_exec_bind", "gi_run", "gi_run_static", "gi_run_timed", "gi_device_status", "gi_selftest_bounded_wait", "gi_exec_destroy",
           "gi_slice8_tensor_bytes", "gi_slice8_pointwise_blob_bytes", "gi_slice8_pointwise_pack", "gi_slice8_pointwise_run",
           "gi_linear_q4_blob_bytes", "gi_linear_q4_pack", "gi_linear_q4_pack_device", "gi_linear_q4_run", "gi_log_probs",
           "gi_status_str", "gi_last_error", "gi_tensor_bytes", "gi_f32_to_f16"]

_lib = None


class GiError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: status {status}: {detail}")
        self.status = status


def lib() -> C.CDLL:
    """Load libgi.so; raises if it has not been built (python -m paper_1907_01989_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python {os.path.join(_HERE, 'build.py')}`; "
                           "there is no CPU fallback")
    L = C.CDLL(LIB_PATH)
    vp = C.c_void_p
    L.gi_graph_create.argtypes = [C.POINTER(vp), C.c_int32, C.c_int32]
    L.gi_graph_input.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
    L.gi_add_op.argtypes = [vp, C.POINTER(gi_op_desc), C.POINTER(C.c_int32)]
    L.gi_graph_output.argtypes = [vp, C.c_int32, C.c_int32]
    L.gi_graph_destroy.argtypes = [vp]
    L.gi_graph_destroy.restype = None
    L.gi_compile.argtypes = [vp, C.POINTER(gi_compile_options), C.POINTER(vp)]
    L.gi_exec_query.argtypes = [vp, C.POINTER(gi_exec_info)]
    L.gi_exec_tensor.argtypes = [vp, C.c_int32, C.POINTER(gi_tensor_info)]
    L.gi_exec_op.argtypes = [vp, C.c_int32, C.POINTER(gi_op_info)]
    L.gi_exec_launch.argtypes = [vp, C.c_int32, C.POINTER(gi_launch_info)]
    L.gi_exec_launch.restype = C.c_int32
    L.gi_exec_bind.argtypes = [vp, vp, C.c_size_t, vp]
    L.gi_run.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp, C.c_size_t, vp]
    L.gi_run_static.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp]
    L.gi_run_static.restype = C.c_int32
    L.gi_run_timed.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp, C.c_size_t, vp, C.POINTER(C.c_float), C.c_int32]
    L.gi_device_status.argtypes = [C.POINTER(C.c_uint32)]
    L.gi_device_status.restype = C.c_int32
    L.gi_selftest_bounded_wait.argtypes = [C.c_uint32, C.POINTER(C.c_uint32), C.POINTER(C.c_int32), vp]
    L.gi_selftest_bounded_wait.restype = C.c_int32
    L.gi_exec_destroy.argtypes = [vp]
    L.gi_exec_destroy.restype = None
    L.gi_slice8_tensor_bytes.argtypes = [C.c_int32] * 4
    L.gi_slice8_tensor_bytes.restype = C.c_uint64
    L.gi_slice8_pointwise_blob_bytes.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_uint64)]
    L.gi_slice8_pointwise_blob_bytes.restype = C.c_int32
    L.gi_slice8_pointwise_pack.argtypes = [vp, vp, C.c_int32, C.c_int32, vp, C.c_uint64]
    L.gi_slice8_pointwise_pack.restype = C.c_int32
    L.gi_slice8_pointwise_run.argtypes = [vp, vp, vp] + [C.c_int32] * 6 + [vp]
    L.gi_slice8_pointwise_run.restype = C.c_int32
    L.gi_linear_q4_blob_bytes.argtypes = [C.POINTER(gi_linear_q4), C.POINTER(C.c_uint64)]
    L.gi_linear_q4_blob_bytes.restype = C.c_int32
    L.gi_linear_q4_pack.argtypes = [C.POINTER(gi_linear_q4), vp, vp, vp, vp, vp, C.c_uint64]
    L.gi_linear_q4_pack.restype = C.c_int32
    L.gi_linear_q4_pack_device.argtypes = [C.POINTER(gi_linear_q4), vp, vp, vp, vp, vp, C.c_uint64, vp]
    L.gi_linear_q4_pack_device.restype = C.c_int32
    L.gi_linear_q4_run.argtypes = [C.POINTER(gi_linear_q4), vp, vp, C.c_int64, vp, C.c_int64, C.c_int32, vp]
    L.gi_linear_q4_run.restype = C.c_int32
    L.gi_log_probs.argtypes = [C.POINTER(gi_log_probs_desc)] + [vp] * 7
    L.gi_log_probs.restype = C.c_int32
    L.gi_status_str.argtypes = [C.c_int32]
    L.gi_status_str.restype = C.c_char_p
    L.gi_last_error.argtypes = []
    L.gi_last_error.restype = C.c_char_p
    L.gi_tensor_bytes.argtypes = [C.c_int32] * 6
    L.gi_tensor_bytes.restype = C.c_uint64
    L.gi_f32_to_f16.argtypes = [vp, vp, C.c_size_t]
    L.gi_f32_to_f16.restype = None
    for name in ("gi_graph_create", "gi_graph_input", "gi_add_op", "gi_graph_output", "gi_compile", "gi_exec_query",
                 "gi_exec_tensor", "gi_exec_op", "gi_exec_bind", "gi_run", "gi_run_timed"):
        getattr(L, name).restype = C.c_int32
    _lib = L
    return L


def _check(status: int, where: str) -> None:
    if status != GI_OK:
        L = lib()
        raise GiError(status, f"{where} [{L.gi_status_str(status).decode()}]", L.gi_last_error().decode())


def gi_tensor_bytes(batch, H, W, Cc, storage=GI_F16, align=256) -> int:
    return int(lib().gi_tensor_bytes(batch, H, W, Cc, storage, align))


def gi_f32_to_f16(x: np.ndarray) -> np.ndarray:
    x = np.ascontiguousarray(x, dtype=np.float32)
    out = np.empty(x.shape, dtype=np.uint16)
    lib().gi_f32_to_f16(x.ctypes.data, out.ctypes.data, x.size)
    return out


def gi_device_status() -> int:
    flags = C.c_uint32(0)
    _check(lib().gi_device_status(C.byref(flags)), "gi_device_status")
    return int(flags.value)


def gi_selftest_bounded_wait(limit_us: int, stream=None):
    """-> (microseconds the wait lasted on the device, True if it ended by running out)."""
    waited, gave_up = C.c_uint32(0), C.c_int32(0)
    _check(lib().gi_selftest_bounded_wait(limit_us, C.byref(waited), C.byref(gave_up), _stream_ptr(stream)), "gi_selftest_bounded_wait")
    return int(waited.value), bool(gave_up.value)


def gi_slice8_tensor_bytes(batch, H, W, Cc) -> int:
    return int(lib().gi_slice8_tensor_bytes(batch, H, W, Cc))


def gi_slice8_pointwise_pack(w: np.ndarray, bias: np.ndarray) -> np.ndarray:
    """Packed weights + bias (uint8 array) of a 1x1 layer w[cout, cin] for gi_slice8_pointwise_run."""
    w = np.ascontiguousarray(w, dtype=np.float32)
    bias = np.ascontiguousarray(bias, dtype=np.float32)
    cout, cin = w.shape
    n = C.c_uint64(0)
    _check(lib().gi_slice8_pointwise_blob_bytes(cin, cout, C.byref(n)), "gi_slice8_pointwise_blob_bytes")
    blob = np.zeros(int(n.value), dtype=np.uint8)
    _check(lib().gi_slice8_pointwise_pack(w.ctypes.data, bias.ctypes.data, cin, cout, blob.ctypes.data, blob.size), "gi_slice8_pointwise_pack")
    return blob


def gi_slice8_pointwise_run(dev_in: int, dev_out: int, dev_blob: int, batch, H, W, cin, cout, act, stream=None) -> None:
    """Argument marshalling only: the three pointers are device addresses (torch tensors' data_ptr())."""
    _check(lib().gi_slice8_pointwise_run(dev_in, dev_out, dev_blob, batch, H, W, cin, cout, act, _stream_ptr(stream)), "gi_slice8_pointwise_run")


def _torch_dtype(dtype: int):
    import torch
    return {GI_F16: torch.float16, GI_BF16: torch.bfloat16, GI_F32: torch.float32}[dtype]


_GI_DTYPES = {}


def _gi_dtype(t) -> int:
    """GI_* of a torch tensor's element type (0 where the library has none)."""
    if not _GI_DTYPES:
        import torch
        _GI_DTYPES.update({torch.float16: GI_F16, torch.bfloat16: GI_BF16, torch.float32: GI_F32})
    return _GI_DTYPES.get(t.dtype, 0)


def _weights(t, what: str, dtypes, shape):
    """`t` (torch tensor on any device, or numpy array) as a contiguous tensor, checked to be one of `dtypes` and of `shape`."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(t)) if isinstance(t, np.ndarray) else t
    if t.dtype not in dtypes or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: need {' or '.join(str(d) for d in dtypes)} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return t.detach().contiguous()


def _rows(t, what: str, dtype, channels: int, device):
    """(pointer, elements between rows, rows) of a device tensor [..., channels] whose leading axes form rows at one pitch."""
    shape = t.shape
    if t.dtype is not dtype or t.device != device or not shape or shape[-1] != channels:
        raise ValueError(f"{what}: need {dtype} of shape [..., {channels}] on {device}, got {t.dtype} {tuple(shape)} on {t.device}")
    if len(shape) == 2:
        pitch, step = t.stride()
        if step == 1 or channels == 1:
            return t.data_ptr(), pitch, shape[0]
    elif t.is_contiguous():
        return t.data_ptr(), channels, t.numel() // channels
    raise ValueError(f"{what}: channels must be contiguous, and all of a tensor of other than two axes (strides {t.stride()})")


def _values(t, what: str, n: int, dtype, device) -> int:
    """Pointer of a contiguous device tensor of n values."""
    if t is None:
        raise ValueError(f"{what}: missing")
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what}: need {n} contiguous values of {dtype} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _on(device, stream, call, *args) -> int:
    """call(*args, stream handle) with `device` current: the library launches on the current device."""
    import torch
    index = device.index
    if stream is None:
        # (the handle alone: torch.cuda.current_stream() takes 2 us to make a Stream of it, a quarter of a small call)
        handle = torch._C._cuda_getCurrentRawStream(index)
    else:
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if torch.cuda.current_device() == index:
        return call(*args, handle)
    with torch.cuda.device(device):
        return call(*args, handle)


def _allocating_on(stream, device):
    """Tensors made in this context belong to `stream` (a torch Stream, or the handle of one): nobody else is given their memory while
    it still uses it."""
    import contextlib
    import torch
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream_ptr(stream)
        stream = torch.cuda.ExternalStream(handle, device) if handle else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


class LinearQ4:
    """gi_linear_q4_*: a fully connected layer with 4-bit weights, kept on a device.

    q [cout, (cin + 1) / 2] uint8, two values a byte, the even input channel in the low half; scales [cout, ceil(cin / group)] float16,
    bfloat16 or float32; zeros (optional, else 8 everywhere) uint8 of the scales' shape, 0 .. 15; bias (optional) [cout] float32.
    Tensors on any device, or numpy arrays; they are copied: packed on the layer's device where all of them are there (on its current
    stream), else on the host.  `dtype` is the type of the rows that run() takes and returns.
    """

    def __init__(self, q, scales, zeros=None, bias=None, *, cin: int, group: int, dtype: int = GI_F16, act: int = GI_ACT_NONE,
                 device="cuda:0"):
        import torch
        cout, groups = int(q.shape[0]), -(-cin // group) if group > 0 else 0
        q = _weights(q, "q", (torch.uint8,), (cout, (cin + 1) // 2))
        scales = _weights(scales, "scales", (torch.float16, torch.bfloat16, torch.float32), (cout, groups))
        zeros = None if zeros is None else _weights(zeros, "zeros", (torch.uint8,), (cout, groups))
        bias = None if bias is None else _weights(bias, "bias", (torch.float32,), (cout,))
        self.desc = gi_linear_q4(cin, cout, group, _gi_dtype(scales), 0 if zeros is None else 1, dtype, act)
        self._ref = C.byref(self.desc)
        n = C.c_uint64(0)
        _check(lib().gi_linear_q4_blob_bytes(self._ref, C.byref(n)), "gi_linear_q4_blob_bytes")
        parts = [t for t in (q, scales, zeros, bias) if t is not None]
        device = torch.empty(0, device=device).device

        def pointers(ts):
            return [None if t is None else t.data_ptr() for t in ts]
        if device.type == "cuda" and all(t.device == device for t in parts):
            if zeros is not None and bool((zeros > 15).any()):
                raise ValueError("zeros: 0 .. 15")
            self.blob = torch.empty(int(n.value), dtype=torch.uint8, device=device)
            _check(_on(device, None, lib().gi_linear_q4_pack_device, self._ref, *pointers((q, scales, zeros, bias)), self.blob.data_ptr(), self.blob.numel()),
                   "gi_linear_q4_pack_device")
        else:
            host = [None if t is None else t.cpu() for t in (q, scales, zeros, bias)]
            blob = torch.empty(int(n.value), dtype=torch.uint8)
            _check(lib().gi_linear_q4_pack(self._ref, *pointers(host), blob.data_ptr(), blob.numel()), "gi_linear_q4_pack")
            self.blob = blob.to(device)
        self.cin, self.cout, self.dtype = cin, cout, _torch_dtype(dtype)
        self.device = self.blob.device
        self._run = lib().gi_linear_q4_run

    @property
    def _blob(self) -> int:
        return self.blob.data_ptr()

    def run(self, x, y=None, stream=None):
        """y[..., cout] = act(x[..., cin] w^T + bias) on `stream` (default: the current one of the layer's device); y is made where none is given.
        Two axes may have any distance between rows; other tensors are contiguous."""
        if self.device.type != "cuda":
            raise ValueError(f"the layer is in host memory: need one on a CUDA device ({self.device})")
        if y is None:
            import torch
            with _allocating_on(stream, self.device):
                y = torch.empty(tuple(x.shape[:-1]) + (self.cout,), dtype=self.dtype, device=self.device)
        xp, ldx, rows = _rows(x, "x", self.dtype, self.cin, self.device)
        yp, ldy, yrows = _rows(y, "y", self.dtype, self.cout, self.device)
        if rows != yrows:
            raise ValueError(f"x has {rows} rows, y {yrows}")
        status = _on(self.device, stream, self._run, self._ref, self._blob, xp, ldx, yp, ldy, rows)
        if status != GI_OK:
            _check(status, "gi_linear_q4_run")
        return y


class LogProbs(NamedTuple):
    """Results of log_probs for rows of logits; None where nothing was asked for."""
    given: Any     # [rows, n] float32: log probabilities of the given classes
    entropy: Any   # [rows] float32
    top: Any       # [rows, top] float32: log probabilities of the most probable classes, the most probable first
    top_ids: Any   # [rows, top] int32: these classes


def log_probs_out(rows: int, n_given: int = 0, top: int = 0, device="cuda:0", entropy: bool = True) -> LogProbs:
    """Result buffers for log_probs."""
    import torch

    def new(n, dtype):
        return torch.empty((rows, n), dtype=dtype, device=device) if n else None
    return LogProbs(new(n_given, torch.float32), torch.empty((rows,), dtype=torch.float32, device=device) if entropy else None,
                    new(top, torch.float32), new(top, torch.int32))


def log_probs(logits, given=None, top: int = 0, temperature: float = 1.0, out: Optional[LogProbs] = None, stream=None) -> LogProbs:
    """gi_log_probs: logits [..., classes] (float16, bfloat16, float32; two axes may have any distance between rows, other tensors are
    contiguous) -> log probabilities of `given` (int32 [..., n], negative: nothing asked), entropy and the `top` leading classes of
    each row, in `out` (log_probs_out; what is not asked for is left as it is there, and None in the result) or in new tensors."""
    import torch
    device = logits.device
    if device.type != "cuda":
        raise ValueError("logits: need a tensor on a CUDA device")
    if not logits.shape or not logits.shape[-1]:
        raise ValueError(f"logits: need [..., classes] with at least one class, got {tuple(logits.shape)}")
    classes = logits.shape[-1]
    ptr, ld, rows = _rows(logits, "logits", logits.dtype, classes, device)
    n_given = 0 if given is None else given.shape[-1]
    if out is None:
        with _allocating_on(stream, device):
            out = log_probs_out(rows, n_given, top, device)

    f32, i32 = torch.float32, torch.int32
    gp = op = ep = ip = tp = None
    if n_given:
        gp, op = _values(given, "given", rows * n_given, i32, device), _values(out.given, "out.given", rows * n_given, f32, device)
    if out.entropy is not None:
        ep = _values(out.entropy, "out.entropy", rows, f32, device)
    if top:
        ip, tp = _values(out.top_ids, "out.top_ids", rows * top, i32, device), _values(out.top, "out.top", rows * top, f32, device)
    d = gi_log_probs_desc(rows, classes, ld, _gi_dtype(logits), temperature, n_given, top)
    status = _on(device, stream, lib().gi_log_probs, C.byref(d), ptr, gp, op, ep, ip, tp)
    if status != GI_OK:
        _check(status, "gi_log_probs")
    if (not n_given and out.given is not None) or (not top and (out.top is not None or out.top_ids is not None)):
        out = out._replace(given=out.given if n_given else None, top=out.top if top else None, top_ids=out.top_ids if top else None)
    return out


class Graph:
    """gi_graph_create / gi_graph_input / gi_add_op / gi_graph_output."""

    def __init__(self, batch: int, storage: int = GI_F16):
        self._h = C.c_void_p()
        _check(lib().gi_graph_create(C.byref(self._h), batch, storage), "gi_graph_create")
        self.batch, self.storage = batch, storage

    def __del__(self):
        if getattr(self, "_h", None) is not None and self._h and _lib is not None:
            _lib.gi_graph_destroy(self._h)
            self._h = None

    def input(self, H: int, W: int, Cc: int, layout: int = GI_NHWC) -> int:
        t = C.c_int32(-1)
        _check(lib().gi_graph_input(self._h, H, W, Cc, layout, C.byref(t)), "gi_graph_input")
        return t.value

    def add_op(self, desc: gi_op_desc) -> int:
        t = C.c_int32(-1)
        _check(lib().gi_add_op(self._h, C.byref(desc), C.byref(t)), "gi_add_op")
        return t.value

    def output(self, t: int, layout: int = GI_NHWC) -> None:
        _check(lib().gi_graph_output(self._h, t, layout), "gi_graph_output")

    def compile(self, planner: int = GI_PLAN_GREEDY_BY_SIZE, fuse: bool = True, align: int = 256,
                pointwise: int = GI_PW_AUTO, cross_op: int = GI_XOP_AUTO) -> "Executable":
        opt = gi_compile_options(planner, 1 if fuse else 0, align, pointwise, cross_op)
        h = C.c_void_p()
        _check(lib().gi_compile(self._h, C.byref(opt), C.byref(h)), "gi_compile")
        return Executable(h, self)


def graph_from_spec(spec: wl.GraphSpec, storage: int = GI_F16, io_layout: int = GI_NHWC, out_layout: int = None):
    """Build a gi graph from a workload description.  Returns (Graph, {spec tensor id -> gi tensor id}).
    `io_layout` is the layout of the graph's inputs and, unless `out_layout` is given, of its outputs."""
    out_layout = io_layout if out_layout is None else out_layout
    g = Graph(spec.batch, storage)
    ids = {}
    for t in spec.inputs:
        H, W, Cc = spec.shapes[t]
        ids[t] = g.input(H, W, Cc, io_layout)
    for op in spec.ops:
        d = gi_op_desc()
        d.kind = _KIND[op.kind]
        d.inputs[0] = ids[op.inputs[0]]
        d.inputs[1] = ids[op.inputs[1]] if len(op.inputs) > 1 else -1
        keep = []
        if op.kind in (wl.CONV2D, wl.DEPTHWISE):
            d.kh, d.kw = op.kh, op.kw
            d.stride_h, d.stride_w = op.stride
            d.dilation_h, d.dilation_w = op.dilation
            d.pad_t, d.pad_l, d.pad_b, d.pad_r = op.pads
            d.cout = op.cout
            if op.q4 is not None:
                q, s = np.ascontiguousarray(op.q4.q, dtype=np.uint8), np.ascontiguousarray(op.q4.scales)
                z = None if op.q4.zeros is None else np.ascontiguousarray(op.q4.zeros, dtype=np.uint8)
                kind = {np.dtype(np.float16): GI_F16, np.dtype(np.float32): GI_F32}[s.dtype]
                w4 = gi_q4_weights(q.ctypes.data, s.ctypes.data, None if z is None else z.ctypes.data, kind, op.q4.group)
                keep += [q, s, z, w4]
                d.weight_dtype = GI_Q4
                d.weights = C.addressof(w4)
            else:
                w = np.ascontiguousarray(op.weights, dtype=np.float32)
                keep.append(w)
                d.weight_dtype = GI_F32
                d.weights = w.ctypes.data
            if op.bias is not None:
                b = np.ascontiguousarray(op.bias, dtype=np.float32)
                keep.append(b)
                d.bias = b.ctypes.data
        elif op.kind == wl.ACTIVATION:
            d.act = _ACT[op.act]
        elif op.kind == wl.RESIZE_BILINEAR:
            d.out_h, d.out_w = op.out_hw
            d.align_corners = 1 if op.align_corners else 0
        ids[op.output] = g.add_op(d)
        del keep
    for t in spec.outputs:
        g.output(ids[t], out_layout)
    return g, ids


class Executable:
    """gi_exec_*: query, bind weights, run.  Device buffers are torch tensors owned here or by the caller."""

    def __init__(self, handle: C.c_void_p, graph: Graph):
        self._h = handle
        self.graph = graph
        self.info = gi_exec_info()
        _check(lib().gi_exec_query(self._h, C.byref(self.info)), "gi_exec_query")
        self._weights = None
        self._arena = None

    def __del__(self):
        if getattr(self, "_h", None) is not None and self._h and _lib is not None:
            _lib.gi_exec_destroy(self._h)
            self._h = None

    def tensor(self, t: int) -> gi_tensor_info:
        ti = gi_tensor_info()
        _check(lib().gi_exec_tensor(self._h, t, C.byref(ti)), "gi_exec_tensor")
        return ti

    def op(self, i: int) -> gi_op_info:
        oi = gi_op_info()
        _check(lib().gi_exec_op(self._h, i, C.byref(oi)), "gi_exec_op")
        return oi

    def ops(self) -> List[gi_op_info]:
        return [self.op(i) for i in range(self.info.n_ops)]

    def launch(self, i: int) -> gi_launch_info:
        """What gi_run launches at executed op i (kernel "none": nothing, another launch covers it)."""
        li = gi_launch_info()
        _check(lib().gi_exec_launch(self._h, i, C.byref(li)), "gi_exec_launch")
        return li

    def launches(self) -> List[gi_launch_info]:
        return [self.launch(i) for i in range(self.info.n_ops)]

    # -- device side -------------------------------------------------------------------
    def bind(self, device="cuda:0", stream=None) -> None:
        """Allocate the weight blob and the arena as torch tensors and upload the packed weights."""
        import torch
        self._weights = torch.empty(max(int(self.info.weight_bytes), 256), dtype=torch.uint8, device=device)
        self._arena = torch.empty(max(int(self.info.arena_bytes), 256), dtype=torch.uint8, device=device)
        self.bind_raw(self._weights.data_ptr(), self._weights.numel(), stream)

    def bind_raw(self, dev_weights: int, nbytes: int, stream=None) -> None:
        _check(lib().gi_exec_bind(self._h, dev_weights, nbytes, _stream_ptr(stream)), "gi_exec_bind")

    @property
    def arena(self):
        return self._arena

    def run_raw(self, in_ptrs: Sequence[int], out_ptrs: Sequence[int], arena_ptr: int, arena_bytes: int,
                stream=None) -> None:
        ins = (C.c_void_p * max(len(in_ptrs), 1))(*in_ptrs)
        outs = (C.c_void_p * max(len(out_ptrs), 1))(*out_ptrs)
        _check(lib().gi_run(self._h, ins, outs, arena_ptr, arena_bytes, _stream_ptr(stream)), "gi_run")

    def run_static(self, inputs, outputs, stream=None) -> None:
        """gi_run_static: intermediates in the library's built-in arena; allocates nothing."""
        ins = (C.c_void_p * max(len(inputs), 1))(*[t.data_ptr() for t in inputs])
        outs = (C.c_void_p * max(len(outputs), 1))(*[t.data_ptr() for t in outputs])
        _check(lib().gi_run_static(self._h, ins, outs, _stream_ptr(stream)), "gi_run_static")

    def run_timed(self, inputs, outputs, stream=None) -> List[float]:
        """gi_run_timed: one run with an event around every executed op; returns per-op milliseconds."""
        n = int(self.info.n_ops)
        ms = (C.c_float * n)()
        ins = (C.c_void_p * max(len(inputs), 1))(*[t.data_ptr() for t in inputs])
        outs = (C.c_void_p * max(len(outputs), 1))(*[t.data_ptr() for t in outputs])
        _check(lib().gi_run_timed(self._h, ins, outs, self._arena.data_ptr(), self._arena.numel(), _stream_ptr(stream),
                                  ms, n), "gi_run_timed")
        return list(ms)

    def run(self, inputs, outputs, stream=None) -> None:
        """inputs / outputs: torch CUDA tensors in the declared layouts (contiguous, storage dtype)."""
        self.run_raw([t.data_ptr() for t in inputs], [t.data_ptr() for t in outputs], self._arena.data_ptr(),
                     self._arena.numel(), stream)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        if torch.cuda.is_available():
            return torch.cuda.current_stream().cuda_stream
        return None
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
