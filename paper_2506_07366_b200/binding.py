"""ctypes binding of libmoegps.so: argument marshalling only.

Every function here has the name of the C entry point it forwards to (include/moegps.h); tensors are
torch CUDA tensors of which only `data_ptr()` crosses the boundary.  There is no CPU path: if the
shared library is missing or cannot be loaded the import of this module raises.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os

import torch

from . import build as _build

_c_int32_p = ctypes.POINTER(ctypes.c_int32)


class moegps_shape_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("T", "D", "F", "E", "K", "S", "gate_mode", "row_align", "c_max")]


@dataclasses.dataclass(frozen=True)
class Shape:
    T: int
    D: int
    F: int
    E: int
    K: int
    S: int
    gate_mode: int = 0
    row_align: int = 128
    c_max: int = 0

    @property
    def R(self) -> int:
        return self.T * self.K

    @property
    def Rcap(self) -> int:
        return self.T * self.K + self.S * (self.row_align - 1)

    @property
    def P(self) -> int:
        """Columns of a row of 8-bit activations: F rounded up to whole blocks of 32."""
        return (self.F + 31) // 32 * 32

    def w4_shapes(self, down: bool = False):
        """Shapes of 4-bit expert matrices: (codes, scales), both uint8.  down False: gate or up [E, F, D]; True: [E, D, F]."""
        n, c = (self.D, self.F) if down else (self.F, self.D)
        tiles, chunks = (n + 127) // 128, (c + 127) // 128
        return (self.E, n, 64 * chunks), (self.E, tiles, chunks, 512)

    def c_struct(self) -> moegps_shape_t:
        return moegps_shape_t(*(getattr(self, f[0]) for f in moegps_shape_t._fields_))


OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED_SHAPE, ERR_WORKSPACE_TOO_SMALL, ERR_CUDA = -1, -2, -3, -4
ERR_UNIMPLEMENTED, ERR_BAD_INDEX, ERR_TIMEOUT, ERR_HIST_MISMATCH = -5, -6, -7, -8
ERR_STATIC_SCRATCH_EXCEEDED = -9

EXPORTS = (
    "moegps_create", "moegps_destroy", "moegps_rcap", "moegps_workspace_bytes", "moegps_route",
    "moegps_route_histogram", "moegps_route_prepare", "moegps_dispatch_prepared", "moegps_route_logits", "moegps_histogram", "moegps_plan", "moegps_pack", "moegps_pack_slots", "moegps_dispatch", "moegps_dispatch_shares", "moegps_dispatch_static",
    "moegps_expert_ffn", "moegps_expert_ffn_gate_up", "moegps_expert_ffn_down", "moegps_combine",
    "moegps_status", "moegps_launch_count", "moegps_last_cuda_error", "moegps_error_string",
    "moegps_selftest_bounded_wait", "moegps_predictor_update", "moegps_predictor_update_ema", "moegps_error_rate",
    "moegps_expert_ffn_gate_up_save", "moegps_expert_ffn_backward", "moegps_expert_ffn_backward_act",
    "moegps_expert_ffn_backward_input", "moegps_expert_ffn_backward_weights", "moegps_combine_backward",
    "moegps_dispatch_backward", "moegps_route_backward", "moegps_route_backward_workspace_bytes",
    "moegps_weights4_bytes", "moegps_weights4_scale_bytes", "moegps_weights_quantize4", "moegps_weights_dequantize4",
    "moegps_expert_ffn4", "moegps_expert_ffn4_workspace_bytes",
)


class MoegpsError(RuntimeError):
    def __init__(self, code: int, where: str, cuda_error: int = 0):
        self.code = code
        msg = _lib().moegps_error_string(code).decode()
        if cuda_error:
            msg += f" (cudaError {cuda_error})"
        super().__init__(f"{where}: {msg} [{code}]")


_LIB = None


def library_path() -> str:
    """The in-tree build, unless MOEGPS_LIBRARY names another build of the same library."""
    return os.environ.get("MOEGPS_LIBRARY") or _build.LIB_PATH


def _lib():
    """Loads libmoegps.so (never builds it implicitly on a machine without nvcc; never falls back)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2506_07366_b200.build` "
                          "(there is no fallback path)")
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    sig = {
        "moegps_create": (ctypes.c_int, [ctypes.POINTER(vp), ctypes.POINTER(moegps_shape_t), ctypes.c_int]),
        "moegps_destroy": (ctypes.c_int, [vp]),
        "moegps_rcap": (i64, [ctypes.POINTER(moegps_shape_t)]),
        "moegps_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(moegps_shape_t)]),
        "moegps_route": (ctypes.c_int, [vp] * 7),
        "moegps_route_histogram": (ctypes.c_int, [vp] * 8),
        "moegps_route_prepare": (ctypes.c_int, [vp] * 9),
        "moegps_dispatch_prepared": (ctypes.c_int, [vp] * 12),
        "moegps_route_logits": (ctypes.c_int, [vp] * 6),
        "moegps_histogram": (ctypes.c_int, [vp] * 4),
        "moegps_plan": (ctypes.c_int, [vp, vp, i32, vp, vp, vp, vp, vp]),
        "moegps_pack": (ctypes.c_int, [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]),
        "moegps_pack_slots": (ctypes.c_int, [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]),
        "moegps_dispatch": (ctypes.c_int, [vp] * 12),
        "moegps_dispatch_shares": (ctypes.c_int, [vp] * 13),
        "moegps_dispatch_static": (ctypes.c_int, [vp] * 11),
        "moegps_expert_ffn": (ctypes.c_int, [vp] * 10),
        "moegps_expert_ffn_gate_up": (ctypes.c_int, [vp] * 8),
        "moegps_expert_ffn_down": (ctypes.c_int, [vp] * 7),
        "moegps_combine": (ctypes.c_int, [vp] * 6),
        "moegps_expert_ffn_gate_up_save": (ctypes.c_int, [vp] * 12),
        "moegps_expert_ffn_backward": (ctypes.c_int, [vp] * 22),
        "moegps_expert_ffn_backward_act": (ctypes.c_int, [vp] * 13),
        "moegps_expert_ffn_backward_input": (ctypes.c_int, [vp] * 9),
        "moegps_expert_ffn_backward_weights": (ctypes.c_int, [vp] * 13),
        "moegps_combine_backward": (ctypes.c_int, [vp] * 8),
        "moegps_dispatch_backward": (ctypes.c_int, [vp] * 8),
        "moegps_route_backward": (ctypes.c_int, [vp] * 15),
        "moegps_route_backward_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(moegps_shape_t)]),
        "moegps_weights4_bytes": (ctypes.c_size_t, [ctypes.POINTER(moegps_shape_t), i32]),
        "moegps_weights4_scale_bytes": (ctypes.c_size_t, [ctypes.POINTER(moegps_shape_t), i32]),
        "moegps_weights_quantize4": (ctypes.c_int, [vp, vp, i32, vp, vp, vp]),
        "moegps_weights_dequantize4": (ctypes.c_int, [vp, vp, vp, i32, vp, vp]),
        "moegps_expert_ffn4": (ctypes.c_int, [vp] * 13),
        "moegps_expert_ffn4_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(moegps_shape_t)]),
        "moegps_selftest_bounded_wait": (ctypes.c_int, [vp, i64, vp]),
        "moegps_predictor_update": (ctypes.c_int, [vp] * 5),
        "moegps_predictor_update_ema": (ctypes.c_int, [vp, vp, vp, i32, vp, vp]),
        "moegps_error_rate": (ctypes.c_int, [vp] * 5),
        "moegps_status": (ctypes.c_int, [vp, vp, _c_int32_p]),
        "moegps_launch_count": (i64, [vp]),
        "moegps_last_cuda_error": (ctypes.c_int, [vp]),
        "moegps_error_string": (ctypes.c_char_p, [ctypes.c_int]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)          # AttributeError if the library does not export it
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


def _ptr(t, dtype, shape, name, allow_none=False):
    """Device address of a tensor that is what the call needs, else an exception that says what is wrong.  A call's
    tensors are checked one by one in front of a launch of a few microseconds, so the usual case is one expression."""
    try:
        if t.is_cuda and t.dtype is dtype and (shape is None or t.shape == shape) and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    if t is None:
        if allow_none:
            return None
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _stream(stream):
    if stream is None:
        # the handle alone: torch.cuda.current_stream() builds an object around it
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    if hasattr(stream, "cuda_stream"):
        return int(stream.cuda_stream)
    try:
        return int(stream)                               # a handle
    except TypeError:
        raise AttributeError(f"{stream!r} is neither a stream nor a stream's handle") from None


def _marshal():
    """The compiled argument checks (csrc/marshal.cpp), or None where they have not been built for this torch."""
    try:
        from . import _marshal as module
    except ImportError:
        return None
    return module if getattr(module, "built_for", None) == _build.marshal_marker() else None


def _training_call(entry, handle: int, specs):
    """A callable (stream, *tensors) that checks every tensor against its spec (type, shape, name, may be None), calls the C
    entry point and returns its code.  The compiled form costs a few microseconds less for each call; both raise the
    exceptions of _ptr."""
    module = _marshal()
    if module is not None:
        return module.Call(ctypes.cast(entry, ctypes.c_void_p).value, handle, _ptr, tuple(specs))

    def run(stream, *tensors):
        if len(tensors) != len(specs):
            raise TypeError(f"expected a stream and {len(specs)} tensors")
        return entry(handle, *[_ptr(t, *spec) for t, spec in zip(tensors, specs)], _stream(stream))

    return run


class Context:
    """Owns one moegps_ctx_t.  Methods carry the C names without the prefix."""

    def __init__(self, shape: Shape, device: int | None = None):
        lib = _lib()
        if not torch.cuda.is_available():
            raise RuntimeError("moegps needs a CUDA device (sm_100a); there is no CPU path")
        self.shape = shape
        self.device = torch.cuda.current_device() if device is None else int(device)
        self._h = ctypes.c_void_p()
        cs = shape.c_struct()
        rc = lib.moegps_create(ctypes.byref(self._h), ctypes.byref(cs), self.device)
        if rc != OK:
            self._h = ctypes.c_void_p()
            raise MoegpsError(rc, "moegps_create")
        self._bind_training_calls()

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            _lib().moegps_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._bind_training_calls()                  # to the null context, which every entry point refuses

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, where):
        if rc != OK:
            raise MoegpsError(rc, where, _lib().moegps_last_cuda_error(self._h))

    # -- the six steps ------------------------------------------------------------------------
    def route(self, x, w_router, bias, topk_idx, topk_w, stream=None):
        s = self.shape
        self._check(_lib().moegps_route(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(w_router, torch.bfloat16, (s.E, s.D), "w_router"),
            _ptr(bias, torch.float32, (s.E,), "bias", allow_none=True),
            _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(topk_w, torch.float32, (s.T, s.K), "topk_w"), _stream(stream)), "moegps_route")

    def route_histogram(self, x, w_router, bias, topk_idx, topk_w, hist, stream=None):
        s = self.shape
        self._check(_lib().moegps_route_histogram(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(w_router, torch.bfloat16, (s.E, s.D), "w_router"),
            _ptr(bias, torch.float32, (s.E,), "bias", allow_none=True),
            _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(topk_w, torch.float32, (s.T, s.K), "topk_w"),
            _ptr(hist, torch.int32, (s.E,), "hist"), _stream(stream)), "moegps_route_histogram")

    def route_prepare(self, x, w_router, bias, topk_idx, topk_w, hist, workspace, stream=None):
        s = self.shape
        if workspace is None or workspace.numel() * workspace.element_size() < workspace_bytes(s):
            raise MoegpsError(ERR_WORKSPACE_TOO_SMALL, "moegps_route_prepare")
        self._check(_lib().moegps_route_prepare(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(w_router, torch.bfloat16, (s.E, s.D), "w_router"),
            _ptr(bias, torch.float32, (s.E,), "bias", allow_none=True),
            _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(topk_w, torch.float32, (s.T, s.K), "topk_w"),
            _ptr(hist, torch.int32, (s.E,), "hist"),
            _ptr(workspace, workspace.dtype, None, "workspace"), _stream(stream)), "moegps_route_prepare")

    def dispatch_prepared(self, x, topk_idx, hist, replicas, slot_off, slot_row_off, row_pair, pair_row, xp,
                          workspace, stream=None):
        s = self.shape
        if workspace is None or workspace.numel() * workspace.element_size() < workspace_bytes(s):
            raise MoegpsError(ERR_WORKSPACE_TOO_SMALL, "moegps_dispatch_prepared")
        self._check(_lib().moegps_dispatch_prepared(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(hist, torch.int32, (s.E,), "hist"),
            _ptr(replicas, torch.int32, (s.E,), "replicas"),
            _ptr(slot_off, torch.int32, (s.E + 1,), "slot_off"),
            _ptr(slot_row_off, torch.int32, (s.S + 1,), "slot_row_off"),
            _ptr(row_pair, torch.int32, (s.Rcap,), "row_pair"),
            _ptr(pair_row, torch.int32, (s.T, s.K), "pair_row"),
            _ptr(xp, torch.bfloat16, (s.Rcap, s.D), "xp"),
            _ptr(workspace, workspace.dtype, None, "workspace"), _stream(stream)), "moegps_dispatch_prepared")

    def route_logits(self, x, w_router, bias, logits, stream=None):
        s = self.shape
        self._check(_lib().moegps_route_logits(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(w_router, torch.bfloat16, (s.E, s.D), "w_router"),
            _ptr(bias, torch.float32, (s.E,), "bias", allow_none=True),
            _ptr(logits, torch.float32, (s.T, s.E), "logits"), _stream(stream)), "moegps_route_logits")

    def histogram(self, topk_idx, hist, stream=None):
        s = self.shape
        self._check(_lib().moegps_histogram(
            self._h, _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(hist, torch.int32, (s.E,), "hist"), _stream(stream)), "moegps_histogram")

    def plan(self, predicted_hist, n_slots, replicas, slot_off, slot_expert, bound, stream=None):
        s = self.shape
        self._check(_lib().moegps_plan(
            self._h, _ptr(predicted_hist, torch.int32, (s.E,), "predicted_hist"), int(n_slots),
            _ptr(replicas, torch.int32, (s.E,), "replicas"),
            _ptr(slot_off, torch.int32, (s.E + 1,), "slot_off"),
            _ptr(slot_expert, torch.int32, (s.S,), "slot_expert"),
            _ptr(bound, torch.int32, (1,), "bound"), _stream(stream)), "moegps_plan")

    def pack(self, predicted_hist, home, capacity, n_devices, placement, share, load, iterations, stream=None):
        s, g = self.shape, int(n_devices)
        self._check(_lib().moegps_pack(
            self._h, _ptr(predicted_hist, torch.int32, (s.E,), "predicted_hist"),
            _ptr(home, torch.int32, (s.E,), "home"), _ptr(capacity, torch.int32, (g,), "capacity"), g,
            _ptr(placement, torch.int32, (s.E, g), "placement"), _ptr(share, torch.int32, (s.E, g), "share"),
            _ptr(load, torch.int32, (g,), "load"), _ptr(iterations, torch.int32, (1,), "iterations"),
            _stream(stream)), "moegps_pack")

    def pack_slots(self, placement, share, n_devices, replicas, slot_off, slot_expert, slot_share, slot_device,
                   stream=None):
        s, g = self.shape, int(n_devices)
        self._check(_lib().moegps_pack_slots(
            self._h, _ptr(placement, torch.int32, (s.E, g), "placement"), _ptr(share, torch.int32, (s.E, g), "share"), g,
            _ptr(replicas, torch.int32, (s.E,), "replicas"), _ptr(slot_off, torch.int32, (s.E + 1,), "slot_off"),
            _ptr(slot_expert, torch.int32, (s.S,), "slot_expert"), _ptr(slot_share, torch.int32, (s.S,), "slot_share"),
            _ptr(slot_device, torch.int32, (s.S,), "slot_device"), _stream(stream)), "moegps_pack_slots")

    def dispatch_shares(self, x, topk_idx, hist, replicas, slot_off, slot_share, slot_row_off, row_pair, pair_row,
                        xp, workspace, stream=None):
        s = self.shape
        if workspace is None or workspace.numel() * workspace.element_size() < workspace_bytes(s):
            raise MoegpsError(ERR_WORKSPACE_TOO_SMALL, "moegps_dispatch_shares")
        self._check(_lib().moegps_dispatch_shares(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(hist, torch.int32, (s.E,), "hist"),
            _ptr(replicas, torch.int32, (s.E,), "replicas"),
            _ptr(slot_off, torch.int32, (s.E + 1,), "slot_off"),
            _ptr(slot_share, torch.int32, (s.S,), "slot_share"),
            _ptr(slot_row_off, torch.int32, (s.S + 1,), "slot_row_off"),
            _ptr(row_pair, torch.int32, (s.Rcap,), "row_pair"),
            _ptr(pair_row, torch.int32, (s.T, s.K), "pair_row"),
            _ptr(xp, torch.bfloat16, (s.Rcap, s.D), "xp"),
            _ptr(workspace, workspace.dtype, None, "workspace"), _stream(stream)), "moegps_dispatch_shares")

    def dispatch(self, x, topk_idx, hist, replicas, slot_off, slot_row_off, row_pair, pair_row, xp,
                 workspace, stream=None):
        s = self.shape
        if workspace is None or workspace.numel() * workspace.element_size() < workspace_bytes(s):
            raise MoegpsError(ERR_WORKSPACE_TOO_SMALL, "moegps_dispatch")
        self._check(_lib().moegps_dispatch(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(hist, torch.int32, (s.E,), "hist"),
            _ptr(replicas, torch.int32, (s.E,), "replicas"),
            _ptr(slot_off, torch.int32, (s.E + 1,), "slot_off"),
            _ptr(slot_row_off, torch.int32, (s.S + 1,), "slot_row_off"),
            _ptr(row_pair, torch.int32, (s.Rcap,), "row_pair"),
            _ptr(pair_row, torch.int32, (s.T, s.K), "pair_row"),
            _ptr(xp, torch.bfloat16, (s.Rcap, s.D), "xp"),
            _ptr(workspace, workspace.dtype, None, "workspace"), _stream(stream)), "moegps_dispatch")

    def dispatch_static(self, x, topk_idx, hist, replicas, slot_off, slot_row_off, row_pair, pair_row, xp,
                        stream=None):
        """dispatch() for callers that cannot hand over a workspace (no allocator available where
        they run): the scratch is a fixed 1 MiB array inside the library, shared by every call on
        the device, so overlapping calls must be serialised; ceil(T*K/256)*E must be <= 262144.
        This method allocates nothing either."""
        s = self.shape
        self._check(_lib().moegps_dispatch_static(
            self._h, _ptr(x, torch.bfloat16, (s.T, s.D), "x"),
            _ptr(topk_idx, torch.int32, (s.T, s.K), "topk_idx"),
            _ptr(hist, torch.int32, (s.E,), "hist"),
            _ptr(replicas, torch.int32, (s.E,), "replicas"),
            _ptr(slot_off, torch.int32, (s.E + 1,), "slot_off"),
            _ptr(slot_row_off, torch.int32, (s.S + 1,), "slot_row_off"),
            _ptr(row_pair, torch.int32, (s.Rcap,), "row_pair"),
            _ptr(pair_row, torch.int32, (s.T, s.K), "pair_row"),
            _ptr(xp, torch.bfloat16, (s.Rcap, s.D), "xp"), _stream(stream)), "moegps_dispatch_static")

    def expert_ffn(self, xp, slot_row_off, slot_expert, w_gate, w_up, w_down, h_ws, yp, stream=None):
        s = self.shape
        self._check(_lib().moegps_expert_ffn(
            self._h, _ptr(xp, torch.bfloat16, (s.Rcap, s.D), "xp"),
            _ptr(slot_row_off, torch.int32, (s.S + 1,), "slot_row_off"),
            _ptr(slot_expert, torch.int32, (s.S,), "slot_expert"),
            _ptr(w_gate, torch.bfloat16, (s.E, s.F, s.D), "w_gate"),
            _ptr(w_up, torch.bfloat16, (s.E, s.F, s.D), "w_up"),
            _ptr(w_down, torch.bfloat16, (s.E, s.D, s.F), "w_down"),
            _ptr(h_ws, torch.bfloat16, (s.Rcap, s.F), "h_ws"),
            _ptr(yp, torch.bfloat16, (s.Rcap, s.D), "yp"), _stream(stream)), "moegps_expert_ffn")

    def expert_ffn_gate_up(self, xp, slot_row_off, slot_expert, w_gate, w_up, h_ws, stream=None):
        s = self.shape
        self._check(_lib().moegps_expert_ffn_gate_up(
            self._h, _ptr(xp, torch.bfloat16, (s.Rcap, s.D), "xp"),
            _ptr(slot_row_off, torch.int32, (s.S + 1,), "slot_row_off"),
            _ptr(slot_expert, torch.int32, (s.S,), "slot_expert"),
            _ptr(w_gate, torch.bfloat16, (s.E, s.F, s.D), "w_gate"),
            _ptr(w_up, torch.bfloat16, (s.E, s.F, s.D), "w_up"),
            _ptr(h_ws, torch.bfloat16, (s.Rcap, s.F), "h_ws"), _stream(stream)), "moegps_expert_ffn_gate_up")

    def expert_ffn_down(self, h_ws, slot_row_off, slot_expert, w_down, yp, stream=None):
        s = self.shape
        self._check(_lib().moegps_expert_ffn_down(
            self._h, _ptr(h_ws, torch.bfloat16, (s.Rcap, s.F), "h_ws"),
            _ptr(slot_row_off, torch.int32, (s.S + 1,), "slot_row_off"),
            _ptr(slot_expert, torch.int32, (s.S,), "slot_expert"),
            _ptr(w_down, torch.bfloat16, (s.E, s.D, s.F), "w_down"),
            _ptr(yp, torch.bfloat16, (s.Rcap, s.D), "yp"), _stream(stream)), "moegps_expert_ffn_down")

    def combine(self, yp, pair_row, topk_w, out, stream=None):
        s = self.shape
        self._check(_lib().moegps_combine(
            self._h, _ptr(yp, torch.bfloat16, (s.Rcap, s.D), "yp"),
            _ptr(pair_row, torch.int32, (s.T, s.K), "pair_row"),
            _ptr(topk_w, torch.float32, (s.T, s.K), "topk_w"),
            _ptr(out, torch.bfloat16, (s.T, s.D), "out"), _stream(stream)), "moegps_combine")

    # -- the training step --------------------------------------------------------------------
    def _bind_training_calls(self):
        """What each tensor of these calls has to be: (type, shape or None, name, may be None)."""
        s = self.shape
        bf16, i32, u8, f32 = torch.bfloat16, torch.int32, torch.uint8, torch.float32

        def t(name, dtype, *shape, optional=False):
            return (dtype, shape or None, name, optional)

        def rows(*names, width=None, dtype=bf16):
            return tuple(t(n, dtype, s.Rcap, width) for n in names)

        row_off, slot_off, expert = t("slot_row_off", i32, s.S + 1), t("slot_off", i32, s.E + 1), t("slot_expert", i32, s.S)
        row_pair, pair_row = t("row_pair", i32, s.Rcap), t("pair_row", i32, s.T, s.K)
        up = tuple(t(n, bf16, s.E, s.F, s.D) for n in ("w_gate", "w_up"))
        down = (t("w_down", bf16, s.E, s.D, s.F),)
        d_up = tuple(t(n, bf16, s.E, s.F, s.D) for n in ("dw_gate", "dw_up")) + (t("dw_down", bf16, s.E, s.D, s.F),)
        kept = rows("gate8", "up8", width=s.P, dtype=u8) + tuple(t(n, u8, s.P // 32, s.Rcap) for n in ("gate_scale", "up_scale"))
        mid, h = rows("dgate", "dup", width=s.F), rows("h_ws", width=s.F)
        xp, dyp, dxp, yp = (rows(n, width=s.D) for n in ("xp", "dyp", "dxp", "yp"))
        topk_idx, topk_w, dtopk_w, dlogit = (t(n, d, s.T, s.K) for n, d in
                                             (("topk_idx", i32), ("topk_w", f32), ("dtopk_w", f32), ("dlogit", f32)))
        w_router, dx = t("w_router", bf16, s.E, s.D), t("dx", bf16, s.T, s.D)
        softmax = s.gate_mode == 0                       # then w_router and topk_idx may be missing
        maybe = lambda spec: spec[:3] + (softmax,)  # noqa: E731

        def call(name, *specs):
            return _training_call(getattr(_lib(), "moegps_" + name), self._h.value or 0, specs)

        self._gate_up_save = call("expert_ffn_gate_up_save", *xp, row_off, expert, *up, *h, *kept)
        self._ffn_backward = call("expert_ffn_backward", *dyp, *xp, row_off, slot_off, expert, row_pair, *up, *down, *kept, *mid,
                                  *h, *dxp, *d_up)
        self._ffn_backward_act = call("expert_ffn_backward_act", *dyp, row_off, expert, *down, *kept, *mid, *h)
        self._ffn_backward_input = call("expert_ffn_backward_input", *mid, row_off, expert, *up, *dxp)
        self._ffn_backward_weights = call("expert_ffn_backward_weights", *dyp, *xp, *mid, *h, row_off, slot_off, row_pair, *d_up)
        self._combine_backward = call("combine_backward", t("dout", bf16, s.T, s.D), *yp, pair_row, topk_w, *dyp, dtopk_w)
        none = (f32, None, "", True)
        self._dispatch_backward = call("dispatch_backward", *dxp, pair_row, none, none, none, dx)
        self._dispatch_backward_router = call("dispatch_backward", *dxp, pair_row, topk_idx, dlogit, w_router, dx)
        self._route_backward = call("route_backward", t("x", bf16, s.T, s.D), maybe(w_router),
                                    t("bias", f32, s.E, optional=True), maybe(topk_idx), topk_w, dtopk_w, row_off, slot_off,
                                    row_pair, dlogit, t("dw_router", f32, s.E, s.D), t("dbias", f32, s.E),
                                    t("workspace", u8))
        self._route_backward_bytes = route_backward_workspace_bytes(s)
        (up_codes, up_scales), (down_codes, down_scales) = s.w4_shapes(), s.w4_shapes(down=True)
        # of a matrix, its codes and its scales; [1]: down
        self._w4_shapes = ((s.E, s.F, s.D), up_codes, up_scales), ((s.E, s.D, s.F), down_codes, down_scales)
        self._expert_ffn4 = call("expert_ffn4", *xp, row_off, expert, t("gate4", u8, *up_codes), t("up4", u8, *up_codes),
                                 t("down4", u8, *down_codes), t("gate4_scale", u8, *up_scales), t("up4_scale", u8, *up_scales),
                                 t("down4_scale", u8, *down_scales), *yp, t("workspace", u8))
        self._ffn4_bytes = expert_ffn4_workspace_bytes(s)

    def expert_ffn_gate_up_save(self, xp, slot_row_off, slot_expert, w_gate, w_up, h_ws, gate8, up8, gate_scale, up_scale,
                                stream=None):
        rc = self._gate_up_save(stream, xp, slot_row_off, slot_expert, w_gate, w_up, h_ws, gate8, up8, gate_scale, up_scale)
        if rc:
            self._check(rc, "moegps_expert_ffn_gate_up_save")

    def expert_ffn_backward(self, dyp, xp, slot_row_off, slot_off, slot_expert, row_pair, w_gate, w_up, w_down, gate8, up8,
                            gate_scale, up_scale, dgate, dup, h_ws, dxp, dw_gate, dw_up, dw_down, stream=None):
        rc = self._ffn_backward(stream, dyp, xp, slot_row_off, slot_off, slot_expert, row_pair, w_gate, w_up, w_down, gate8, up8,
                                gate_scale, up_scale, dgate, dup, h_ws, dxp, dw_gate, dw_up, dw_down)
        if rc:
            self._check(rc, "moegps_expert_ffn_backward")

    def expert_ffn_backward_act(self, dyp, slot_row_off, slot_expert, w_down, gate8, up8, gate_scale, up_scale, dgate, dup,
                                h_ws, stream=None):
        rc = self._ffn_backward_act(stream, dyp, slot_row_off, slot_expert, w_down, gate8, up8, gate_scale, up_scale, dgate, dup,
                                    h_ws)
        if rc:
            self._check(rc, "moegps_expert_ffn_backward_act")

    def expert_ffn_backward_input(self, dgate, dup, slot_row_off, slot_expert, w_gate, w_up, dxp, stream=None):
        rc = self._ffn_backward_input(stream, dgate, dup, slot_row_off, slot_expert, w_gate, w_up, dxp)
        if rc:
            self._check(rc, "moegps_expert_ffn_backward_input")

    def expert_ffn_backward_weights(self, dyp, xp, dgate, dup, h_ws, slot_row_off, slot_off, row_pair, dw_gate, dw_up, dw_down,
                                    stream=None):
        rc = self._ffn_backward_weights(stream, dyp, xp, dgate, dup, h_ws, slot_row_off, slot_off, row_pair, dw_gate, dw_up,
                                        dw_down)
        if rc:
            self._check(rc, "moegps_expert_ffn_backward_weights")

    def combine_backward(self, dout, yp, pair_row, topk_w, dyp, dtopk_w, stream=None):
        rc = self._combine_backward(stream, dout, yp, pair_row, topk_w, dyp, dtopk_w)
        if rc:
            self._check(rc, "moegps_combine_backward")

    def dispatch_backward(self, dxp, pair_row, topk_idx, dlogit, w_router, dx, stream=None):
        """dlogit None: without the router's part (topk_idx and w_router are not read)."""
        if dlogit is None:
            rc = self._dispatch_backward(stream, dxp, pair_row, None, None, None, dx)
        else:
            rc = self._dispatch_backward_router(stream, dxp, pair_row, topk_idx, dlogit, w_router, dx)
        if rc:
            self._check(rc, "moegps_dispatch_backward")

    def route_backward(self, x, w_router, bias, topk_idx, topk_w, dtopk_w, slot_row_off, slot_off, row_pair, dlogit,
                       dw_router, dbias, workspace, stream=None):
        if workspace is None or workspace.nbytes < self._route_backward_bytes:
            raise MoegpsError(ERR_WORKSPACE_TOO_SMALL, "moegps_route_backward")
        rc = self._route_backward(stream, x, w_router, bias, topk_idx, topk_w, dtopk_w, slot_row_off, slot_off, row_pair, dlogit,
                                  dw_router, dbias, workspace)
        if rc:
            self._check(rc, "moegps_route_backward")

    # -- experts in 4 bits --------------------------------------------------------------------
    def weights_quantize4(self, w, w4, w4_scale, down=False, stream=None):
        """w: bf16 [E, F, D] (down: [E, D, F]) -> codes and scales of Shape.w4_shapes(down)."""
        down = bool(down)
        dense, codes, scales = self._w4_shapes[down]
        self._check(_lib().moegps_weights_quantize4(
            self._h, _ptr(w, torch.bfloat16, dense, "w"), down, _ptr(w4, torch.uint8, codes, "w4"),
            _ptr(w4_scale, torch.uint8, scales, "w4_scale"), _stream(stream)), "moegps_weights_quantize4")

    def weights_dequantize4(self, w4, w4_scale, w, down=False, stream=None):
        """What the codes stand for, exactly, into w: bf16 [E, F, D] (down: [E, D, F])."""
        down = bool(down)
        dense, codes, scales = self._w4_shapes[down]
        self._check(_lib().moegps_weights_dequantize4(
            self._h, _ptr(w4, torch.uint8, codes, "w4"), _ptr(w4_scale, torch.uint8, scales, "w4_scale"), down,
            _ptr(w, torch.bfloat16, dense, "w"), _stream(stream)), "moegps_weights_dequantize4")

    def expert_ffn4(self, xp, slot_row_off, slot_expert, gate4, up4, down4, gate4_scale, up4_scale, down4_scale, yp, workspace,
                    stream=None):
        if workspace is None or workspace.nbytes < self._ffn4_bytes:
            raise MoegpsError(ERR_WORKSPACE_TOO_SMALL, "moegps_expert_ffn4")
        rc = self._expert_ffn4(stream, xp, slot_row_off, slot_expert, gate4, up4, down4, gate4_scale, up4_scale, down4_scale, yp,
                               workspace)
        if rc:
            self._check(rc, "moegps_expert_ffn4")

    def predictor_update(self, hist, state, predicted_hist, stream=None):
        s = self.shape
        self._check(_lib().moegps_predictor_update(
            self._h, _ptr(hist, torch.int32, (s.E,), "hist"), _ptr(state, torch.int64, (s.E,), "state"),
            _ptr(predicted_hist, torch.int32, (s.E,), "predicted_hist"), _stream(stream)),
            "moegps_predictor_update")

    def predictor_update_ema(self, hist, state, shift, predicted_hist, stream=None):
        s = self.shape
        self._check(_lib().moegps_predictor_update_ema(
            self._h, _ptr(hist, torch.int32, (s.E,), "hist"), _ptr(state, torch.int64, (s.E,), "state"), int(shift),
            _ptr(predicted_hist, torch.int32, (s.E,), "predicted_hist"), _stream(stream)),
            "moegps_predictor_update_ema")

    def error_rate(self, predicted_hist, hist, error_rate, stream=None):
        s = self.shape
        self._check(_lib().moegps_error_rate(
            self._h, _ptr(predicted_hist, torch.int32, (s.E,), "predicted_hist"),
            _ptr(hist, torch.int32, (s.E,), "hist"), _ptr(error_rate, torch.float64, (1,), "error_rate"),
            _stream(stream)), "moegps_error_rate")

    def selftest_bounded_wait(self, limit_cycles: int = 2_000_000, stream=None):
        """Launches a kernel whose wait can never be satisfied; status() then reports ERR_TIMEOUT."""
        self._check(_lib().moegps_selftest_bounded_wait(self._h, int(limit_cycles), _stream(stream)),
                    "moegps_selftest_bounded_wait")

    # -- bookkeeping --------------------------------------------------------------------------
    def status(self, stream=None) -> int:
        """Synchronises the stream and returns (and clears) the device status word."""
        h = ctypes.c_int32(0)
        self._check(_lib().moegps_status(self._h, _stream(stream), ctypes.byref(h)), "moegps_status")
        return int(h.value)

    def check_status(self, stream=None):
        st = self.status(stream)
        if st != OK:
            raise MoegpsError(st, "device status")

    def launch_count(self) -> int:
        return int(_lib().moegps_launch_count(self._h))


def rcap(shape: Shape) -> int:
    cs = shape.c_struct()
    return int(_lib().moegps_rcap(ctypes.byref(cs)))


def workspace_bytes(shape: Shape) -> int:
    cs = shape.c_struct()
    return int(_lib().moegps_workspace_bytes(ctypes.byref(cs)))


def route_backward_workspace_bytes(shape: Shape) -> int:
    cs = shape.c_struct()
    return int(_lib().moegps_route_backward_workspace_bytes(ctypes.byref(cs)))


def expert_ffn4_workspace_bytes(shape: Shape) -> int:
    cs = shape.c_struct()
    return int(_lib().moegps_expert_ffn4_workspace_bytes(ctypes.byref(cs)))


def w4_scale_tiles(scale):
    """Scale bytes [E, N, C / 32 rounded up] (one for each 32 inputs of an output, as a checkpoint holds them) in the order of
    Shape.w4_shapes: [E, tiles, chunks, 512]."""
    e, n, b = scale.shape
    tiles, chunks = (n + 127) // 128, (b + 3) // 4
    full = torch.zeros(e, tiles * 128, chunks * 4, dtype=scale.dtype, device=scale.device)
    full[:, :n, :b] = scale
    return full.view(e, tiles, 4, 32, chunks, 4).permute(0, 1, 4, 3, 2, 5).reshape(e, tiles, chunks, 512)


def error_string(code: int) -> str:
    return _lib().moegps_error_string(int(code)).decode()
