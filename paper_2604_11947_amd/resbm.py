"""ctypes binding of ``libresbm`` -- the C ABI declared in ``include/resbm.h``.

Argument marshalling only: torch tensors supply device pointers, row strides
and the current HIP stream; every step of the module runs in the library's
kernels.  A missing library raises ``LibraryNotBuilt``; nothing falls back to
another implementation.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
import warnings

import torch

from . import build as _build

# Native argument marshalling of the short ops; the Python path below does the same checks.
_marshal = None
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    try:
        from . import _marshal
        _marshal.init(torch._C._cuda_getCurrentRawStream)
    except ImportError as e:
        warnings.warn(f"native argument marshalling not loaded ({e}): every op costs about 9 us more of host time; "
                      "run `python -m paper_2604_11947_amd.build`", RuntimeWarning)

ACT_IDENTITY = 0
ACT_SILU = 1
IO_BF16 = 0
IO_F32 = 1

OK = 0
E_NULL = -1
E_SHAPE = -2
E_ALIGN = -3
E_WORKSPACE = -4
E_ACT = -5
E_HIP = -6
E_ALIAS = -7
E_KIND = -8

TYPE_F32 = 0
TYPE_BF16 = 1
STATE_F32 = 0
STATE_E4M3 = 1
STATE_BLOCK = 256  # elements per scale of an 8-bit state
STATE8_BETAS = (0.9, 0.95)  # the largest betas that 8-bit states follow

# Newton-Schulz coefficients of the Muon method the paper cites (Sec. 3.4)
NS_QUINTIC = (3.4445, -4.7750, 2.0315)
NS_CUBIC = (1.5, -0.5, 0.0)

# (name, restype, argtypes) of every exported symbol
_i64, _i32, _p, _sz, _d = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double
SIGNATURES = [
    ("resbm_encode_fwd", _i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _i64, _p, _p, _p, _p, _sz, _p]),
    ("resbm_decode_fwd", _i32, [_i64, _i32, _i32, _i32, _p, _p, _p, _i64, _p, _sz, _p]),
    ("resbm_decode_bwd", _i32, [_i64, _i32, _i32, _p, _p, _p, _i64, _p, _i64, _p, _p, _i32, _p, _sz, _p]),
    ("resbm_encode_bwd", _i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _p, _p, _p, _i64, _p, _i64, _p, _i32,
                                _p, _sz, _p]),
    ("resbm_encode_bwd_noalloc", _i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _p, _p, _p, _i64, _p, _i64, _p,
                                        _i32, _p]),
    ("resbm_newton_schulz", _i32, [_i32, _i32, _p, _p, _i32, _d, _d, _d, _p, _sz, _p]),
    ("resbm_muon_update", _i32, [_i32, _i32, _p, _p, _p, _d, _d, _d, _d, _i32, _i32, _d, _d, _d, _p, _sz, _p]),
    ("resbm_spectrum", _i32, [_i32, _i32, _p, _p, _p, _p, _sz, _p]),
    ("resbm_matrix_workspace_bytes", _sz, [_i32, _i32]),
    ("resbm_workspace_bytes", _sz, [_i64, _i32, _i32]),
    ("resbm2_encode_fwd", _i32, [_i64, _i32, _i32, _i32, _i32, _p, _i64, _p, _i64, _p, _p, _p, _p, _p, _sz, _p]),
    ("resbm2_decode_fwd", _i32, [_i64, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _i64, _p, _p, _sz, _p]),
    ("resbm2_decode_bwd", _i32, [_i64, _i32, _i32, _i32, _i32, _p, _p, _p, _i64, _p, _i64, _p, _p, _p, _p, _p,
                                 _p, _sz, _p]),
    ("resbm2_encode_bwd", _i32, [_i64, _i32, _i32, _i32, _i32, _p, _i64, _p, _p, _p, _p, _p, _i64, _p, _i64,
                                 _p, _p, _p, _sz, _p]),
    ("resbm2_workspace_bytes", _sz, [_i64, _i32, _i32, _i32]),
    ("resbm_ffn_encode_fwd", _i32, [_i64, _i32, _i32, _i32, _i32, _p, _i64, _p, _p, _i64, _p, _p, _i64, _p, _p, _p,
                                    _sz, _p]),
    ("resbm_ffn_encode_workspace_bytes", _sz, [_i64, _i32, _i32]),
    ("resbm_decode_qkv_fwd", _i32, [_i64, _i32, _i32, _i32, _p, _p, _p, _p, ctypes.c_float, _p, _i64, _p, _sz, _p]),
    ("resbm_decode_qkv_workspace_bytes", _sz, [_i32, _i32]),
    ("resbm_skip_norm_fwd", _i32, [_i64, _i32, _i32, _p, _i64, _p, _i64, _p, _p, ctypes.c_float, _p, _i64, _p, _i64, _p,
                                   _p]),
    ("resbm_skip_norm_q8_fwd", _i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _i64, _p, _p, ctypes.c_float, _p, _i64, _p,
                                      _i64, _p, _p, _p]),
    ("resbm_skip_norm_bwd", _i32, [_i64, _i32, _p, _i64, _p, _p, _p, _i64, _p, _i64, _p, _i64, _p, _i32, _p, _sz, _p]),
    ("resbm_norm_workspace_bytes", _sz, [_i64, _i32]),
    ("resbm_adamw_plan_bytes", _sz, [_p, _i64]),
    ("resbm_adamw_plan", _i32, [_p, _i64, _p, _sz]),
    ("resbm_adamw_update", _i32, [_p, _p, _d, _d, _d, _d, _i64, _p, _p, _p]),
    ("resbm_grad_norm_workspace_bytes", _sz, [_p]),
    ("resbm_grad_norm", _i32, [_p, _p, _d, _p, _p, _sz, _p]),
    ("resbm_io_dtype", _i32, []),
    ("resbm_strerror", ctypes.c_char_p, [_i32]),
]


class LibraryNotBuilt(RuntimeError):
    pass


class ResbmError(RuntimeError):
    def __init__(self, op: str, status: int, message: str):
        super().__init__(f"{op}: status {status}: {message}")
        self.status = status


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _room(ws):
    """A workspace's address and bytes."""
    if ws is None:
        return None, 0
    if not ws.is_contiguous():  # an expanded one has fewer bytes than elements
        raise ValueError(f"ws: expected a contiguous tensor, got strides {tuple(ws.stride())}")
    return _ptr(ws), ws.numel()


def _ld(t: torch.Tensor, rows: int, cols: int, name: str) -> int:
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name}: expected shape ({rows}, {cols}), got {tuple(t.shape)}")
    if rows > 0 and cols > 1 and t.stride(1) != 1:  # one row's too
        raise ValueError(f"{name}: rows must be contiguous")
    return t.stride(0) if rows > 1 else max(t.stride(0), cols)


def _packed(t: torch.Tensor, rows: int, cols: int, name: str) -> None:
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous ({rows}, {cols}) tensor, got {tuple(t.shape)}")


def _dtype(t, dtype, name):
    if t is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")


def _vector(t: torch.Tensor, size: int, name: str) -> None:
    _dtype(t, torch.float32, name)
    if t.dim() != 1 or t.numel() != size or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous vector of {size} elements, got {tuple(t.shape)}")


def _one_gpu(op: str, *tensors) -> None:
    """All of an op's tensors on the GPU that the first is on."""
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1 or next(iter(devices)).type != "cuda":
        raise ValueError(f"{op}: expected tensors of one GPU, got {sorted(map(str, devices))}")


def _grad_dtype(t: torch.Tensor, i: int) -> None:
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"g[{i}]: expected torch.float32 or torch.bfloat16, got {t.dtype}")


def _stream(stream, ref):
    if stream is None:
        stream = torch.cuda.current_stream(ref.device)
    return ctypes.c_void_p(getattr(stream, "cuda_stream", stream))


class AdamWTensor(ctypes.Structure):
    """resbm_adamw_tensor."""
    _fields_ = [("numel", ctypes.c_int64)] + [(k, ctypes.c_void_p) for k in ("p", "g", "m", "v", "m_scale", "v_scale",
                                                                             "copy")] + [
        ("g_type", ctypes.c_int32), ("state", ctypes.c_int32), ("weight_decay", ctypes.c_float),
        ("reserved", ctypes.c_int32)]


_ENTRY = struct.Struct("=q7Q2ifi")  # its fields in order


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # a device's current stream, as a handle


class AdamWPlan:
    """A plan's host and device copies, and the tensors whose addresses it holds.

    Made by ``Library.adamw_plan`` or ``Library.grad_plan`` with the tensors' current
    addresses; a tensor that moves needs a new plan.  A plan may be dropped while a step
    still runs, on whichever stream (tensors that nothing else holds are the caller's to
    keep, as for any op on another stream).  A graph that captured a step reads the plan's
    table at every replay: the plan has to live as long as the graph."""

    def __init__(self, host, device_table, tensors, device, q8=False):
        self.host, self.table, self.tensors, self.device = host, device_table, tensors, device
        self.q8 = q8  # whether there are states in 8 bits
        self.host_ptr, self.table_ptr = ctypes.addressof(host), device_table.data_ptr()
        self.index = device.index
        self.streams = {_raw_stream(self.index)}  # that the table's memory waits for before it is used again

    def used_on(self, stream):
        """Ties the table's memory to the stream of a step: freed with the plan, it is not handed out before that
        step has read it."""
        raw = _raw_stream(self.index) if stream is None else int(getattr(stream, "cuda_stream", stream))
        if raw not in self.streams:
            self.table.record_stream(torch.cuda.current_stream(self.device) if stream is None
                                     else _torch_stream(stream, self.device))
            self.streams.add(raw)


def _torch_stream(stream, device):
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)), device=device)


def _allocating_on(stream, device):
    """The context in which a workspace belongs to the stream that uses it: freed with the call's return, it is
    not handed out on another stream while the kernels run."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(_torch_stream(stream, device))


class Library:
    """One loaded variant of the library ("bf16" or "f32")."""

    def __init__(self, variant: str = "bf16"):
        path = _build.lib_path(variant)
        if not os.path.exists(path):
            raise LibraryNotBuilt(f"{path} is missing; run `python -m paper_2604_11947_amd.build`")
        self.path = path
        self.cdll = ctypes.CDLL(path)
        for name, res, args in SIGNATURES:
            fn = getattr(self.cdll, name)
            fn.restype = res
            fn.argtypes = args
        # addresses for the marshalling module
        self._at = {name: ctypes.cast(getattr(self.cdll, name), ctypes.c_void_p).value for name, _, _ in SIGNATURES}
        self.io_code = int(self.cdll.resbm_io_dtype())
        self.io_dtype = torch.bfloat16 if self.io_code == IO_BF16 else torch.float32

    # ------------------------------------------------------------ helpers
    def workspace_bytes(self, T: int, n: int, r: int) -> int:
        return int(self.cdll.resbm_workspace_bytes(T, n, r))

    def strerror(self, status: int) -> str:
        return self.cdll.resbm_strerror(status).decode()

    def workspace(self, T: int, n: int, r: int, device) -> torch.Tensor:
        nbytes = self.workspace_bytes(T, n, r)
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-buf.data_ptr()) % 256
        return buf[off:off + nbytes]

    def matrix_workspace_bytes(self, p: int, q: int) -> int:
        return int(self.cdll.resbm_matrix_workspace_bytes(p, q))

    def matrix_workspace(self, p: int, q: int, device) -> torch.Tensor:
        nbytes = self.matrix_workspace_bytes(p, q)
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-buf.data_ptr()) % 256
        return buf[off:off + nbytes]

    def _check(self, op: str, status: int) -> None:
        if status != OK:
            raise ResbmError(op, status, self.strerror(status))

    def _run(self, op: str, ref, stream, *args) -> None:
        """Calls the library's function on `stream`, or on the current stream of the device that `ref` is on.  A launch
        on a device's default stream goes to the current device, so that device is the current one meanwhile."""
        s = _stream(stream, ref)
        if ref.device.type == "cuda" and ref.device.index != torch.cuda.current_device():
            with torch.cuda.device(ref.device):
                st = getattr(self.cdll, op)(*args, s)
        else:
            st = getattr(self.cdll, op)(*args, s)
        self._check(op, st)

    # ------------------------------------------------------------ ops
    def encode_fwd(self, x_attn, z, W_e, b, a_save=None, act=ACT_SILU, ws=None, stream=None):
        if _marshal is not None and stream is None:
            st = _marshal.encode_fwd(self._at["resbm_encode_fwd"], self.io_code, x_attn, z, W_e, b, a_save, act, ws)
            if st is not None:
                return self._check("resbm_encode_fwd", st)
        T = z.shape[0]
        n, r = W_e.shape
        io = self.io_dtype
        for t, nm in ((x_attn, "x_attn"), (z, "z"), (b, "b")):
            _dtype(t, io, nm)
        _dtype(W_e, torch.float32, "W_e")
        _dtype(a_save, torch.float32, "a_save")
        ld_x, ld_z = _ld(x_attn, T, n, "x_attn"), _ld(z, T, n, "z")
        _packed(b, T, r, "b")
        _packed(W_e, n, r, "W_e")
        if a_save is not None:
            _packed(a_save, T, r, "a_save")
        if ws is None:
            with _allocating_on(stream, z.device):
                ws = self.workspace(T, n, r, z.device)
        self._run("resbm_encode_fwd", z, stream, T, n, r, act, _ptr(x_attn), ld_x, _ptr(z), ld_z, _ptr(W_e), _ptr(b),
                  _ptr(a_save), *_room(ws))

    def decode_fwd(self, b, W_d, z_tilde, add_identity=False, ws=None, stream=None):
        if _marshal is not None and stream is None:
            st = _marshal.decode_fwd(self._at["resbm_decode_fwd"], self.io_code, b, W_d, z_tilde, add_identity, ws)
            if st is not None:
                return self._check("resbm_decode_fwd", st)
        T = b.shape[0]
        r, n = W_d.shape
        _dtype(b, self.io_dtype, "b")
        _dtype(z_tilde, self.io_dtype, "z_tilde")
        _dtype(W_d, torch.float32, "W_d")
        _packed(b, T, r, "b")
        _packed(W_d, r, n, "W_d")
        ld = _ld(z_tilde, T, n, "z_tilde")
        self._run("resbm_decode_fwd", b, stream, T, n, r, int(bool(add_identity)), _ptr(b), _ptr(W_d), _ptr(z_tilde),
                  ld, *_room(ws))

    def decode_bwd(self, b, W_d, g_zt, g_id, g_b, dW_d, accumulate=False, ws=None, stream=None):
        if _marshal is not None and stream is None:
            st = _marshal.decode_bwd(self._at["resbm_decode_bwd"], self.io_code, b, W_d, g_zt, g_id, g_b, dW_d,
                                     accumulate, ws)
            if st is not None:
                return self._check("resbm_decode_bwd", st)
        T = b.shape[0]
        r, n = W_d.shape
        io = self.io_dtype
        for t, nm in ((b, "b"), (g_zt, "g_zt"), (g_id, "g_id"), (g_b, "g_b")):
            _dtype(t, io, nm)
        _dtype(W_d, torch.float32, "W_d")
        _dtype(dW_d, torch.float32, "dW_d")
        _packed(b, T, r, "b")
        _packed(g_b, T, r, "g_b")
        _packed(W_d, r, n, "W_d")
        _packed(dW_d, r, n, "dW_d")
        ld_g = _ld(g_zt, T, n, "g_zt")
        ld_i = _ld(g_id, T, n, "g_id") if g_id is not None else 0
        if ws is None:
            with _allocating_on(stream, g_zt.device):
                ws = self.workspace(T, n, r, g_zt.device)
        self._run("resbm_decode_bwd", g_zt, stream, T, n, r, _ptr(b), _ptr(W_d), _ptr(g_zt), ld_g, _ptr(g_id), ld_i,
                  _ptr(g_b), _ptr(dW_d), int(bool(accumulate)), *_room(ws))

    def encode_bwd(self, z, W_e, a_save, g_b, g_z, dW_e, g_x=None, act=ACT_SILU, accumulate=False, ws=None,
                   stream=None):
        if _marshal is not None and stream is None:
            st = _marshal.encode_bwd(self._at["resbm_encode_bwd"], self.io_code, z, W_e, a_save, g_b, g_z, dW_e, g_x,
                                     act, accumulate, ws)
            if st is not None:
                return self._check("resbm_encode_bwd", st)
        T = z.shape[0]
        n, r = W_e.shape
        io = self.io_dtype
        for t, nm in ((z, "z"), (g_b, "g_b"), (g_z, "g_z"), (g_x, "g_x")):
            _dtype(t, io, nm)
        _dtype(W_e, torch.float32, "W_e")
        _dtype(a_save, torch.float32, "a_save")
        _dtype(dW_e, torch.float32, "dW_e")
        ld_z = _ld(z, T, n, "z")
        ld_gz = _ld(g_z, T, n, "g_z")
        ld_gx = _ld(g_x, T, n, "g_x") if g_x is not None else 0
        _packed(W_e, n, r, "W_e")
        _packed(g_b, T, r, "g_b")
        _packed(dW_e, n, r, "dW_e")
        if a_save is not None:
            _packed(a_save, T, r, "a_save")
        if ws is None:
            with _allocating_on(stream, z.device):
                ws = self.workspace(T, n, r, z.device)
        self._run("resbm_encode_bwd", z, stream, T, n, r, act, _ptr(z), ld_z, _ptr(W_e), _ptr(a_save), _ptr(g_b),
                  _ptr(g_z), ld_gz, _ptr(g_x), ld_gx, _ptr(dW_e), int(bool(accumulate)), *_room(ws))


    def encode_bwd_noalloc(self, z, W_e, a_save, g_b, g_z, dW_e, g_x=None, act=ACT_SILU, accumulate=False,
                           stream=None):
        """resbm_encode_bwd_noalloc: encode_bwd on the library's fixed device-resident
        scratch (no workspace argument, nothing allocated)."""
        T = z.shape[0]
        n, r = W_e.shape
        io = self.io_dtype
        for t, nm in ((z, "z"), (g_b, "g_b"), (g_z, "g_z"), (g_x, "g_x")):
            _dtype(t, io, nm)
        _dtype(W_e, torch.float32, "W_e")
        _dtype(a_save, torch.float32, "a_save")
        _dtype(dW_e, torch.float32, "dW_e")
        ld_z = _ld(z, T, n, "z")
        ld_gz = _ld(g_z, T, n, "g_z")
        ld_gx = _ld(g_x, T, n, "g_x") if g_x is not None else 0
        _packed(W_e, n, r, "W_e")
        _packed(g_b, T, r, "g_b")
        _packed(dW_e, n, r, "dW_e")
        if a_save is not None:
            _packed(a_save, T, r, "a_save")
        self._run("resbm_encode_bwd_noalloc", z, stream, T, n, r, act, _ptr(z), ld_z, _ptr(W_e), _ptr(a_save),
                  _ptr(g_b), _ptr(g_z), ld_gz, _ptr(g_x), ld_gx, _ptr(dW_e), int(bool(accumulate)))

    # ------------------------------------------------------------ two-linears-per-side ops
    # Weights W1 (n x m), W2 (m x r), W3 (r x m), W4 (m x n) and every activation
    # are bf16; the weight gradients float32.
    def two_workspace_bytes(self, T: int, n: int, m: int, r: int) -> int:
        return int(self.cdll.resbm2_workspace_bytes(T, n, m, r))

    def two_workspace(self, T: int, n: int, m: int, r: int, device) -> torch.Tensor:
        nbytes = self.two_workspace_bytes(T, n, m, r)
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-buf.data_ptr()) % 256
        return buf[off:off + nbytes]

    @staticmethod
    def _two_weights(W1, W2, W3=None, W4=None):
        n, m = W1.shape
        r = W2.shape[1]
        for t, nm, shape in ((W1, "W1", (n, m)), (W2, "W2", (m, r)), (W3, "W3", (r, m)), (W4, "W4", (m, n))):
            if t is not None:
                _dtype(t, torch.bfloat16, nm)
                _packed(t, *shape, nm)
        return n, m, r

    def encode2_fwd(self, x_attn, z, W1, W2, b, u, act=ACT_SILU, ws=None, stream=None):
        T = z.shape[0]
        n, m, r = self._two_weights(W1, W2)
        for t, nm in ((x_attn, "x_attn"), (z, "z"), (b, "b"), (u, "u")):
            _dtype(t, torch.bfloat16, nm)
        ld_x, ld_z = _ld(x_attn, T, n, "x_attn"), _ld(z, T, n, "z")
        _packed(b, T, r, "b")
        _packed(u, T, m, "u")
        if ws is None and act != ACT_IDENTITY:
            with _allocating_on(stream, z.device):
                ws = self.two_workspace(T, n, m, r, z.device)
        self._run("resbm2_encode_fwd", z, stream, T, n, m, r, act, _ptr(x_attn), ld_x, _ptr(z), ld_z, _ptr(W1),
                  _ptr(W2), _ptr(b), _ptr(u), *_room(ws))

    def decode2_fwd(self, b, W3, W4, z_tilde, v, act=ACT_SILU, ws=None, stream=None):
        T = b.shape[0]
        m, n = W4.shape
        r = W3.shape[0]
        for t, nm, shape in ((W3, "W3", (r, m)), (W4, "W4", (m, n))):
            _dtype(t, torch.bfloat16, nm)
            _packed(t, *shape, nm)
        for t, nm in ((b, "b"), (z_tilde, "z_tilde"), (v, "v")):
            _dtype(t, torch.bfloat16, nm)
        _packed(b, T, r, "b")
        _packed(v, T, m, "v")
        ld_zt = _ld(z_tilde, T, n, "z_tilde")
        if ws is None:
            with _allocating_on(stream, b.device):
                ws = self.two_workspace(T, n, m, r, b.device)
        self._run("resbm2_decode_fwd", b, stream, T, n, m, r, act, _ptr(b), _ptr(W3), _ptr(W4), _ptr(z_tilde), ld_zt,
                  _ptr(v), *_room(ws))

    def decode2_bwd(self, b, v, g_zt, g_id, W3, W4, g_b, dW3, dW4, act=ACT_SILU, ws=None, stream=None):
        T = b.shape[0]
        m, n = W4.shape
        r = W3.shape[0]
        for t, nm, shape in ((W3, "W3", (r, m)), (W4, "W4", (m, n))):
            _dtype(t, torch.bfloat16, nm)
            _packed(t, *shape, nm)
        for t, nm in ((b, "b"), (v, "v"), (g_zt, "g_zt"), (g_id, "g_id"), (g_b, "g_b")):
            _dtype(t, torch.bfloat16, nm)
        _dtype(dW3, torch.float32, "dW3")
        _dtype(dW4, torch.float32, "dW4")
        _packed(b, T, r, "b")
        _packed(v, T, m, "v")
        _packed(g_b, T, r, "g_b")
        _packed(dW3, r, m, "dW3")
        _packed(dW4, m, n, "dW4")
        ld_gzt = _ld(g_zt, T, n, "g_zt")
        ld_gid = _ld(g_id, T, n, "g_id") if g_id is not None else 0
        if ws is None:
            with _allocating_on(stream, b.device):
                ws = self.two_workspace(T, n, m, r, b.device)
        self._run("resbm2_decode_bwd", b, stream, T, n, m, r, act, _ptr(b), _ptr(v), _ptr(g_zt), ld_gzt, _ptr(g_id),
                  ld_gid, _ptr(W3), _ptr(W4), _ptr(g_b), _ptr(dW3), _ptr(dW4), *_room(ws))

    def encode2_bwd(self, z, u, g_b, W1, W2, g_z, dW1, dW2, g_x=None, act=ACT_SILU, ws=None, stream=None):
        T = z.shape[0]
        n, m, r = self._two_weights(W1, W2)
        for t, nm in ((z, "z"), (u, "u"), (g_b, "g_b"), (g_z, "g_z"), (g_x, "g_x")):
            _dtype(t, torch.bfloat16, nm)
        _dtype(dW1, torch.float32, "dW1")
        _dtype(dW2, torch.float32, "dW2")
        _packed(u, T, m, "u")
        _packed(g_b, T, r, "g_b")
        _packed(dW1, n, m, "dW1")
        _packed(dW2, m, r, "dW2")
        ld_z, ld_gz = _ld(z, T, n, "z"), _ld(g_z, T, n, "g_z")
        ld_gx = _ld(g_x, T, n, "g_x") if g_x is not None else 0
        if ws is None:
            with _allocating_on(stream, z.device):
                ws = self.two_workspace(T, n, m, r, z.device)
        self._run("resbm2_encode_bwd", z, stream, T, n, m, r, act, _ptr(z), ld_z, _ptr(u), _ptr(g_b), _ptr(W1),
                  _ptr(W2), _ptr(g_z), ld_gz, _ptr(g_x), ld_gx, _ptr(dW1), _ptr(dW2), *_room(ws))

    # ------------------------------------------------------------ encoder fused into the FFN output projection
    def ffn_encode_fwd(self, h, W_down, x_attn, W_e, z, b, a_save=None, act=ACT_SILU, ws=None, stream=None):
        T, d_ff = h.shape
        n, r = W_e.shape
        for t, nm in ((h, "h"), (W_down, "W_down"), (x_attn, "x_attn"), (z, "z"), (b, "b")):
            _dtype(t, torch.bfloat16, nm)
        _dtype(W_e, torch.float32, "W_e")
        _dtype(a_save, torch.float32, "a_save")
        _packed(W_down, d_ff, n, "W_down")
        _packed(W_e, n, r, "W_e")
        _packed(b, T, r, "b")
        if a_save is not None:
            _packed(a_save, T, r, "a_save")
        ld_h, ld_x, ld_z = _ld(h, T, d_ff, "h"), _ld(x_attn, T, n, "x_attn"), _ld(z, T, n, "z")
        if ws is None:
            nbytes = int(self.cdll.resbm_ffn_encode_workspace_bytes(T, n, r))
            with _allocating_on(stream, h.device):
                ws = self._buffer(nbytes, h.device)
        self._run("resbm_ffn_encode_fwd", h, stream, T, d_ff, n, r, act, _ptr(h), ld_h, _ptr(W_down), _ptr(x_attn),
                  ld_x, _ptr(W_e), _ptr(z), ld_z, _ptr(b), _ptr(a_save), *_room(ws))

    def decode_qkv_fwd(self, b, W_d, gamma, W_qkv, out, eps=1e-5, ws=None, stream=None):
        T, r = b.shape
        n, N = W_qkv.shape
        for t, nm in ((b, "b"), (W_qkv, "W_qkv"), (out, "out")):
            _dtype(t, torch.bfloat16, nm)
        _dtype(W_d, torch.float32, "W_d")
        _dtype(gamma, torch.float32, "gamma")
        _packed(b, T, r, "b")
        _packed(W_d, r, n, "W_d")
        _packed(W_qkv, n, N, "W_qkv")
        if gamma.dim() != 1 or gamma.numel() != n or not gamma.is_contiguous():
            raise ValueError("gamma: expected a contiguous vector of n elements")
        ld_out = _ld(out, T, N, "out")
        if ws is None:
            nbytes = int(self.cdll.resbm_decode_qkv_workspace_bytes(n, r))
            with _allocating_on(stream, b.device):
                ws = self._buffer(nbytes, b.device)
        self._run("resbm_decode_qkv_fwd", b, stream, T, n, r, N, _ptr(b), _ptr(W_d), _ptr(gamma), _ptr(W_qkv), eps,
                  _ptr(out), ld_out, *_room(ws))

    # ------------------------------------------------------------ optimizer-side ops
    def newton_schulz(self, G, O, steps=5, coeffs=NS_QUINTIC, ws=None, stream=None):
        p, q = G.shape
        _dtype(G, torch.float32, "G")
        _dtype(O, torch.float32, "O")
        _packed(G, p, q, "G")
        _packed(O, p, q, "O")
        if ws is None:
            with _allocating_on(stream, G.device):
                ws = self.matrix_workspace(p, q, G.device)
        a, b, c = coeffs
        self._run("resbm_newton_schulz", G, stream, p, q, _ptr(G), _ptr(O), steps, a, b, c, *_room(ws))

    def muon_update(self, W, G, M, lr, momentum=0.95, weight_decay=0.0, scale=None, nesterov=False, steps=5,
                    coeffs=NS_QUINTIC, ws=None, stream=None):
        if _marshal is not None and stream is None:
            st = _marshal.muon_update(self._at["resbm_muon_update"], W, G, M, lr, momentum, weight_decay,
                                      -1.0 if scale is None else scale, nesterov, steps, coeffs, ws)
            if st is not None:
                return self._check("resbm_muon_update", st)
        p, q = W.shape
        for t, nm in ((W, "W"), (G, "G"), (M, "M")):
            _dtype(t, torch.float32, nm)
            if t is not None:
                _packed(t, p, q, nm)
        if scale is None:
            scale = -1.0  # the library's default (negative selects it)
        if ws is None:
            with _allocating_on(stream, W.device):
                ws = self.matrix_workspace(p, q, W.device)
        a, b, c = coeffs
        self._run("resbm_muon_update", W, stream, p, q, _ptr(W), _ptr(G), _ptr(M), lr, momentum, weight_decay, scale,
                  int(bool(nesterov)), steps, a, b, c, *_room(ws))

    def spectrum(self, W, sigma, r_eff, ws=None, stream=None):
        p, q = W.shape
        _dtype(W, torch.float32, "W")
        _packed(W, p, q, "W")
        _dtype(sigma, torch.float64, "sigma")
        _dtype(r_eff, torch.float64, "r_eff")
        if sigma.numel() < min(p, q) or r_eff.numel() < 1 or not sigma.is_contiguous():
            raise ValueError("sigma needs min(p, q) contiguous float64 elements, r_eff one")
        if ws is None:
            with _allocating_on(stream, W.device):
                ws = self.matrix_workspace(p, q, W.device)
        self._run("resbm_spectrum", W, stream, p, q, _ptr(W), _ptr(sigma), _ptr(r_eff), *_room(ws))

    # ------------------------------------------------------------ residual addition and RMS norm
    def norm_workspace(self, T: int, n: int, device) -> torch.Tensor:
        return self._buffer(int(self.cdll.resbm_norm_workspace_bytes(T, n)), device)

    @staticmethod
    def _buffer(nbytes: int, device) -> torch.Tensor:
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        return buf[(-buf.data_ptr()) % 256:][:nbytes]

    def _norm_inputs(self, x, gamma, res, b, h, rstd):
        """Checks what the two forward norms share; (T, n, r, ld_x, ld_res, ld_h)."""
        T, n = x.shape
        for t, nm in ((x, "x"), (res, "res"), (b, "b"), (h, "h")):
            _dtype(t, self.io_dtype, nm)
        _vector(gamma, n, "gamma")
        if rstd is not None:
            _vector(rstd, T, "rstd")
        r = 0
        if b is not None:
            r = b.shape[1] if b.dim() == 2 else -1
            _packed(b, T, r, "b")
        return (T, n, r, _ld(x, T, n, "x"), 0 if res is None else _ld(res, T, n, "res"),
                0 if h is None else _ld(h, T, n, "h"))

    def skip_norm_fwd(self, x, gamma, y, res=None, b=None, h=None, rstd=None, eps=1e-5, stream=None):
        """h = x + res + b I (rounded once; written when ``h`` is given), y = RMSNorm(h) gamma."""
        if _marshal is not None and stream is None:
            st = _marshal.skip_norm_fwd(self._at["resbm_skip_norm_fwd"], self.io_code, x, gamma, res, b, h, rstd, eps, y)
            if st is not None:
                return self._check("resbm_skip_norm_fwd", st)
        T, n, r, ld_x, ld_res, ld_h = self._norm_inputs(x, gamma, res, b, h, rstd)
        _dtype(y, self.io_dtype, "y")
        ld_y = _ld(y, T, n, "y")
        _one_gpu("skip_norm_fwd", x, gamma, y, res, b, h, rstd)
        self._run("resbm_skip_norm_fwd", x, stream, T, n, r, _ptr(x), ld_x, _ptr(res), ld_res, _ptr(b), _ptr(gamma),
                  eps, _ptr(h), ld_h, _ptr(y), ld_y, _ptr(rstd))

    def skip_norm_q8_fwd(self, x, gamma, y, scale, res=None, b=None, h=None, rstd=None, eps=1e-5, stream=None):
        """skip_norm_fwd with y in e4m3 and float32 scales; ``scale`` (T, n / group) sets the group of columns."""
        if _marshal is not None and stream is None:
            st = _marshal.skip_norm_q8_fwd(self._at["resbm_skip_norm_q8_fwd"], self.io_code, x, gamma, res, b, h, rstd,
                                           eps, y, scale)
            if st is not None:
                return self._check("resbm_skip_norm_q8_fwd", st)
        T, n, r, ld_x, ld_res, ld_h = self._norm_inputs(x, gamma, res, b, h, rstd)
        _dtype(y, torch.float8_e4m3fn, "y")
        _dtype(scale, torch.float32, "scale")
        ld_y = _ld(y, T, n, "y")
        groups = scale.shape[1] if scale.dim() == 2 else 0
        if groups < 1 or n % groups:
            raise ValueError(f"scale: expected shape ({T}, n / group), got {tuple(scale.shape)}")
        _packed(scale, T, groups, "scale")
        _one_gpu("skip_norm_q8_fwd", x, gamma, y, scale, res, b, h, rstd)
        self._run("resbm_skip_norm_q8_fwd", x, stream, T, n, r, n // groups, _ptr(x), ld_x, _ptr(res), ld_res, _ptr(b),
                  _ptr(gamma), eps, _ptr(h), ld_h, _ptr(y), ld_y, _ptr(scale), _ptr(rstd))

    def skip_norm_bwd(self, h, gamma, rstd, g_y, g_x, dgamma, g_h=None, accumulate=False, ws=None, stream=None):
        """The norm's gradient plus g_h in g_x (which may be g_y or g_h), the gain's in dgamma."""
        if _marshal is not None and stream is None:
            st = _marshal.skip_norm_bwd(self._at["resbm_skip_norm_bwd"], self.io_code, h, gamma, rstd, g_y, g_x, dgamma,
                                        g_h, accumulate, ws)
            if st is not None:
                return self._check("resbm_skip_norm_bwd", st)
        T, n = h.shape
        for t, nm in ((h, "h"), (g_y, "g_y"), (g_h, "g_h"), (g_x, "g_x")):
            _dtype(t, self.io_dtype, nm)
        _vector(gamma, n, "gamma")
        _vector(rstd, T, "rstd")
        _vector(dgamma, n, "dgamma")
        ld_h, ld_gy, ld_gx = _ld(h, T, n, "h"), _ld(g_y, T, n, "g_y"), _ld(g_x, T, n, "g_x")
        ld_gh = _ld(g_h, T, n, "g_h") if g_h is not None else 0
        if ws is None:
            with _allocating_on(stream, h.device):
                ws = self.norm_workspace(T, n, h.device)
        _one_gpu("skip_norm_bwd", h, gamma, rstd, g_y, g_x, dgamma, g_h, ws)
        self._run("resbm_skip_norm_bwd", h, stream, T, n, _ptr(h), ld_h, _ptr(gamma), _ptr(rstd), _ptr(g_y), ld_gy,
                  _ptr(g_h), ld_gh, _ptr(g_x), ld_gx, _ptr(dgamma), int(bool(accumulate)), *_room(ws))

    # ------------------------------------------------------------ AdamW over many tensors
    def adamw_plan(self, p, g, m, v, m_scale=None, v_scale=None, copy=None, weight_decay=0.0) -> AdamWPlan:
        """The plan of the lists' tensors: float32 ``p``, gradients float32 or bf16, states float32 or, with
        ``m_scale`` and ``v_scale`` (an entry may be None), float8_e4m3fn; ``copy``: bf16 tensors or None.
        It copies its table to the device, so it is made outside a graph capture; its updates may be captured.
        It holds addresses: gradients stay where they are (``zero_grad(set_to_none=False)``), or a new plan is made
        for the new ones; until it goes, it keeps its tensors."""
        k = len(p)
        none = [None] * k
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * k
        lists = [list(t) if t is not None else none for t in (p, g, m, v, m_scale, v_scale, copy)]
        if any(len(t) != k for t in lists + [decay]):
            raise ValueError("adamw_plan: lists of different lengths")
        entries = (AdamWTensor * max(k, 1))()
        f32, bf16, f8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
        at, size, pack = 0, ctypes.sizeof(AdamWTensor), _ENTRY.pack_into
        for i, (wd, row) in enumerate(zip(decay, zip(*lists))):
            P, G, M, V, ms, vs, cp = row
            n, q8, g16 = P.numel(), ms is not None, G.dtype is bf16
            state = f8 if q8 else f32
            good = (P.dtype is f32 and (g16 or G.dtype is f32) and M.dtype is state and V.dtype is state
                    and G.numel() == n and M.numel() == n and V.numel() == n and P.is_contiguous() and G.is_contiguous()
                    and M.is_contiguous() and V.is_contiguous()
                    and (cp is None or (cp.dtype is bf16 and cp.numel() == n and cp.is_contiguous())))
            if good and q8:
                nb = (-(-n // STATE_BLOCK),)
                good = (vs is not None and ms.dtype is f32 and vs.dtype is f32 and ms.shape == nb and vs.shape == nb
                        and ms.is_contiguous() and vs.is_contiguous())
            if not good or (vs is not None) != q8:
                self._explain_entry(i, *row)
            pack(entries, at, n, P.data_ptr(), G.data_ptr(), M.data_ptr(), V.data_ptr(), ms.data_ptr() if q8 else 0,
                 vs.data_ptr() if q8 else 0, 0 if cp is None else cp.data_ptr(), TYPE_BF16 if g16 else TYPE_F32,
                 STATE_E4M3 if q8 else STATE_F32, wd, 0)
            at += size
        return self._plan(entries, k, lists, any(s is not None and s.numel() > 0 for s in lists[4]))

    @staticmethod
    def _explain_entry(i, P, G, M, V, ms, vs, cp):
        """Raises the error of an entry that adamw_plan does not take."""
        _dtype(P, torch.float32, f"p[{i}]")
        _grad_dtype(G, i)
        for t, nm in ((M, "m"), (V, "v")):
            _dtype(t, torch.float32 if ms is None else torch.float8_e4m3fn, f"{nm}[{i}]")
        _dtype(cp, torch.bfloat16, f"copy[{i}]")
        if (vs is None) != (ms is None):
            raise ValueError(f"m_scale[{i}], v_scale[{i}]: both or neither")
        for t, nm in ((P, "p"), (G, "g"), (M, "m"), (V, "v"), (cp, "copy")):
            if t is not None and (t.numel() != P.numel() or not t.is_contiguous()):
                raise ValueError(f"{nm}[{i}]: expected a contiguous tensor of {P.numel()} elements")
        for t, nm in ((ms, "m_scale"), (vs, "v_scale")):
            if t is not None:
                _vector(t, -(-P.numel() // STATE_BLOCK), f"{nm}[{i}]")
        raise ValueError(f"entry {i}: not a set of tensors that a plan takes")

    def grad_plan(self, g) -> AdamWPlan:
        """A plan of gradients alone, for grad_norm."""
        entries = (AdamWTensor * max(len(g), 1))()
        for i, (e, G) in enumerate(zip(entries, g)):
            _grad_dtype(G, i)
            if not G.is_contiguous():
                raise ValueError(f"g[{i}]: expected a contiguous tensor")
            e.numel, e.g, e.g_type = G.numel(), G.data_ptr(), TYPE_BF16 if G.dtype == torch.bfloat16 else TYPE_F32
        return self._plan(entries, len(g), [list(g)])

    def _plan(self, entries, count, lists, q8=False) -> AdamWPlan:
        tensors = [t for row in lists for t in row if t is not None]
        if tensors and (len(set(map(torch.Tensor.get_device, tensors))) > 1 or not tensors[0].is_cuda):
            _one_gpu("plan", *tensors)
        device = tensors[0].device if tensors else torch.device("cuda", torch.cuda.current_device())
        nbytes = int(self.cdll.resbm_adamw_plan_bytes(entries, count))
        host = (ctypes.c_int64 * (max(nbytes, 256) // 8))()
        self._check("resbm_adamw_plan", self.cdll.resbm_adamw_plan(entries, count, host, nbytes))
        table = self._buffer(nbytes, device)
        table.copy_(torch.frombuffer(host, dtype=torch.uint8)[:nbytes])
        return AdamWPlan(host, table, tensors, device, q8)

    def adamw_update(self, plan: AdamWPlan, lr=0.0, step=1, betas=(0.9, 0.95), eps=1e-8, grad_scale=None, lr_step=None,
                     stream=None):
        """One AdamW step on the plan's tensors.  ``grad_scale``: a float32 tensor of one element on the device, the
        gradients' factor (NaN leaves the step out); ``lr_step``: a float64 tensor {lr, step} there, read when the
        kernel runs, in place of ``lr`` and ``step``.  8-bit states take betas up to (0.9, 0.95): beyond, their
        rounding would hold them where they are."""
        if plan.q8 and (betas[0] > STATE8_BETAS[0] or betas[1] > STATE8_BETAS[1]):
            raise ValueError(f"adamw_update: 8-bit states take betas up to {STATE8_BETAS}, got {tuple(betas)}")
        plan.used_on(stream)
        if _marshal is not None and stream is None:
            st = _marshal.adamw_update(self._at["resbm_adamw_update"], plan.host_ptr, plan.table, lr, step, betas, eps,
                                       grad_scale, lr_step)
            if st is not None:
                return self._check("resbm_adamw_update", st)
        for t, dt, k, nm in ((grad_scale, torch.float32, 1, "grad_scale"), (lr_step, torch.float64, 2, "lr_step")):
            if t is not None:
                _dtype(t, dt, nm)
                if t.numel() != k or not t.is_contiguous() or t.device != plan.device:
                    raise ValueError(f"{nm}: expected {k} contiguous elements on {plan.device}")
        self._run("resbm_adamw_update", plan, stream, plan.host_ptr, plan.table_ptr, lr, betas[0], betas[1], eps, step,
                  _ptr(lr_step), _ptr(grad_scale))

    def grad_norm_workspace(self, plan: AdamWPlan) -> torch.Tensor:
        return self._buffer(int(self.cdll.resbm_grad_norm_workspace_bytes(plan.host_ptr)), plan.device)

    def grad_norm(self, plan: AdamWPlan, max_norm, out, ws=None, stream=None):
        """out[0] = the 2-norm of the plan's gradients, out[1] = min(1, max_norm / norm): adamw_update's grad_scale.
        Over several plans or ranks: the root of the sum of their squared out[0], and the factor from that."""
        plan.used_on(stream)
        if _marshal is not None and stream is None:
            st = _marshal.grad_norm(self._at["resbm_grad_norm"], plan.host_ptr, plan.table, max_norm, out, ws)
            if st is not None:
                return self._check("resbm_grad_norm", st)
        _vector(out, 2, "out")
        if out.device != plan.device:
            raise ValueError(f"out: expected a tensor on {plan.device}")
        if ws is None:
            with _allocating_on(stream, plan.device):
                ws = self.grad_norm_workspace(plan)
        _one_gpu("grad_norm", plan.table, out, ws)
        self._run("resbm_grad_norm", plan, stream, plan.host_ptr, plan.table_ptr, max_norm, _ptr(out), *_room(ws))


_LOADED: dict[str, Library] = {}


def library(variant: str = "bf16") -> Library:
    """The loaded library variant ("bf16" = libresbm.so, "f32" = libresbm_f32.so)."""
    if variant not in _LOADED:
        _LOADED[variant] = Library(variant)
    return _LOADED[variant]
