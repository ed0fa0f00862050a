"""ctypes binding of liblstm355 (include/lstm355.h).

Argument marshalling only: every computation runs in the library's HIP
kernels.  torch supplies device memory (`data_ptr()`) and streams
(`torch.cuda.current_stream().cuda_stream`).  If the shared library is
missing, importing this module raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Dict, List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "liblstm355.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "lstm355.h")

LSTM_OK, LSTM_ERR_INVALID_ARG, LSTM_ERR_UNSUPPORTED, LSTM_ERR_WORKSPACE, LSTM_ERR_HIP, LSTM_ERR_TIMEOUT = range(6)
LSTM_F32, LSTM_BF16 = 0, 1


class lstm_desc_t(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("B", ctypes.c_int), ("I", ctypes.c_int), ("H", ctypes.c_int),
                ("Hp", ctypes.c_int), ("dtype", ctypes.c_int), ("reverse", ctypes.c_int),
                ("ldx", ctypes.c_long), ("ldy", ctypes.c_long)]


class lstm_kernel_stat_t(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int), ("total_ms", ctypes.c_double),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


class lstm_linattn_desc_t(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("B", ctypes.c_int), ("N", ctypes.c_int), ("K", ctypes.c_int),
                ("M", ctypes.c_int), ("dtype", ctypes.c_int), ("scale", ctypes.c_float),
                ("ldq", ctypes.c_long), ("ldk", ctypes.c_long), ("ldv", ctypes.c_long), ("ldo", ctypes.c_long)]


class LSTMError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: status {status} ({detail})")
        self.status = status


_lib = None


def load_library():
    """Loads liblstm355.so (built by paper_1907_13257_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_1907_13257_amd.build` "
                          "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i, sz, lg, fl = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_long, ctypes.c_float
    LA = ctypes.POINTER(lstm_linattn_desc_t)
    H = ctypes.c_void_p  # lstm_handle_t
    sig = {
        "lstm_create": ([ctypes.POINTER(lstm_desc_t), ctypes.POINTER(H)], i),
        "lstm_reserve_size": ([H], sz),
        "lstm_workspace_size": ([H], sz),
        "lstm_forward": ([H] + [vp] * 11 + [sz, vp, sz, vp], i),
        "lstm_backward": ([H] + [vp] * 11 + [sz] + [vp] * 7 + [i, vp, sz, vp], i),
        "lstm_forward_noalloc": ([H] + [vp] * 11 + [sz, vp], i),
        "lstm_forward_stack": ([i] + [vp] * 9 + [sz, vp, sz, vp], i),
        "lstm_backward_stack": ([i] + [vp] * 9 + [sz] + [vp] * 4 + [i, vp, sz, vp], i),
        "lstm_backward_stack_workspace_size": ([i, vp], sz),
        "lstm_check": ([H, vp, vp], i),
        "lstm_destroy": ([H], i),
        "lstm_status_string": ([i], ctypes.c_char_p),
        "lstm_last_error_detail": ([], ctypes.c_char_p),
        "lstm_describe_tiling": ([H, ctypes.POINTER(ctypes.c_int)], i),
        "lstm_add": ([i, sz, vp, vp, vp, vp], i),
        "lstm_embed_forward": ([i, lg, lg, i, vp, vp, fl, vp, lg, vp], i),
        "lstm_embed_workspace_size": ([lg, lg, i], sz),
        "lstm_embed_backward": ([i, lg, lg, i, vp, vp, lg, fl, vp, i, vp, sz, vp], i),
        "lstm_add_norm": ([i, lg, i, vp, lg, vp, lg, vp, fl, vp, vp, lg, vp], i),
        "lstm_add_norm_q8": ([i, lg, i, vp, lg, vp, lg, vp, fl, vp, vp, vp, vp], i),
        "lstm_add_norm_workspace_size": ([lg, i], sz),
        "lstm_add_norm_backward": ([i, lg, i, vp, lg, vp, vp, lg, vp, fl, vp, lg, vp, i, vp, sz, vp], i),
        "lstm_linattn_workspace_size": ([LA], sz),
        "lstm_linattn_forward": ([LA] + [vp] * 9 + [sz, vp], i),
        "lstm_linattn_backward": ([LA] + [vp] * 13 + [sz, vp], i),
        "lstm_linattn_step": ([LA] + [vp] * 9, i),
        "lstm_profile_enable": ([i], i),
        "lstm_profile_reset": ([], i),
        "lstm_profile_read": ([ctypes.POINTER(lstm_kernel_stat_t), i, ctypes.POINTER(i)], i),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def header_functions() -> List[str]:
    """Names of the functions include/lstm355.h declares."""
    with open(HEADER) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(lstm_[a-z_0-9]+)\s*\(", text)))


def _check(st: int, where: str):
    if st != LSTM_OK:
        lib = load_library()
        raise LSTMError(st, where, lib.lstm_last_error_detail().decode())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _nbytes(t, given=None) -> int:
    """Size of a buffer: `given` when stated, else a torch tensor's bytes."""
    if given is not None:
        return int(given)
    if t is None or isinstance(t, int):
        raise ValueError("the size of a raw-pointer buffer must be given")
    return t.numel() * t.element_size()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ---------------------------------------------------------------------------
# one-to-one wrappers of the C entry points
# ---------------------------------------------------------------------------
def lstm_create(T, B, I, H, Hp=0, dtype="bf16", reverse=False, ldx=0, ldy=0) -> int:
    lib = load_library()
    d = lstm_desc_t(T, B, I, H, Hp, LSTM_BF16 if dtype == "bf16" else LSTM_F32, int(bool(reverse)), ldx, ldy)
    h = ctypes.c_void_p()
    _check(lib.lstm_create(ctypes.byref(d), ctypes.byref(h)), "lstm_create")
    return h.value


def lstm_reserve_size(h) -> int:
    return load_library().lstm_reserve_size(h)


def lstm_workspace_size(h) -> int:
    return load_library().lstm_workspace_size(h)


def lstm_forward(h, x, h0, c0, W, R, b, P, y, hT, cT, reserve, workspace, stream=None, reserve_bytes=None,
                 workspace_bytes=None):
    _check(load_library().lstm_forward(h, _ptr(x), _ptr(h0), _ptr(c0), _ptr(W), _ptr(R), _ptr(b), _ptr(P), _ptr(y),
                                       _ptr(hT), _ptr(cT), _ptr(reserve), _nbytes(reserve, reserve_bytes),
                                       _ptr(workspace), _nbytes(workspace, workspace_bytes), _stream(stream)),
           "lstm_forward")


def lstm_forward_noalloc(h, x, h0, c0, W, R, b, P, y, hT, cT, reserve, stream=None, reserve_bytes=None):
    _check(load_library().lstm_forward_noalloc(h, _ptr(x), _ptr(h0), _ptr(c0), _ptr(W), _ptr(R), _ptr(b), _ptr(P),
                                               _ptr(y), _ptr(hT), _ptr(cT), _ptr(reserve),
                                               _nbytes(reserve, reserve_bytes), _stream(stream)),
           "lstm_forward_noalloc")


def _residual_args(n, residual, sums):
    if not residual or not any(residual):
        return None, None
    flags = (ctypes.c_int * n)(*[int(bool(r)) for r in residual])
    return flags, (ctypes.c_void_p * n)(*[_ptr(v) for v in sums])


def lstm_forward_stack(handles, x, Ws, Rs, bs, ys, reserves, workspace, stream=None, residual=None,
                       sums=None) -> bool:
    """Layer-wavefront forward of a stack (lstm_forward_stack).  Returns False,
    having computed nothing that counts, when the stack does not fit it
    (LSTM_ERR_UNSUPPORTED); raises on any other error.  residual[l] / sums[l]:
    layer l's output is y_l plus its input, stored in sums[l]."""
    n = len(handles)
    arr = lambda vals: (ctypes.c_void_p * n)(*[_ptr(v) for v in vals])
    rf, sp = _residual_args(n, residual, sums)
    st = load_library().lstm_forward_stack(n, arr(handles), _ptr(x), arr(Ws), arr(Rs), arr(bs), arr(ys), rf, sp,
                                           arr(reserves), min(_nbytes(r) for r in reserves), _ptr(workspace),
                                           _nbytes(workspace), _stream(stream))
    if st == LSTM_ERR_UNSUPPORTED:
        return False
    _check(st, "lstm_forward_stack")
    return True


def lstm_backward_stack_workspace_size(handles) -> int:
    n = len(handles)
    return load_library().lstm_backward_stack_workspace_size(n, (ctypes.c_void_p * n)(*handles))


def lstm_backward_stack(handles, dy, x, Ws, Rs, ys, reserves, dx, dWs, dRs, dbs, accumulate, workspace,
                        stream=None, residual=None, sums=None) -> bool:
    """Layer-wavefront backward of a stack (lstm_backward_stack).  Returns
    False when the stack does not fit it (LSTM_ERR_UNSUPPORTED); raises on
    any other error."""
    n = len(handles)
    arr = lambda vals: (ctypes.c_void_p * n)(*[_ptr(v) for v in vals])
    rf, sp = _residual_args(n, residual, sums)
    st = load_library().lstm_backward_stack(n, arr(handles), _ptr(dy), _ptr(x), arr(Ws), arr(Rs), arr(ys), rf, sp,
                                            arr(reserves), min(_nbytes(r) for r in reserves), _ptr(dx), arr(dWs),
                                            arr(dRs), arr(dbs), int(bool(accumulate)), _ptr(workspace),
                                            _nbytes(workspace), _stream(stream))
    if st == LSTM_ERR_UNSUPPORTED:
        return False
    _check(st, "lstm_backward_stack")
    return True


def lstm_backward(h, dy, dhT, dcT, x, h0, c0, W, R, P, y, reserve, dx, dh0, dc0, dW, dR, db, dP, accumulate,
                  workspace, stream=None, reserve_bytes=None, workspace_bytes=None):
    _check(load_library().lstm_backward(h, _ptr(dy), _ptr(dhT), _ptr(dcT), _ptr(x), _ptr(h0), _ptr(c0), _ptr(W),
                                        _ptr(R), _ptr(P), _ptr(y), _ptr(reserve), _nbytes(reserve, reserve_bytes),
                                        _ptr(dx), _ptr(dh0), _ptr(dc0), _ptr(dW), _ptr(dR), _ptr(db), _ptr(dP),
                                        int(bool(accumulate)), _ptr(workspace), _nbytes(workspace, workspace_bytes),
                                        _stream(stream)),
           "lstm_backward")


def lstm_check(h, workspace, stream=None) -> int:
    return load_library().lstm_check(h, _ptr(workspace), _stream(stream))


def lstm_destroy(h):
    _check(load_library().lstm_destroy(h), "lstm_destroy")


def lstm_status_string(s: int) -> str:
    return load_library().lstm_status_string(s).decode()


def lstm_last_error_detail() -> str:
    return load_library().lstm_last_error_detail().decode()


def lstm_describe_tiling(h) -> List[int]:
    out = (ctypes.c_int * 8)()
    _check(load_library().lstm_describe_tiling(h, out), "lstm_describe_tiling")
    return list(out)


def lstm_add(dtype, n, a, b, out, stream=None):
    _check(load_library().lstm_add(LSTM_BF16 if dtype == "bf16" else LSTM_F32, n, _ptr(a), _ptr(b), _ptr(out),
                                   _stream(stream)), "lstm_add")


def _dtype_code(dtype) -> int:
    if dtype not in ("bf16", "f32"):
        raise ValueError(f"dtype must be 'bf16' or 'f32', got {dtype!r}")
    return LSTM_BF16 if dtype == "bf16" else LSTM_F32


def lstm_embed_forward(dtype, N, V, D, ids, table, scale, out, ldo=0, stream=None):
    _check(load_library().lstm_embed_forward(_dtype_code(dtype), N, V, D, _ptr(ids), _ptr(table), scale, _ptr(out),
                                             ldo, _stream(stream)), "lstm_embed_forward")


def lstm_embed_workspace_size(N, V, D) -> int:
    return load_library().lstm_embed_workspace_size(N, V, D)


def lstm_embed_backward(dtype, N, V, D, ids, dout, scale, dtable, accumulate, workspace, ldo=0, stream=None,
                        workspace_bytes=None):
    _check(load_library().lstm_embed_backward(_dtype_code(dtype), N, V, D, _ptr(ids), _ptr(dout), ldo, scale,
                                              _ptr(dtable), int(bool(accumulate)), _ptr(workspace),
                                              _nbytes(workspace, workspace_bytes), _stream(stream)),
           "lstm_embed_backward")


def lstm_add_norm(dtype, rows, D, x, res, g, eps, sum, y, ldx=0, ldr=0, ldy=0, stream=None):
    _check(load_library().lstm_add_norm(_dtype_code(dtype), rows, D, _ptr(x), ldx, _ptr(res), ldr, _ptr(g), eps,
                                        _ptr(sum), _ptr(y), ldy, _stream(stream)), "lstm_add_norm")


def lstm_add_norm_q8(dtype, rows, D, x, res, g, eps, sum, y8, scale, ldx=0, ldr=0, stream=None):
    _check(load_library().lstm_add_norm_q8(_dtype_code(dtype), rows, D, _ptr(x), ldx, _ptr(res), ldr, _ptr(g), eps,
                                           _ptr(sum), _ptr(y8), _ptr(scale), _stream(stream)), "lstm_add_norm_q8")


def lstm_add_norm_workspace_size(rows, D) -> int:
    return load_library().lstm_add_norm_workspace_size(rows, D)


def lstm_add_norm_backward(dtype, rows, D, dy, dsum, sum, g, eps, dx, dg, accumulate, workspace, ldx=0, ldr=0, ldy=0,
                           stream=None, workspace_bytes=None):
    _check(load_library().lstm_add_norm_backward(_dtype_code(dtype), rows, D, _ptr(dy), ldy, _ptr(dsum), _ptr(sum),
                                                 ldr, _ptr(g), eps, _ptr(dx), ldx, _ptr(dg), int(bool(accumulate)),
                                                 _ptr(workspace), _nbytes(workspace, workspace_bytes),
                                                 _stream(stream)), "lstm_add_norm_backward")


def lstm_linattn_desc(T, B, N, K, M, dtype="bf16", scale=1.0, ldq=0, ldk=0, ldv=0, ldo=0) -> lstm_linattn_desc_t:
    return lstm_linattn_desc_t(T, B, N, K, M, _dtype_code(dtype), scale, ldq, ldk, ldv, ldo)


def lstm_linattn_workspace_size(desc) -> int:
    return load_library().lstm_linattn_workspace_size(ctypes.byref(desc))


def lstm_linattn_forward(desc, q, k, v, decay, lengths, S0, o, ST, workspace, stream=None, workspace_bytes=None):
    _check(load_library().lstm_linattn_forward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(decay),
                                               _ptr(lengths), _ptr(S0), _ptr(o), _ptr(ST), _ptr(workspace),
                                               _nbytes(workspace, workspace_bytes), _stream(stream)),
           "lstm_linattn_forward")


def lstm_linattn_backward(desc, do, q, k, v, decay, lengths, S0, dST, dq, dk, dv, dS0, workspace, stream=None,
                          workspace_bytes=None):
    _check(load_library().lstm_linattn_backward(ctypes.byref(desc), _ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(decay),
                                                _ptr(lengths), _ptr(S0), _ptr(dST), _ptr(dq), _ptr(dk), _ptr(dv),
                                                _ptr(dS0), _ptr(workspace), _nbytes(workspace, workspace_bytes),
                                                _stream(stream)), "lstm_linattn_backward")


def lstm_linattn_step(desc, q, k, v, decay, lengths, S, S_out, o, stream=None):
    _check(load_library().lstm_linattn_step(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(decay), _ptr(lengths),
                                            _ptr(S), _ptr(S_out), _ptr(o), _stream(stream)), "lstm_linattn_step")


def lstm_profile_enable(on: bool):
    _check(load_library().lstm_profile_enable(int(bool(on))), "lstm_profile_enable")


def lstm_profile_reset():
    _check(load_library().lstm_profile_reset(), "lstm_profile_reset")


def lstm_profile_read() -> Dict[str, dict]:
    arr = (lstm_kernel_stat_t * 16)()
    n = ctypes.c_int()
    _check(load_library().lstm_profile_read(arr, 16, ctypes.byref(n)), "lstm_profile_read")
    return {arr[k].name.decode(): dict(launches=arr[k].launches, total_ms=arr[k].total_ms, flops=arr[k].flops,
                                       bytes=arr[k].bytes) for k in range(n.value)}


# ---------------------------------------------------------------------------
# layers and stacks over torch-allocated device memory
# ---------------------------------------------------------------------------
def torch_dtype(dtype: str):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class Layer:
    """One LSTM/LSTMP layer or direction: owns a handle and its reserve; the
    workspace may be shared between layers whose calls are ordered."""

    def __init__(self, T, B, I, H, Hp=0, dtype="bf16", reverse=False, ldx=0, ldy=0, device="cuda",
                 workspace=None):
        import torch
        self.T, self.B, self.I, self.H, self.Hp, self.dtype, self.reverse = T, B, I, H, Hp, dtype, bool(reverse)
        self.Hr = Hp if Hp else H
        self.ldx = ldx or I
        self.ldy = ldy or self.Hr
        self.handle = lstm_create(T, B, I, H, Hp, dtype, reverse, self.ldx, self.ldy)
        self.reserve = torch.empty(lstm_reserve_size(self.handle), dtype=torch.uint8, device=device)
        self.ws_bytes = lstm_workspace_size(self.handle)
        if workspace is None:
            workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        if workspace.numel() < self.ws_bytes:
            raise ValueError("workspace too small")
        self.workspace = workspace
        self.device = device

    def close(self):
        if self.handle:
            lstm_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def forward(self, x, W, R, b, P=None, h0=None, c0=None, y=None, hT=None, cT=None, stream=None):
        lstm_forward(self.handle, x, h0, c0, W, R, b, P, y, hT, cT, self.reserve, self.workspace, stream)

    def backward(self, dy, x, W, R, y, grads, P=None, h0=None, c0=None, dhT=None, dcT=None, dx=None, dh0=None,
                 dc0=None, accumulate=False, stream=None):
        lstm_backward(self.handle, dy, dhT, dcT, x, h0, c0, W, R, P, y, self.reserve, dx, dh0, dc0, grads["dW"],
                      grads["dR"], grads["db"], grads.get("dP"), accumulate, self.workspace, stream)

    def check(self, stream=None) -> int:
        return lstm_check(self.handle, self.workspace, stream)

    def tiling(self) -> List[int]:
        return lstm_describe_tiling(self.handle)


def _rows_arg(what, dtype, rows, width, ld, gpu, optional=False):
    """A function that gives the address of a tensor on GPU `gpu` holding `rows`
    rows of `width` elements, `ld` elements apart (its leading dimensions are
    the rows, however many there are), after checking that it does.  Addresses
    pass through; None does where the argument is optional."""
    n, dense = rows * width, ld == width

    def address(t):
        if t is None or t.__class__ is int:
            if t is None and not optional:
                raise ValueError(f"{what} is required")
            return t
        if t.dtype is not dtype:
            raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
        if t.get_device() != gpu:
            raise ValueError(f"{what} is on {t.device}, the operator on cuda:{gpu}")
        if dense and t.is_contiguous() and t.numel() == n and t.dim() and t.size(-1) == width:
            return t.data_ptr()
        shape = t.shape
        found, expect = 1, ld
        ok = bool(shape) and shape[-1] == width and (width == 1 or t.stride(-1) == 1)
        for dim in range(len(shape) - 2, -1, -1):
            ok = ok and (shape[dim] == 1 or t.stride(dim) == expect)
            found *= shape[dim]
            expect *= shape[dim]
        if not ok or found != rows:
            raise ValueError(f"{what} must be {rows} rows of {width} elements, {ld} apart: got shape {tuple(shape)}, "
                             f"strides {t.stride()}")
        return t.data_ptr()

    return address


def _vector_arg(what, dtype, n, gpu, optional=False):
    """The same for n contiguous elements of any shape."""

    def address(t):
        if t is None or t.__class__ is int:
            if t is None and not optional:
                raise ValueError(f"{what} is required")
            return t
        if t.dtype is not dtype:
            raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
        if t.get_device() != gpu:
            raise ValueError(f"{what} is on {t.device}, the operator on cuda:{gpu}")
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{what} must be {n} contiguous elements, got shape {tuple(t.shape)}, strides {t.stride()}")
        return t.data_ptr()

    return address


class _Operator:
    """What the operators' classes share: the device they were made on, their
    workspace, and the stream of a call.  Calls of one object that overlap (on
    several streams) would share its workspace: order them, or make an object
    for each.  The checks of a call's tensors are made once, as functions."""

    def __init__(self, dtype, device, workspace_bytes):
        import torch
        self.code = _dtype_code(dtype)
        self.dtype, self.torch_dtype = dtype, torch_dtype(dtype)
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError(f"the operators run on a GPU, not on {self.device}")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.gpu = self.device.index
        self._current = torch.cuda.current_device
        # the current stream's handle without a Stream object around it (2.7 us
        # less per call), where this torch offers it
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.workspace = torch.empty(workspace_bytes, dtype=torch.uint8, device=self.device)
        self.ws_ptr, self.ws_bytes = (self.workspace.data_ptr() if workspace_bytes else None), workspace_bytes
        self.lib = load_library()

    def _stream(self, stream):
        if self._current() != self.gpu:
            raise ValueError(f"the operator is on {self.device}, the current device is cuda:{self._current()}")
        if stream is None and self._raw_stream:
            return self._raw_stream(self.gpu)
        return _stream(stream)

    def _rows(self, what, rows, width, ld=None, optional=False, dtype=None):
        return _rows_arg(what, dtype or self.torch_dtype, rows, width, ld or width, self.gpu, optional)

    def _vector(self, what, dtype, n, optional=False):
        return _vector_arg(what, dtype, n, self.gpu, optional)


class Embedding(_Operator):
    """Rows of a table [V][D] for N tokens (any leading shape, e.g. [T][B]),
    scaled, and the table's fp32 gradient.  Tokens outside 0 .. V-1 are
    padding: rows of zeros, no gradient."""

    def __init__(self, N, V, D, dtype="bf16", scale=1.0, ldo=0, device="cuda"):
        super().__init__(dtype, device, lstm_embed_workspace_size(N, V, D))
        import torch
        self.N, self.V, self.D, self.scale, self.ldo = N, V, D, float(scale), ldo or D
        self._ids = self._vector("ids", torch.int64, N)
        self._table, self._dtable = self._rows("table", V, D), self._rows("dtable", V, D, dtype=torch.float32)
        self._out, self._dout = self._rows("out", N, D, ldo), self._rows("dout", N, D, ldo)

    def forward(self, ids, table, out, stream=None):
        st = self.lib.lstm_embed_forward(self.code, self.N, self.V, self.D, self._ids(ids), self._table(table),
                                         self.scale, self._out(out), self.ldo, self._stream(stream))
        _check(st, "lstm_embed_forward")

    def backward(self, ids, dout, dtable, accumulate=False, stream=None):
        st = self.lib.lstm_embed_backward(self.code, self.N, self.V, self.D, self._ids(ids), self._dout(dout), self.ldo,
                                          self.scale, self._dtable(dtable), int(bool(accumulate)), self.ws_ptr,
                                          self.ws_bytes, self._stream(stream))
        _check(st, "lstm_embed_backward")


class AddNorm(_Operator):
    """Residual addition and root-mean-square norm of `rows` rows of D values:
    sum = x + res, y = sum * g / rms(sum), with y in the storage type
    (`forward`, `backward`) or in e4m3 with a scale per row (`forward_q8`)."""

    def __init__(self, rows, D, dtype="bf16", eps=1e-5, ldx=0, ldr=0, ldy=0, device="cuda"):
        super().__init__(dtype, device, lstm_add_norm_workspace_size(rows, D))
        import torch
        self.rows, self.D, self.eps = rows, D, float(eps)
        self.ldx, self.ldr, self.ldy = ldx or D, ldr or D, ldy or D
        self._x, self._res = self._rows("x", rows, D, ldx), self._rows("res", rows, D, ldr, True)
        self._sum, self._kept = self._rows("sum", rows, D, ldr, True), self._rows("sum", rows, D, ldr)
        self._y, self._dy = self._rows("y", rows, D, ldy), self._rows("dy", rows, D, ldy)
        self._dsum, self._dx = self._rows("dsum", rows, D, ldr, True), self._rows("dx", rows, D, ldx)
        self._g, self._dg = self._vector("g", self.torch_dtype, D), self._vector("dg", torch.float32, D)
        self._scale, self._uint8 = self._vector("scale", torch.float32, rows), torch.uint8
        self._y8 = self._rows("y8", rows, D, dtype=torch.float8_e4m3fn)
        self._bits = self._rows("y8", rows, D, dtype=torch.uint8)

    def forward(self, x, res, g, sum, y, stream=None):
        st = self.lib.lstm_add_norm(self.code, self.rows, self.D, self._x(x), self.ldx, self._res(res), self.ldr,
                                    self._g(g), self.eps, self._sum(sum), self._y(y), self.ldy, self._stream(stream))
        _check(st, "lstm_add_norm")

    def forward_q8(self, x, res, g, sum, y8, scale, stream=None):
        eight = self._bits if getattr(y8, "dtype", None) is self._uint8 else self._y8
        st = self.lib.lstm_add_norm_q8(self.code, self.rows, self.D, self._x(x), self.ldx, self._res(res), self.ldr,
                                       self._g(g), self.eps, self._sum(sum), eight(y8), self._scale(scale),
                                       self._stream(stream))
        _check(st, "lstm_add_norm_q8")

    def backward(self, dy, dsum, sum, g, dx, dg, accumulate=False, stream=None):
        st = self.lib.lstm_add_norm_backward(self.code, self.rows, self.D, self._dy(dy), self.ldy, self._dsum(dsum),
                                             self._kept(sum), self.ldr, self._g(g), self.eps, self._dx(dx), self.ldx,
                                             self._dg(dg), int(bool(accumulate)), self.ws_ptr, self.ws_bytes,
                                             self._stream(stream))
        _check(st, "lstm_add_norm_backward")


class LinearAttention(_Operator):
    """A recurrent layer of linear attention with one decay per head:
    S_t = decay S_{t-1} + k_t v_t^T, o_t = scale q_t S_t (scale defaults to
    1 / sqrt(K)).  q, k [T][B][heads*K], v, o [T][B][heads*M], states
    [B][heads][K][M] fp32, decay [heads] fp32, lengths [B] int32 or None.
    `step` takes one token of every row (T = 1)."""

    def __init__(self, T, B, heads, K, M, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0, ldo=0, device="cuda"):
        scale = K ** -0.5 if scale is None else float(scale)
        self.desc = lstm_linattn_desc(T, B, heads, K, M, dtype, scale, ldq, ldk, ldv, ldo)
        super().__init__(dtype, device, lstm_linattn_workspace_size(self.desc))
        import torch
        self.T, self.B, self.heads, self.K, self.M, self.scale = T, B, heads, K, M, scale
        self._desc = ctypes.byref(self.desc)
        rows, hk, hm, states = T * B, heads * K, heads * M, B * heads * K * M
        self._q, self._k, self._v = (self._rows("q", rows, hk, ldq), self._rows("k", rows, hk, ldk),
                                     self._rows("v", rows, hm, ldv))
        self._o, self._do = self._rows("o", rows, hm, ldo), self._rows("do", rows, hm, ldo)
        self._dq, self._dk, self._dv = (self._rows("dq", rows, hk, ldq, True), self._rows("dk", rows, hk, ldk, True),
                                        self._rows("dv", rows, hm, ldv, True))
        self._decay = self._vector("decay", torch.float32, heads)
        self._lengths = self._vector("lengths", torch.int32, B, True)
        self._S, self._S_out = self._vector("S", torch.float32, states), self._vector("S_out", torch.float32, states)
        self._S0, self._ST, self._dST, self._dS0 = (self._vector(n, torch.float32, states, True)
                                                    for n in ("S0", "ST", "dST", "dS0"))

    def forward(self, q, k, v, decay, o, lengths=None, S0=None, ST=None, stream=None):
        st = self.lib.lstm_linattn_forward(self._desc, self._q(q), self._k(k), self._v(v), self._decay(decay),
                                           self._lengths(lengths), self._S0(S0), self._o(o), self._ST(ST), self.ws_ptr,
                                           self.ws_bytes, self._stream(stream))
        _check(st, "lstm_linattn_forward")

    def backward(self, do, q, k, v, decay, dq, dk, dv, lengths=None, S0=None, dST=None, dS0=None, stream=None):
        st = self.lib.lstm_linattn_backward(self._desc, self._do(do), self._q(q), self._k(k), self._v(v),
                                            self._decay(decay), self._lengths(lengths), self._S0(S0), self._dST(dST),
                                            self._dq(dq), self._dk(dk), self._dv(dv), self._dS0(dS0), self.ws_ptr,
                                            self.ws_bytes, self._stream(stream))
        _check(st, "lstm_linattn_backward")

    def step(self, q, k, v, decay, S, S_out, o, lengths=None, stream=None):
        st = self.lib.lstm_linattn_step(self._desc, self._q(q), self._k(k), self._v(v), self._decay(decay),
                                        self._lengths(lengths), self._S(S), self._S_out(S_out), self._o(o),
                                        self._stream(stream))
        _check(st, "lstm_linattn_step")


class StackLayer:
    """A layer of a Stack.  residual: its output is y plus the residual stream
    (for a layer without norms below it, its own input).  norm (residual layers
    only): the sum goes on as the residual stream and its root-mean-square norm
    with the gain params["g"] is what the next layer reads."""

    def __init__(self, I, H, Hp=0, bidirectional=False, residual=False, norm=False):
        self.I, self.H, self.Hp, self.bidirectional, self.residual, self.norm = I, H, Hp, bidirectional, residual, norm
        if norm and not residual:
            raise ValueError("a layer with a norm is a residual layer")
        self.Hr = Hp if Hp else H
        self.out = self.Hr * (2 if bidirectional else 1)


class Stack:
    """A stack of layers composed through the C ABI: a bidirectional layer
    runs its two directions into the halves of one output buffer (row stride
    2*Hr); a residual layer's output is y + x (lstm_add).  Backward mirrors it:
    the directions' input gradients and the identity path are summed with
    lstm_add.  Initial states are zero and the final states get no gradient.
    A residual layer with a norm hands its sum on as the residual stream of the
    layers above and the norm of the sum as their input (lstm_add_norm).  With
    `vocab` rows of an embedding the stack's input is token ids [T][B] and a
    table [vocab][I], its rows scaled by embed_scale.

    params[l][d] = dict(W, R, b[, P]) device tensors; grads likewise with
    dW, dR, db[, dP] (fp32), allocated here.  params[l][0]["g"] and
    grads[l][0]["dg"]: the gain of a layer's norm."""

    def __init__(self, T, B, layers: Sequence[StackLayer], dtype="bf16", device="cuda", wavefront=True, vocab=0,
                 embed_scale=1.0, eps=1e-5):
        import torch
        self.T, self.B, self.dtype, self.device = T, B, dtype, device
        self.wavefront = wavefront
        self.last_forward = None
        self.last_backward = None
        self.wave_ws = None
        self.layers = list(layers)
        td = torch_dtype(dtype)
        self.dirs: List[List[Layer]] = []
        ws_bytes = 0
        shapes = []
        for L in self.layers:
            if L.residual and L.out != L.I:
                raise ValueError("residual layer needs input width == output width")
            nd = 2 if L.bidirectional else 1
            shapes.append(nd)
            for d in range(nd):
                h = lstm_create(T, B, L.I, L.H, L.Hp, dtype, d == 1, L.I, L.out)
                ws_bytes = max(ws_bytes, lstm_workspace_size(h))
                lstm_destroy(h)
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
        for L, nd in zip(self.layers, shapes):
            self.dirs.append([Layer(T, B, L.I, L.H, L.Hp, dtype, d == 1, L.I, L.out, device, self.workspace)
                              for d in range(nd)])
        self.y = [torch.empty((T, B, L.out), dtype=td, device=device) for L in self.layers]
        self.xout = [torch.empty((T, B, L.out), dtype=td, device=device) if L.residual else None
                     for L in self.layers]
        self.inputs: List = [None] * len(self.layers)
        self.dxbuf = [[torch.empty((T, B, L.I), dtype=td, device=device) for _ in range(2 if L.bidirectional else 1)]
                      for L in self.layers]
        self.gbuf = [torch.empty((T, B, L.I), dtype=td, device=device) for L in self.layers]
        self.norms = [AddNorm(T * B, L.out, dtype, eps, device=device) if L.norm else None for L in self.layers]
        self.nout = [torch.empty((T, B, L.out), dtype=td, device=device) if L.norm else None for L in self.layers]
        self.dsum = [torch.empty((T, B, L.out), dtype=td, device=device) if L.norm else None for L in self.layers]
        self.embedding = self.rows = self.ids = None
        if vocab:
            self.embedding = Embedding(T * B, vocab, self.layers[0].I, dtype, embed_scale, device=device)
            self.rows = torch.empty((T, B, self.layers[0].I), dtype=td, device=device)

    def alloc_grads(self, params):
        import torch
        grads = []
        for L, prm in zip(self.layers, params):
            gl = []
            for p in prm:
                g = dict(dW=torch.empty(p["W"].shape, dtype=torch.float32, device=self.device),
                         dR=torch.empty(p["R"].shape, dtype=torch.float32, device=self.device),
                         db=torch.empty(p["b"].shape, dtype=torch.float32, device=self.device))
                if L.Hp:
                    g["dP"] = torch.empty(p["P"].shape, dtype=torch.float32, device=self.device)
                if "g" in p:
                    g["dg"] = torch.empty(p["g"].shape, dtype=torch.float32, device=self.device)
                gl.append(g)
            grads.append(gl)
        return grads

    def forward(self, x, params, stream=None, table=None):
        if self.embedding is not None:
            self.ids = x
            self.embedding.forward(x, table, self.rows, stream)
            x = self.rows
        # a stack of unidirectional LSTM layers (residual ones included) runs
        # as one layer wavefront when the library supports its shape
        # (lstm_forward_stack)
        self.last_forward = "layers"
        if (self.wavefront and 2 <= len(self.layers) <= 4 and self.dtype == "bf16"
                and all(not L.bidirectional and not L.Hp and not L.norm for L in self.layers)):
            lays = [d[0] for d in self.dirs]
            residual = [L.residual for L in self.layers]
            if lstm_forward_stack([l.handle for l in lays], x, [p[0]["W"] for p in params],
                                  [p[0]["R"] for p in params], [p[0]["b"] for p in params], self.y,
                                  [l.reserve for l in lays], self.workspace, stream, residual=residual,
                                  sums=self.xout):
                outs = [self.xout[li] if L.residual else self.y[li] for li, L in enumerate(self.layers)]
                self.inputs = [x] + outs[:-1]
                self.last_forward = "wavefront"
                return outs[-1]
        cur = carry = x   # the layer's input, and the residual stream beside it
        for li, L in enumerate(self.layers):
            self.inputs[li] = cur
            y = self.y[li]
            for d, lay in enumerate(self.dirs[li]):
                p = params[li][d]
                yd = y[:, :, d * L.Hr:] if d else y
                lay.forward(cur, p["W"], p["R"], p["b"], p.get("P"), y=yd, stream=stream)
            if L.norm:
                self.norms[li].forward(y, carry, params[li][0]["g"], self.xout[li], self.nout[li], stream)
                cur, carry = self.nout[li], self.xout[li]
            elif L.residual:
                lstm_add(self.dtype, y.numel(), y, carry, self.xout[li], stream)
                cur = carry = self.xout[li]
            else:
                cur = carry = y
        return cur

    def backward(self, d_out, params, grads, accumulate=False, stream=None, dtable=None):
        """Gradients of the layers, and of the embedding's table into `dtable`
        where there is one; returns the gradient of the first layer's input."""
        if self.embedding is not None and dtable is None:
            raise ValueError("dtable is required: the stack has an embedding")
        dx = self._backward_layers(d_out, params, grads, accumulate, stream)
        if self.embedding is not None:
            self.embedding.backward(self.ids, dx, dtable, accumulate, stream)
        return dx

    def _backward_layers(self, d_out, params, grads, accumulate, stream):
        # after a wavefront forward, the backward runs as one too when its
        # shapes allow (lstm_backward_stack)
        self.last_backward = "layers"
        if self.last_forward == "wavefront":
            lays = [d[0] for d in self.dirs]
            hs = [l.handle for l in lays]
            need = lstm_backward_stack_workspace_size(hs)
            if need:
                import torch
                if self.wave_ws is None or self.wave_ws.numel() < need:
                    self.wave_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
                dx = self.dxbuf[0][0]
                if lstm_backward_stack(hs, d_out, self.inputs[0], [p[0]["W"] for p in params],
                                       [p[0]["R"] for p in params], self.y, [l.reserve for l in lays], dx,
                                       [g[0]["dW"] for g in grads], [g[0]["dR"] for g in grads],
                                       [g[0]["db"] for g in grads], accumulate, self.wave_ws, stream,
                                       residual=[L.residual for L in self.layers], sums=self.xout):
                    self.last_backward = "wavefront"
                    return dx
        g, gc = d_out, None   # gradients of the layer's output and, past a norm, of the residual stream
        for li in range(len(self.layers) - 1, -1, -1):
            L = self.layers[li]
            x = self.inputs[li]
            y = self.y[li]
            if L.norm:
                self.norms[li].backward(g, gc, self.xout[li], params[li][0]["g"], self.dsum[li], grads[li][0]["dg"],
                                        accumulate, stream)
                g = self.dsum[li]
            for d, lay in enumerate(self.dirs[li]):
                p = params[li][d]
                off = d * L.Hr
                lay.backward(g[:, :, off:] if d else g, x, p["W"], p["R"], y[:, :, off:] if d else y,
                             grads[li][d], P=p.get("P"), dx=self.dxbuf[li][d], accumulate=accumulate,
                             stream=stream)
            dx = self.dxbuf[li][0]
            out = self.gbuf[li]
            if L.bidirectional:
                lstm_add(self.dtype, dx.numel(), dx, self.dxbuf[li][1], out, stream)
                dx = out
            if li > 0 and self.layers[li - 1].norm:
                g, gc = dx, (g if L.residual else None)
                continue
            if L.residual:
                lstm_add(self.dtype, dx.numel(), dx, g, out, stream)
                dx = out
            g, gc = dx, None
        return g

    def check(self, stream=None) -> int:
        return lstm_check(self.dirs[0][0].handle, self.workspace, stream)
