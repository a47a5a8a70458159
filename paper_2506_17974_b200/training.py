"""Training operators of liblqsgd.so: the layers whose weight gradients a round compresses.

    linear / linear_grad_input / linear_grad_weight    a linear layer's three products, bias, activation and residual in the
                                                       epilogue
    pack8 / unpack8 / act_grad                         activations kept in 8 bits until the backward pass
    group_norm / group_norm_grad                       group norm with an activation, channels last
    rms_norm / rms_norm_grad                           root-mean-square norm of rows, dropout and the residual's addition in front
    dropout                                            from a counter-based generator, the mask is never stored
    pack_rows8 / unpack_rows8 / linear_rows8           rows of signed 8-bit codes, a linear layer's forward product of them

A tensor given as `out` is written in place, which autograd is told.

Argument marshalling only, as in binding.py: tensors are checked here for type, device and layout, everything else by the
library; the arithmetic runs in its CUDA kernels, on the current stream of the tensors' device.  The `*_layer` functions
are the same operators as differentiable functions that keep only 8-bit activations between the passes.
"""
from __future__ import annotations

import ctypes as C
import struct
import threading
from operator import index
from typing import NamedTuple, Optional, Tuple, Union

import torch
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from . import binding as B

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
GROUP = 32
FORWARD, GRAD_INPUT, GRAD_WEIGHT = 0, 1, 2


# lqsgd_packed8, lqsgd_linear and lqsgd_group_norm as they lie in memory, fields in the header's order.  The calls are short
# enough on the device for the host to be their cost, so arguments are packed in one go.
_PACKED8 = struct.Struct("@PqPq")
_LINEAR = struct.Struct("@Iiii q ii PqPqPq P Pq Pq PqPq PqPq PqPq P PN")
_NORM = struct.Struct("@Iiiiiiif PqqPqqPqq PP PP PP PqPq PqPq PN")
_NONE8 = (0, 0, 0, 0)
# lqsgd_rows8, lqsgd_drop, lqsgd_rms_norm and lqsgd_linear_rows8 (whose operands and kept copies are the first two's fields)
_ROWS8 = struct.Struct("@PqP")
_DROP = struct.Struct("@fIQQP")
_RMS = struct.Struct("@Ii q if fIQQP PqPqPqPq PqPqPqPq PPP PqPq PqPq PqP PN")
_LINEAR8 = struct.Struct("@IiiI q ii PqP PqP P Pq Pq PqPq PqPq P PN")
_NO_ROWS8 = (0, 0, 0)

_lib = None


def _library() -> C.CDLL:
    global _lib
    if _lib is None:
        lib = B.load_library()
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        lib.lqsgd_pack8.argtypes = [vp, i64, i32, i64, i32, vp, vp]
        lib.lqsgd_unpack8.argtypes = [vp, i64, i32, vp, i64, i32, vp]
        lib.lqsgd_act_grad_workspace_bytes.argtypes = [i64, i32, C.POINTER(sz)]
        lib.lqsgd_act_grad.argtypes = [vp, i64, vp, i32, i32, i64, i32, vp, i64, vp, vp, sz, vp]
        lib.lqsgd_linear_workspace_bytes.argtypes = [i32, vp, C.POINTER(sz)]
        lib.lqsgd_group_norm_workspace_bytes.argtypes = [i32, vp, C.POINTER(sz)]
        lib.lqsgd_pack_rows8.argtypes = [vp, i64, i32, i64, i32, vp, vp]
        lib.lqsgd_unpack_rows8.argtypes = [vp, i64, i32, vp, i64, i32, vp]
        lib.lqsgd_dropout.argtypes = [vp, i64, vp, i64, i32, i64, i32, vp, vp, i64, vp]
        lib.lqsgd_rms_norm_workspace_bytes.argtypes = [i32, vp, C.POINTER(sz)]
        lib.lqsgd_linear_rows8_workspace_bytes.argtypes = [vp, C.POINTER(sz)]
        for f in (lib.lqsgd_rms_norm_forward, lib.lqsgd_rms_norm_backward, lib.lqsgd_linear_rows8_forward, lib.lqsgd_linear_forward, lib.lqsgd_linear_grad_input, lib.lqsgd_linear_grad_weight,
                  lib.lqsgd_group_norm_forward, lib.lqsgd_group_norm_backward):
            f.argtypes = [vp, vp]
        _lib = lib
    return _lib


def _act(name: str) -> int:
    code = ACTS.get(name)
    if code is None:
        raise ValueError(f"act must be one of {sorted(ACTS)}, not {name!r}")
    return code


def _dtype(t: torch.Tensor, what: str, products: bool = False) -> int:
    code = DTYPES.get(t.dtype)
    if code is None or (products and code == 2):
        raise ValueError(f"{what} must be bfloat16 or float16" + ("" if products else " or float32") + f", not {t.dtype}")
    return code


# The calls below are short on the device, so their own cost on the host counts: a matrix is checked and taken apart in one
# go, arguments are packed in one go, and nothing is formatted unless it is refused.

def _matrix(t: torch.Tensor, what: str, device: int, dtype: Optional[torch.dtype] = None, rows: int = -1, cols: int = -1) -> Tuple[int, int]:
    """(address, elements between rows) of a checked matrix; device is the index that all tensors of the call are on."""
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{what} must be a matrix")
    r, c = shape
    ld, one = t.stride()
    if one != 1 and c > 1:
        raise ValueError(f"{what} must have unit stride along its rows")
    if t.get_device() != device or device < 0:
        raise ValueError(f"{what} must be a CUDA tensor on the device of the call's other tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, not {t.dtype}")
    if c >> 31:                       # the library's counts of columns are 32 bits wide: more would arrive as another number
        raise ValueError(f"{what} must have fewer than 2^31 columns, not {c}")
    if (rows >= 0 and r != rows) or (cols >= 0 and c != cols):
        raise ValueError(f"{what} must have {rows if rows >= 0 else 'any number of'} rows and {cols if cols >= 0 else 'any number of'} columns, "
                         f"not {tuple(shape)}")
    return t.data_ptr(), ld if r > 1 or ld > c else c


def _vector(t: torch.Tensor, what: str, device: int, n: int) -> int:
    """Address of a checked float32 vector."""
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what} must be a contiguous float32 vector of {n} on the call's device")
    return t.data_ptr()


_MOST, _WORD = 3.4028234663852886e38, 0xFFFFFFFFFFFFFFFF


def _real(v: float, what: str) -> float:
    """v, which the library takes as a float32; what that cannot hold would not be packed."""
    if abs(v) > _MOST:
        raise ValueError(f"{what} must be a number of float32's range, not {v}")
    return v


def _elsewhere(device: int) -> bool:
    """Whether `device` is not the current one: the calls then run again under torch.cuda.device."""
    if device < 0:
        raise ValueError("the tensors must be CUDA tensors")
    return torch._C._cuda_getDevice() != device


_stream = torch._C._cuda_getCurrentRawStream


# Workspaces up to _KEEP bytes are kept per host thread, device and stream for the life of the thread, so that a call in a training step needs no
# allocation of its own; larger ones, and those of calls that are being captured in a graph (whose memory has to last as
# long as the graph), come from PyTorch's allocator for the one call.  Calls of one thread on one stream follow one
# another, so they may share one; the allocator does not hand out a call's own workspace again before its kernels are done.
_KEEP = 16 << 20


class _Scratch(threading.local):
    def __init__(self):
        self.kept = {}


_scratch = _Scratch()


def _workspace(need: int, device: torch.device, stream: int) -> torch.Tensor:
    if need > _KEEP or torch._C._cuda_isCurrentStreamCapturing():
        return torch.empty_strided((need,), (1,), dtype=torch.uint8, device=device)
    ws = torch.empty_strided((max(need, 1 << 20),), (1,), dtype=torch.uint8, device=device)
    _scratch.kept[(device.index, stream)] = (ws, ws.data_ptr(), ws.numel())
    return ws


_NO_SCRATCH = (None, 0, 0)


def _kept_scratch(index: int, stream: int) -> tuple:
    if torch._C._cuda_isCurrentStreamCapturing():
        return _NO_SCRATCH
    return _scratch.kept.get((index, stream), _NO_SCRATCH)


def _call(fn, args: tuple, layout: struct.Struct, bytes_fn, which: int, device: torch.device) -> None:
    """Runs fn on a packed argument struct whose last two fields are the workspace: the kept one, or, where the library refuses
    that as too small (on the host, before anything is launched), one of the size it asks for."""
    stream = _stream(device.index)
    _, ptr, size = _kept_scratch(device.index, stream)
    rc = fn(layout.pack(*args, ptr, size), stream)
    if rc == B.ERR_WORKSPACE_TOO_SMALL:
        need = C.c_size_t(0)
        B._check(bytes_fn(which, layout.pack(*args, 0, 0), C.byref(need)))
        ws = _workspace(need.value, device, stream)
        rc = fn(layout.pack(*args, ws.data_ptr(), ws.numel()), stream)
    if rc != 0:
        B._check(rc)


def _written(*tensors: torch.Tensor) -> None:
    """Tells autograd that a caller's tensors were written in place: a backward pass that saved one then raises, as after
    PyTorch's own in-place operators (tensors of inference mode have no such history)."""
    for t in tensors:
        if not t.is_inference():
            increment_version(t)


def _empty(rows: int, cols: int, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)


_status = {}


def _status_word(device: torch.device) -> int:
    word = _status.get(device.index)
    if word is None:
        if torch.cuda.is_current_stream_capturing():
            return 0
        word = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.current_stream(device).synchronize()
        _status[device.index] = word
    return word.data_ptr()


def status(device: Union[str, int, torch.device] = "cuda:0") -> int:
    """Status bits (binding.STATUS_TIMEOUT) that the linear layers' kernels have raised on a device ("cuda": the current one) so
    far; synchronises.  Products captured in a graph before the device's first ordinary one have no status word and raise none."""
    index = torch.device(device).index
    word = _status.get(torch.cuda.current_device() if index is None else index)
    return 0 if word is None else int(word.item())


# ------------------------------------------------------------------------------------------------ activations in 8 bits

class Packed8:
    """A matrix kept in 8 bits: codes, uint8 rows x cols, and exps, uint8 rows x ceil(cols / 32) (see lqsgd_packed8)."""

    __slots__ = ("codes", "exps")

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor):
        self.codes, self.exps = codes, exps
        self.fields()

    @staticmethod
    def empty(rows: int, cols: int, device) -> "Packed8":
        """Uninitialised; rows of codes start on 16-byte boundaries."""
        p = object.__new__(Packed8)
        p.codes = torch.empty_strided((rows, cols), ((cols + 15) & -16, 1), dtype=torch.uint8, device=device)
        p.exps = _empty(rows, (cols + GROUP - 1) // GROUP, torch.uint8, device)
        return p

    def _fresh(self) -> Tuple[int, int, int, int]:
        """fields() of what empty() just made."""
        rows, cols = self.codes.shape
        return self.codes.data_ptr(), (cols + 15) & -16, self.exps.data_ptr(), (cols + GROUP - 1) // GROUP

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def fields(self) -> Tuple[int, int, int, int]:
        """The members of lqsgd_packed8, checked."""
        codes, exps = self.codes, self.exps
        dev = codes.get_device()
        cp, cl = _matrix(codes, "codes", dev, torch.uint8)
        ep, el = _matrix(exps, "exps", dev, torch.uint8, codes.shape[0], (codes.shape[1] + GROUP - 1) // GROUP)
        return cp, cl, ep, el


def _kept(p: Optional[Packed8], what: str, device: int, rows: int, cols: int = -1) -> Tuple[int, int, int, int]:
    """The fields of an 8-bit argument of rows x cols (any number of columns where -1)."""
    if p is None:
        raise ValueError(f"{what} must be the 8-bit form of a matrix")
    r, c = p.codes.shape
    if r != rows or (cols >= 0 and c != cols) or p.codes.get_device() != device:
        raise ValueError(f"{what} must be the 8-bit form of {rows} x {cols if cols >= 0 else 'any'} values on the call's device, not of {r} x {c}")
    return p.fields()


def pack8(x: torch.Tensor, out: Optional[Packed8] = None) -> Packed8:
    """The 8-bit form of a matrix (bfloat16, float16 or float32)."""
    dev = x.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return pack8(x, out)
    xp, xl = _matrix(x, "x", dev)
    rows, cols = x.shape
    given = out is not None
    if given:
        of = _kept(out, "out", dev, rows, cols)
    else:
        out = Packed8.empty(rows, cols, x.device)
        of = out._fresh()
    rc = _library().lqsgd_pack8(xp, xl, _dtype(x, "x"), rows, cols, _PACKED8.pack(*of), _stream(dev))
    if rc:
        B._check(rc)
    if given:
        _written(out.codes, out.exps)
    return out


def unpack8(p: Packed8, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values an 8-bit form stands for: exact in bfloat16 and float32 (float16: within its range)."""
    codes = p.codes
    dev = codes.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return unpack8(p, dtype, out)
    rows, cols = codes.shape
    if dtype not in DTYPES:
        raise ValueError(f"dtype must be one of {list(DTYPES)}")
    y = _empty(rows, cols, dtype, codes.device) if out is None else out
    yp, yl = _matrix(y, "out", dev, dtype, rows, cols)
    rc = _library().lqsgd_unpack8(_PACKED8.pack(*p.fields()), rows, cols, yp, yl, DTYPES[dtype], _stream(dev))
    if rc:
        B._check(rc)
    if out is not None:
        _written(out)
    return y


def act_grad(dy: torch.Tensor, z8: Optional[Packed8], act: str = "none", bias_grad: bool = True,
             out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(dz, db): dz = dy act'(z) with z from its 8-bit form, db its column sums in float32 (None without bias_grad).
    `out` may be dy.  With act "none" dz is dy itself, or `out`, to which dy is copied."""
    dev = dy.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return act_grad(dy, z8, act, bias_grad, out)
    yp, yl = _matrix(dy, "dy", dev)
    dt, a = _dtype(dy, "dy"), _act(act)
    rows, cols = dy.shape
    dz, dp, dl, zf = dy, 0, 0, None
    if a:
        zf = _PACKED8.pack(*_kept(z8, "z8", dev, rows, cols))
    if a or (out is not None and out is not dy):
        dz = _empty(rows, cols, dy.dtype, dy.device) if out is None else out
        dp, dl = _matrix(dz, "out", dev, dy.dtype, rows, cols)
    elif not bias_grad:
        return dy, None
    lib, stream = _library(), _stream(dev)
    db, bp = None, 0
    if bias_grad:
        db = torch.empty_strided((cols,), (1,), dtype=torch.float32, device=dy.device)
        bp = db.data_ptr()
    _, wp, size = _kept_scratch(dev, stream)
    rc = lib.lqsgd_act_grad(yp, yl, zf, a, dt, rows, cols, dp, dl, bp, wp, size, stream)
    if rc == B.ERR_WORKSPACE_TOO_SMALL:
        need = C.c_size_t(0)
        B._check(lib.lqsgd_act_grad_workspace_bytes(rows, cols, C.byref(need)))
        ws = _workspace(need.value, dy.device, stream)
        rc = lib.lqsgd_act_grad(yp, yl, zf, a, dt, rows, cols, dp, dl, bp, ws.data_ptr(), ws.numel(), stream)
    if rc:
        B._check(rc)
    if dp and out is not None:
        _written(out)
    return dz, db


# ------------------------------------------------------------------------------------------- rows of signed 8-bit codes

def _pitch(cols: int) -> int:
    return (cols + 127) & -128 if cols >= 1024 else (cols + 15) & -16


class Rows8:
    """A matrix as rows of signed 8-bit codes: codes, int8 rows x cols, and scales, float32 rows (see lqsgd_rows8)."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        self.codes, self.scales = codes, scales
        self.fields()

    @staticmethod
    def empty(rows: int, cols: int, device) -> "Rows8":
        """Uninitialised; rows of codes start on 16-byte boundaries, long ones on those of 128 bytes (4096 x 4097 x 4096: 55 against 72 us)."""
        p = object.__new__(Rows8)
        p.codes = torch.empty_strided((rows, cols), (_pitch(cols), 1), dtype=torch.int8, device=device)
        p.scales = torch.empty_strided((rows,), (1,), dtype=torch.float32, device=device)
        return p

    def _fresh(self) -> Tuple[int, int, int]:
        """fields() of what empty() just made."""
        return self.codes.data_ptr(), _pitch(self.codes.shape[1]), self.scales.data_ptr()

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def fields(self) -> Tuple[int, int, int]:
        """The members of lqsgd_rows8, checked."""
        codes = self.codes
        dev = codes.get_device()
        cp, cl = _matrix(codes, "codes", dev, torch.int8)
        return cp, cl, _vector(self.scales, "scales", dev, codes.shape[0])


def _rows(p: "Rows8", what: str, device: int, rows: int = -1, cols: int = -1) -> Tuple[int, int, int]:
    """The fields of an argument in rows of signed codes (any number of rows or columns where -1)."""
    if not isinstance(p, Rows8):
        raise ValueError(f"{what} must be the Rows8 form of a matrix")
    r, c = p.codes.shape
    if (rows >= 0 and r != rows) or (cols >= 0 and c != cols) or p.codes.get_device() != device:
        raise ValueError(f"{what} must be the Rows8 form of {rows if rows >= 0 else 'any'} x {cols if cols >= 0 else 'any'} values on the call's device, "
                         f"not of {r} x {c}")
    return p.fields()


def pack_rows8(x: torch.Tensor, out: Optional[Rows8] = None) -> Rows8:
    """A matrix (bfloat16, float16 or float32) as rows of signed 8-bit codes with one scale each."""
    dev = x.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return pack_rows8(x, out)
    xp, xl = _matrix(x, "x", dev)
    rows, cols = x.shape
    given = out is not None
    if given:
        of = _rows(out, "out", dev, rows, cols)
    else:
        out = Rows8.empty(rows, cols, x.device)
        of = out._fresh()
    rc = _library().lqsgd_pack_rows8(xp, xl, _dtype(x, "x"), rows, cols, _ROWS8.pack(*of), _stream(dev))
    if rc:
        B._check(rc)
    if given:
        _written(out.codes, out.scales)
    return out


def unpack_rows8(p: Rows8, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values that rows of signed codes stand for, rounded to dtype."""
    codes = p.codes
    dev = codes.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return unpack_rows8(p, dtype, out)
    rows, cols = codes.shape
    if dtype not in DTYPES:
        raise ValueError(f"dtype must be one of {list(DTYPES)}")
    y = _empty(rows, cols, dtype, codes.device) if out is None else out
    yp, yl = _matrix(y, "out", dev, dtype, rows, cols)
    rc = _library().lqsgd_unpack_rows8(_ROWS8.pack(*p.fields()), rows, cols, yp, yl, DTYPES[dtype], _stream(dev))
    if rc:
        B._check(rc)
    if out is not None:
        _written(out)
    return y


# -------------------------------------------------------------------------------------------------------------- dropout

Seed = Union[int, torch.Tensor]


def _drop(p: float, seed: Seed, offset: int, device: int) -> Tuple[float, int, int, int, int]:
    """The members of lqsgd_drop."""
    if not -_MOST <= p <= _MOST:
        _real(p, "p")
    if isinstance(seed, torch.Tensor):
        if seed.dtype != torch.int64 or seed.numel() != 2 or not seed.is_contiguous() or seed.get_device() != device:
            raise ValueError("seed must be a whole number or a contiguous int64 tensor of two on the call's device: the seed and what is added to offset")
        return p, 0, 0, index(offset) & _WORD, seed.data_ptr()
    try:
        return p, 0, seed & _WORD, offset & _WORD, 0
    except OverflowError:                                    # numpy's whole numbers
        return p, 0, index(seed) & _WORD, index(offset) & _WORD, 0


def dropout(x: torch.Tensor, p: float, seed: Seed, offset: int = 0, residual: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout(x): a value is dropped with probability rint(65536 p) / 65536, 0 <= p < 1, what is kept grows by the inverse of the
    rest.  The mask is a function of seed, offset and the value's row and column alone and never stored: dropout(dy, p, seed, offset) is the
    gradient.  Take an offset once per mask.  seed: a whole number, or a CUDA int64 tensor (seed, what is added to offset), read when the
    kernels run, so that the replays of a captured graph need not repeat a mask.  `out` may be x or the residual."""
    dev = x.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return dropout(x, p, seed, offset, residual, out)
    xp, xl = _matrix(x, "x", dev)
    dtype = x.dtype
    rows, cols = x.shape
    rp = rl = 0
    if residual is not None:
        rp, rl = _matrix(residual, "residual", dev, dtype, rows, cols)
    y = _empty(rows, cols, dtype, x.device) if out is None else out
    yp, yl = _matrix(y, "out", dev, dtype, rows, cols)
    rc = _library().lqsgd_dropout(xp, xl, rp, rl, _dtype(x, "x"), rows, cols, _DROP.pack(*_drop(p, seed, offset, dev)), yp, yl, _stream(dev))
    if rc:
        B._check(rc)
    if out is not None:
        _written(out)
    return y


# ----------------------------------------------------------------------------------------------- root-mean-square norm

class RmsNormOut(NamedTuple):
    y: Optional[torch.Tensor]
    h: torch.Tensor
    rstd: torch.Tensor
    h8: Optional[Packed8]
    y8: Optional[Packed8]
    rows8: Optional[Rows8]


def rms_norm(x: torch.Tensor, gamma: torch.Tensor, eps: float = 1e-6, residual: Optional[torch.Tensor] = None, p: float = 0.0, seed: Seed = 0,
             offset: int = 0, want_y: bool = True, save_h8: bool = False, save_y8: bool = False, save_rows8: bool = False) -> RmsNormOut:
    """h = residual + dropout(x, p, seed, offset) and y = gamma h rstd, rstd = 1 / sqrt(mean(h^2) + eps) over each row; x and residual rows x cols,
    bfloat16, float16 or float32, gamma float32.  Without a residual and with p = 0, h is x itself.  save_h8 / save_y8 also return the 8-bit
    forms of h / of y as stored, save_rows8 y (before its rounding) in rows of signed codes; y itself is None without want_y."""
    dev = x.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return rms_norm(x, gamma, eps, residual, p, seed, offset, want_y, save_h8, save_y8, save_rows8)
    dtype, device = x.dtype, x.device
    xp, xl = _matrix(x, "x", dev)
    rows, cols = x.shape
    rp = rl = hp = yp = 0
    if residual is not None:
        rp, rl = _matrix(residual, "residual", dev, dtype, rows, cols)
    h, y = x, None
    if residual is not None or p > 0:
        h = _empty(rows, cols, dtype, device)
        hp = h.data_ptr()
    if want_y:
        y = _empty(rows, cols, dtype, device)
        yp = y.data_ptr()
    rstd = torch.empty_strided((rows,), (1,), dtype=torch.float32, device=device)
    h8 = Packed8.empty(rows, cols, device) if save_h8 else None
    y8 = Packed8.empty(rows, cols, device) if save_y8 else None
    r8 = Rows8.empty(rows, cols, device) if save_rows8 else None
    rc = _library().lqsgd_rms_norm_forward(
        _RMS.pack(_RMS.size, _dtype(x, "x"), rows, cols, eps if -_MOST <= eps <= _MOST else _real(eps, "eps"), *_drop(p, seed, offset, dev), xp, xl, rp, rl, 0, 0, 0, 0, hp, cols, yp, cols, 0, 0, 0, 0,
                  _vector(gamma, "gamma", dev, cols), rstd.data_ptr(), 0, *(h8._fresh() if save_h8 else _NONE8), *(y8._fresh() if save_y8 else _NONE8),
                  *(r8._fresh() if save_rows8 else _NO_ROWS8), 0, 0), _stream(dev))
    if rc:
        B._check(rc)
    return RmsNormOut(y, h, rstd, h8, y8, r8)


def rms_norm_grad(dy: torch.Tensor, h: Union[torch.Tensor, Packed8], gamma: torch.Tensor, rstd: torch.Tensor, skip: Optional[torch.Tensor] = None,
                  p: float = 0.0, seed: Seed = 0, offset: int = 0, gamma_grad: bool = True) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(dx, dresidual, dgamma) of rms_norm: h as the forward call returned it, or its 8-bit form, rstd as it returned it, skip the gradient that
    arrives at h from elsewhere, p, seed and offset the forward call's.  With p = 0 dx and dresidual are one tensor.  dgamma is None without
    gamma_grad."""
    dev = dy.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return rms_norm_grad(dy, h, gamma, rstd, skip, p, seed, offset, gamma_grad)
    dtype, device = dy.dtype, dy.device
    yp, yl = _matrix(dy, "dy", dev)
    rows, cols = dy.shape
    hp, hl, hf, sp, sl = 0, 0, _NONE8, 0, 0
    if isinstance(h, Packed8):
        hf = _kept(h, "h", dev, rows, cols)
    else:
        hp, hl = _matrix(h, "h", dev, dtype, rows, cols)
    if skip is not None:
        sp, sl = _matrix(skip, "skip", dev, dtype, rows, cols)
    dx = _empty(rows, cols, dtype, device)
    dres, dp = dx, 0
    if p > 0:
        dres = _empty(rows, cols, dtype, device)
        dp = dres.data_ptr()
    dgamma, gp = None, 0
    if gamma_grad:
        dgamma = torch.empty_strided((cols,), (1,), dtype=torch.float32, device=device)
        gp = dgamma.data_ptr()
    lib = _library()
    _call(lib.lqsgd_rms_norm_backward,
          (_RMS.size, _dtype(dy, "dy"), rows, cols, 0.0, *_drop(p, seed, offset, dev), 0, 0, 0, 0, yp, yl, sp, sl, hp, hl, 0, 0, dx.data_ptr(), cols, dp, cols,
           _vector(gamma, "gamma", dev, cols), _vector(rstd, "rstd", dev, rows), gp, *hf, *_NONE8, *_NO_ROWS8),
          _RMS, lib.lqsgd_rms_norm_workspace_bytes, 1, device)
    return dx, dres, dgamma


# -------------------------------------------------------------------------------------------------------- linear layers

class LinearOut(NamedTuple):
    y: torch.Tensor
    z8: Optional[Packed8]
    y8: Optional[Packed8]


def linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
           residual: Optional[torch.Tensor] = None, save_z8: bool = False, save_y8: bool = False,
           out: Optional[torch.Tensor] = None) -> LinearOut:
    """y = act(x w^T + bias) + residual, x rows x in and w out x in, bfloat16 or float16; bias float32.
    save_z8 / save_y8 also return the 8-bit form of the pre-activation x w^T + bias / of y.  `out` may be the residual."""
    dev = x.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return linear(x, w, bias, act, residual, save_z8, save_y8, out)
    dtype, device = x.dtype, x.device
    xp, xl = _matrix(x, "x", dev)
    rows, cin = x.shape
    wp, wl = _matrix(w, "w", dev, dtype, -1, cin)
    cout = w.shape[0]
    rp = rl = 0
    if residual is not None:
        rp, rl = _matrix(residual, "residual", dev, dtype, rows, cout)
    y = _empty(rows, cout, dtype, device) if out is None else out
    yp, yl = _matrix(y, "out", dev, dtype, rows, cout)
    z8 = Packed8.empty(rows, cout, device) if save_z8 else None
    y8 = Packed8.empty(rows, cout, device) if save_y8 else None
    lib = _library()
    _call(lib.lqsgd_linear_forward,
          (_LINEAR.size, _dtype(x, "x", True), _act(act), 0, rows, cin, cout, xp, xl, wp, wl, 0, 0,
           0 if bias is None else _vector(bias, "bias", dev, cout), rp, rl, yp, yl, *_NONE8,
           *(z8._fresh() if save_z8 else _NONE8), *(y8._fresh() if save_y8 else _NONE8), _status_word(device)),
          _LINEAR, lib.lqsgd_linear_workspace_bytes, FORWARD, device)
    if out is not None:
        _written(out)
    return LinearOut(y, z8, y8)


def linear_grad_input(dz: torch.Tensor, w: torch.Tensor, residual: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx = dz w + residual (the gradient that came down the skip connection).  `out` may be the residual."""
    dev = dz.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return linear_grad_input(dz, w, residual, out)
    dtype, device = dz.dtype, dz.device
    zp, zl = _matrix(dz, "dz", dev)
    rows, cout = dz.shape
    wp, wl = _matrix(w, "w", dev, dtype, cout)
    cin = w.shape[1]
    rp = rl = 0
    if residual is not None:
        rp, rl = _matrix(residual, "residual", dev, dtype, rows, cin)
    dx = _empty(rows, cin, dtype, device) if out is None else out
    op, ol = _matrix(dx, "out", dev, dtype, rows, cin)
    lib = _library()
    _call(lib.lqsgd_linear_grad_input,
          (_LINEAR.size, _dtype(dz, "dz", True), 0, 0, rows, cin, cout, 0, 0, wp, wl, zp, zl, 0, rp, rl, op, ol, *_NONE8, *_NONE8, *_NONE8,
           _status_word(device)),
          _LINEAR, lib.lqsgd_linear_workspace_bytes, GRAD_INPUT, device)
    if out is not None:
        _written(out)
    return dx


def linear_grad_weight(dz: torch.Tensor, x: Union[torch.Tensor, Packed8], out: Optional[torch.Tensor] = None,
                       accumulate: bool = False) -> torch.Tensor:
    """dw = dz^T x in float32, out x in: the gradient a round takes.  x is a matrix of dz's type or its 8-bit form (which is
    decoded into a workspace of rows x in 16-bit values for the call).  accumulate adds to `out` (a gradient over several
    micro-batches)."""
    dev = dz.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return linear_grad_weight(dz, x, out, accumulate)
    device = dz.device
    zp, zl = _matrix(dz, "dz", dev)
    rows, cout = dz.shape
    xp, xl, xf = 0, 0, _NONE8
    if isinstance(x, Packed8):
        xf = _kept(x, "x", dev, rows)
    else:
        xp, xl = _matrix(x, "x", dev, dz.dtype, rows)
    cin = x.shape[1]
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    dw = _empty(cout, cin, torch.float32, device) if out is None else out
    op, ol = _matrix(dw, "out", dev, torch.float32, cout, cin)
    lib = _library()
    _call(lib.lqsgd_linear_grad_weight,
          (_LINEAR.size, _dtype(dz, "dz", True), 0, int(accumulate), rows, cin, cout, xp, xl, 0, 0, zp, zl, 0, 0, 0, op, ol,
           *xf, *_NONE8, *_NONE8, _status_word(device)),
          _LINEAR, lib.lqsgd_linear_workspace_bytes, GRAD_WEIGHT, device)
    if out is not None:
        _written(out)
    return dw


def _rows8_bytes(_, args: bytes, need) -> int:
    return _library().lqsgd_linear_rows8_workspace_bytes(args, need)


def linear_rows8(x: Rows8, w: Rows8, bias: Optional[torch.Tensor] = None, act: str = "none", residual: Optional[torch.Tensor] = None,
                 dtype: torch.dtype = torch.bfloat16, save_z8: bool = False, save_y8: bool = False, out: Optional[torch.Tensor] = None) -> LinearOut:
    """y = act(x w^T + bias) + residual in 8-bit integers: x rows x in with a scale per row, w out x in with a scale per output channel, the
    sums exact in 32 bits (in <= 131071).  residual and y have `dtype`, bfloat16 or float16 (that of residual or out where one is given); bias
    float32.  save_z8 / save_y8 as of linear.  `out` may be the residual."""
    if not isinstance(x, Rows8):
        raise ValueError("x must be the Rows8 form of a matrix")
    dev = x.codes.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return linear_rows8(x, w, bias, act, residual, dtype, save_z8, save_y8, out)
    device = x.codes.device
    if residual is not None or out is not None:
        dtype = (residual if residual is not None else out).dtype
    code = DTYPES.get(dtype)
    if code is None or code == 2:
        raise ValueError(f"dtype must be bfloat16 or float16, not {dtype}")
    xf = _rows(x, "x", dev)
    rows, cin = x.codes.shape
    wf = _rows(w, "w", dev, -1, cin)
    cout = w.codes.shape[0]
    rp = rl = 0
    if residual is not None:
        rp, rl = _matrix(residual, "residual", dev, dtype, rows, cout)
    y = _empty(rows, cout, dtype, device) if out is None else out
    yp, yl = _matrix(y, "out", dev, dtype, rows, cout)
    z8 = Packed8.empty(rows, cout, device) if save_z8 else None
    y8 = Packed8.empty(rows, cout, device) if save_y8 else None
    _call(_library().lqsgd_linear_rows8_forward,
          (_LINEAR8.size, code, _act(act), 0, rows, cin, cout, *xf, *wf, 0 if bias is None else _vector(bias, "bias", dev, cout), rp, rl, yp, yl,
           *(z8._fresh() if save_z8 else _NONE8), *(y8._fresh() if save_y8 else _NONE8), _status_word(device)),
          _LINEAR8, _rows8_bytes, 0, device)
    if out is not None:
        _written(out)
    return LinearOut(y, z8, y8)


# ------------------------------------------------------------------------------------------------------------ group norm

class GroupNormOut(NamedTuple):
    y: torch.Tensor
    mean: torch.Tensor
    rstd: torch.Tensor
    x8: Optional[Packed8]
    y8: Optional[Packed8]


def _pixels(t: torch.Tensor, what: str) -> Tuple[int, int, int, int, int]:
    """(n, hw, c, elements between pixels, between samples) of a channels-last tensor n x ... x c."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    dims, strides = t.shape, t.stride()
    if len(dims) < 2 or (strides[-1] != 1 and dims[-1] > 1):
        raise ValueError(f"{what} must be samples x ... x channels, channels with unit stride")
    n, c = dims[0], dims[-1]
    hw, ld = 1, None
    for d in range(len(dims) - 2, 0, -1):                   # the pixel dimensions must fold into one with a fixed distance
        if dims[d] == 1:
            continue
        if ld is None:
            ld = strides[d]
        elif strides[d] != ld * hw:
            raise ValueError(f"{what}'s pixel dimensions must be contiguous with one another")
        hw *= dims[d]
    if ld is None:
        ld = c
    return n, hw, c, ld, (strides[0] if n > 1 else hw * ld)


def group_norm(x: torch.Tensor, groups: int, gamma: torch.Tensor, beta: torch.Tensor, eps: float = 1e-5, act: str = "none",
               save_x8: bool = False, save_y8: bool = False) -> GroupNormOut:
    """y = act(gamma (x - mean) rstd + beta) over `groups` groups of channels of each sample; x is samples x ... x channels,
    bfloat16, float16 or float32, gamma and beta float32.  save_x8 / save_y8 also return 8-bit forms (rows = pixels)."""
    dev = x.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return group_norm(x, groups, gamma, beta, eps, act, save_x8, save_y8)
    n, hw, c, ld, sample = _pixels(x, "x")
    device = x.device
    y = torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=device)
    mean = _empty(n, max(1, groups), torch.float32, device)
    rstd = _empty(n, max(1, groups), torch.float32, device)
    x8 = Packed8.empty(n * hw, c, device) if save_x8 else None
    y8 = Packed8.empty(n * hw, c, device) if save_y8 else None
    lib = _library()
    _call(lib.lqsgd_group_norm_forward,
          (_NORM.size, _dtype(x, "x"), _act(act), groups, n, hw, c, _real(eps, "eps"), x.data_ptr(), ld, sample, 0, 0, 0, y.data_ptr(), c, hw * c,
           _vector(gamma, "gamma", dev, c), _vector(beta, "beta", dev, c), mean.data_ptr(), rstd.data_ptr(), 0, 0,
           *(x8._fresh() if save_x8 else _NONE8), *(y8._fresh() if save_y8 else _NONE8)),
          _NORM, lib.lqsgd_group_norm_workspace_bytes, 0, device)
    return GroupNormOut(y, mean, rstd, x8, y8)


def group_norm_grad(dy: torch.Tensor, x: Union[torch.Tensor, Packed8], groups: int, gamma: torch.Tensor, beta: torch.Tensor,
                    mean: torch.Tensor, rstd: torch.Tensor, act: str = "none") -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dgamma, dbeta) of group_norm; x as the forward call had it, or its 8-bit form; mean and rstd as it returned them."""
    dev = dy.get_device()
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return group_norm_grad(dy, x, groups, gamma, beta, mean, rstd, act)
    n, hw, c, ld, sample = _pixels(dy, "dy")
    device = dy.device
    xp, xl, xs, xf = 0, 0, 0, _NONE8
    if isinstance(x, Packed8):
        xf = _kept(x, "x", dev, n * hw, c)
    else:
        if x.dtype != dy.dtype or x.shape != dy.shape or x.get_device() != dev:
            raise ValueError("x must have dy's type, shape and device")
        _, _, _, xl, xs = _pixels(x, "x")
        xp = x.data_ptr()
    dx = torch.empty_like(dy) if dy.is_contiguous() else torch.empty(dy.shape, dtype=dy.dtype, device=device)
    dgamma = torch.empty_strided((c,), (1,), dtype=torch.float32, device=device)
    dbeta = torch.empty_strided((c,), (1,), dtype=torch.float32, device=device)
    lib = _library()
    _call(lib.lqsgd_group_norm_backward,
          (_NORM.size, _dtype(dy, "dy"), _act(act), groups, n, hw, c, 1.0, xp, xl, xs, dy.data_ptr(), ld, sample, dx.data_ptr(), c, hw * c,
           _vector(gamma, "gamma", dev, c), _vector(beta, "beta", dev, c), _vector(mean, "mean", dev, n * groups),
           _vector(rstd, "rstd", dev, n * groups), dgamma.data_ptr(), dbeta.data_ptr(), *xf, *_NONE8),
          _NORM, lib.lqsgd_group_norm_workspace_bytes, 1, device)
    return dx, dgamma, dbeta


# ------------------------------------------------------------------------------------- differentiable layers, 8 bits in between
# Differentiable once: the kernels of a backward pass leave nothing for autograd to follow, so a second derivative raises.

def _apart(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy of it where its rows overlap (an expanded tensor, the gradient of a sum) or do not lie along memory."""
    row = t.shape[-1]
    return t if t.stride(-1) == 1 and all(s >= row or n == 1 for n, s in zip(t.shape[:-1], t.stride()[:-1])) else t.contiguous()


class _LinearLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act, x8, recording):
        x, w = _apart(x), _apart(weight.to(x.dtype))
        residual = residual if residual is None else _apart(residual)
        for_x, for_w, for_bias = (n and recording for n in ctx.needs_input_grad[:3])
        r = linear(x, w, bias, act, residual, save_z8=act != "none" and (for_x or for_w or for_bias))
        if for_w and x8 is None:
            x8 = pack8(x)
        kept = (x8 if for_w else None), r.z8
        ctx.save_for_backward(w if for_x else None, *(t for p in kept for t in ((p.codes, p.exps) if p is not None else (None, None))))
        ctx.act = act
        return r.y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        w, xc, xe, zc, ze = ctx.saved_tensors
        for_x, for_w, for_bias, for_residual = ctx.needs_input_grad[:4]
        dy = _apart(dy)
        dx = dw = db = None
        if for_x or for_w or for_bias:
            dz, db = act_grad(dy, None if zc is None else Packed8(zc, ze), ctx.act, bias_grad=for_bias)
            dx = linear_grad_input(dz, w) if for_x else None
            dw = linear_grad_weight(dz, Packed8(xc, xe)) if for_w else None
        return dx, dw, db, (dy if for_residual else None), None, None, None


def linear_layer(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
                 residual: Optional[torch.Tensor] = None, x8: Optional[Packed8] = None) -> torch.Tensor:
    """linear() as a differentiable function: weight and bias float32 (the weights a round updates; the products run in x's
    type), x and the pre-activation kept in 8 bits, the weight gradient float32.  x8: x's 8-bit form where it exists
    already (norm_layer and other producers can hand it on).  Kept is what the wanted gradients need: nothing under no_grad, no x
    where the weight is frozen.  Differentiable once: a second derivative raises.  Should a bounded wait on the device run out,
    output and gradients are undefined and status() says so: a training loop asks it where it reads its loss."""
    return _LinearLayer.apply(x, weight, bias, residual, act, x8, torch.is_grad_enabled())


class _NormLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, groups, eps, act, keep, recording):
        wanted = recording and any(ctx.needs_input_grad[:3])
        r = group_norm(_apart(x), groups, gamma, beta, eps, act, save_x8=wanted, save_y8=keep is not None)
        if wanted:
            ctx.save_for_backward(r.x8.codes, r.x8.exps, gamma, beta, r.mean, r.rstd)
        ctx.groups, ctx.act = groups, act
        if keep is not None:
            keep.append(r.y8)
        return r.y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        codes, exps, gamma, beta, mean, rstd = ctx.saved_tensors
        dx, dgamma, dbeta = group_norm_grad(dy.contiguous(), Packed8(codes, exps), ctx.groups, gamma, beta, mean, rstd, ctx.act)
        return dx, dgamma, dbeta, None, None, None, None, None


def norm_layer(x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, groups: int, eps: float = 1e-5, act: str = "none",
               keep: Optional[list] = None) -> torch.Tensor:
    """group_norm() as a differentiable function with x kept in 8 bits.  `keep`, a list, receives the output's 8-bit form
    (for the linear layer that follows).  Differentiable once: a second derivative raises."""
    return _NormLayer.apply(x, gamma, beta, groups, eps, act, keep, torch.is_grad_enabled())


def _kept_seed(ctx, p: float, seed: Seed, offset: int, *tensors) -> None:
    """Keeps a dropout's arguments for the backward pass, a seed on the device among the saved tensors (writing it in between raises)."""
    on_device = isinstance(seed, torch.Tensor)
    ctx.save_for_backward(*tensors, seed if on_device else None)
    ctx.drop = p, None if on_device else seed, offset


def _drop_again(ctx, saved: Optional[torch.Tensor]) -> Tuple[float, Seed, int]:
    p, seed, offset = ctx.drop
    return p, saved if seed is None else seed, offset


class _DropoutLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, offset):
        _kept_seed(ctx, p, seed, offset)
        return dropout(_apart(x), p, seed, offset, residual if residual is None else _apart(residual))

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        p, seed, offset = _drop_again(ctx, *ctx.saved_tensors)
        dx = dropout(_apart(dy), p, seed, offset) if ctx.needs_input_grad[0] else None
        return dx, (dy if ctx.needs_input_grad[1] else None), None, None, None


def dropout_layer(x: torch.Tensor, p: float, seed: Seed, offset: int = 0, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dropout() as a differentiable function that keeps nothing but its arguments.  Differentiable once: a second derivative raises."""
    return _DropoutLayer.apply(x, residual, p, seed, offset)


class _RmsLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, gamma, eps, p, seed, offset, keep, keep_rows8, recording):
        wanted = recording and any(ctx.needs_input_grad[:3])
        r = rms_norm(_apart(x), gamma, eps, residual if residual is None else _apart(residual), p, seed, offset, save_h8=wanted, save_y8=keep is not None,
                     save_rows8=keep_rows8 is not None)
        ctx.set_materialize_grads(False)
        if wanted:
            _kept_seed(ctx, p, seed, offset, r.h8.codes, r.h8.exps, gamma, r.rstd)
        if keep is not None:
            keep.append(r.y8)
        if keep_rows8 is not None:
            keep_rows8.append(r.rows8)
        return r.y if residual is None else (r.y, r.h)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh=None):
        codes, exps, gamma, rstd, seed = ctx.saved_tensors
        for_x, for_residual, for_gamma = ctx.needs_input_grad[:3]
        drop = _drop_again(ctx, seed)
        dh = None if dh is None else _apart(dh)
        if dy is not None:
            dx, dresidual, dgamma = rms_norm_grad(_apart(dy), Packed8(codes, exps), gamma, rstd, dh, *drop, gamma_grad=for_gamma)
        elif dh is not None:                            # y was not used: only the sum's gradient arrives
            dx, dresidual, dgamma = dropout(dh, *drop) if drop[0] > 0 else dh, dh, None
        else:
            dx = dresidual = dgamma = None
        return (dx if for_x else None), (dresidual if for_residual else None), dgamma, None, None, None, None, None, None, None


def rms_norm_layer(x: torch.Tensor, gamma: torch.Tensor, eps: float = 1e-6, keep: Optional[list] = None, keep_rows8: Optional[list] = None) -> torch.Tensor:
    """rms_norm() of a matrix as a differentiable function with x kept in 8 bits.  `keep` and `keep_rows8`, lists, receive the output's 8-bit
    forms: of kept activations (linear_layer's x8) and of rows of signed codes (linear_rows8_layer's rows8).  Differentiable once."""
    return _RmsLayer.apply(x, None, gamma, eps, 0.0, 0, 0, keep, keep_rows8, torch.is_grad_enabled())


def add_rms_norm_layer(x: torch.Tensor, residual: torch.Tensor, gamma: torch.Tensor, eps: float = 1e-6, p: float = 0.0, seed: Seed = 0, offset: int = 0,
                       keep: Optional[list] = None, keep_rows8: Optional[list] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(y, h) of rms_norm() with a residual, h = residual + dropout(x), as a differentiable function that keeps h in 8 bits and no mask;
    `keep` and `keep_rows8` as of rms_norm_layer.  Differentiable once."""
    return _RmsLayer.apply(x, residual, gamma, eps, p, seed, offset, keep, keep_rows8, torch.is_grad_enabled())


class _LinearRows8Layer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act, rows8, weight8, recording):
        _dtype(x, "x", True)
        if residual is not None and residual.dtype != x.dtype:
            raise ValueError(f"residual must have x's type {x.dtype}, not {residual.dtype}")
        for p, t, what in ((rows8, x, "rows8"), (weight8, weight, "weight8")):
            if p is not None and p.shape != t.shape:
                raise ValueError(f"{what} must be the Rows8 form of {tuple(t.shape)} values, not of {tuple(p.shape)}")
        for_x, for_w, for_bias = (n and recording for n in ctx.needs_input_grad[:3])
        x8 = pack_rows8(_apart(x)) if rows8 is None else rows8
        w8 = pack_rows8(_apart(weight.detach())) if weight8 is None else weight8
        r = linear_rows8(x8, w8, bias, act, residual if residual is None else _apart(residual), x.dtype, save_z8=act != "none" and (for_x or for_w or for_bias))
        z8 = (None, None) if r.z8 is None else (r.z8.codes, r.z8.exps)
        ctx.save_for_backward(weight if for_x else None, *((x8.codes, x8.scales) if for_w else (None, None)), *z8)
        ctx.act, ctx.dtype = act, x.dtype
        return r.y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        weight, xc, xs, zc, ze = ctx.saved_tensors
        for_x, for_w, for_bias, for_residual = ctx.needs_input_grad[:4]
        dy = _apart(dy)
        dx = dw = db = None
        if for_x or for_w or for_bias:
            dz, db = act_grad(dy, None if zc is None else Packed8(zc, ze), ctx.act, bias_grad=for_bias)
            dx = linear_grad_input(dz, _apart(weight.to(ctx.dtype))) if for_x else None
            dw = linear_grad_weight(dz, unpack_rows8(Rows8(xc, xs), ctx.dtype)) if for_w else None
        return dx, dw, db, (dy if for_residual else None), None, None, None, None


def linear_rows8_layer(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none", residual: Optional[torch.Tensor] = None,
                       rows8: Optional[Rows8] = None, weight8: Optional[Rows8] = None) -> torch.Tensor:
    """linear_rows8() as a differentiable function: x bfloat16 or float16, weight and bias float32; both operands of the forward product become
    rows of signed codes, unless the caller has them (rows8 from the norm in front, weight8 = pack_rows8(weight) kept over micro-batches;
    x's values are then not read).  The gradients pass the rounding to 8 bits straight through: dx = dz w with the weight in x's type, dw = dz^T x in
    float32 with x as it was multiplied, and x is kept in those 8 bits.  Differentiable once."""
    return _LinearRows8Layer.apply(x, weight, bias, residual, act, rows8, weight8, torch.is_grad_enabled())
