"""Training operators of liblqsgd.so: the layers whose weight gradients a round compresses.

    linear / linear_grad_input / linear_grad_weight    a linear layer's three products, bias, activation and residual in the
                                                       epilogue
    pack8 / unpack8 / act_grad                         activations kept in 8 bits until the backward pass
    group_norm / group_norm_grad                       group norm with an activation, channels last

Argument marshalling only, as in binding.py: tensors are checked here for type, device and layout, everything else by the
library; the arithmetic runs in its CUDA kernels, on the current stream of the tensors' device.  `linear_layer` and
`norm_layer` are the same operators as differentiable functions that keep only 8-bit activations between the passes.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import NamedTuple, Optional, Tuple, Union

import torch

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
        for f in (lib.lqsgd_linear_forward, lib.lqsgd_linear_grad_input, lib.lqsgd_linear_grad_weight,
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


def _matrix(t: torch.Tensor, what: str, device: int, dtype: Optional[torch.dtype] = None, shape=None) -> torch.Tensor:
    """Checks a matrix argument; device is the index all tensors of the call must be on."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what} must be a matrix with unit stride along its rows")
    if t.get_device() != device:
        raise ValueError(f"{what} must be on the device of the call's other tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, not {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    return t


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _vector(t: torch.Tensor, what: str, device: int, n: int) -> int:
    """Address of a checked float32 vector."""
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what} must be a contiguous float32 vector of {n} on the call's device")
    return t.data_ptr()


class _On:
    """Makes a device current for a call (nothing to do when it already is) and gives its current stream's handle."""
    __slots__ = ("guard", "index")

    def __init__(self, index: int):
        self.index = index
        self.guard = None if torch.cuda.current_device() == index else torch.cuda.device(index)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch._C._cuda_getCurrentRawStream(self.index)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _call(fn, args: tuple, layout: struct.Struct, bytes_fn, which: int, device: torch.device, stream) -> None:
    """Runs fn on a packed argument struct whose last two fields are the workspace.  Calls that need none are done at once;
    the others are refused on the host, before anything is launched, and get one from PyTorch's allocator (on the current
    stream, so its memory is not handed out again before the call's kernels are done)."""
    rc = fn(layout.pack(*args, 0, 0), stream)
    if rc == B.ERR_WORKSPACE_TOO_SMALL:
        need = C.c_size_t(0)
        B._check(bytes_fn(which, layout.pack(*args, 0, 0), C.byref(need)))
        ws = torch.empty(need.value, dtype=torch.uint8, device=device)
        rc = fn(layout.pack(*args, ws.data_ptr(), need.value), stream)
    if rc != 0:
        B._check(rc)


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
    """Status bits (binding.STATUS_TIMEOUT) that the linear layers' kernels have raised on a device so far; synchronises."""
    word = _status.get(torch.device(device).index or 0)
    return 0 if word is None else int(word.item())


# ------------------------------------------------------------------------------------------------ activations in 8 bits

class Packed8:
    """A matrix kept in 8 bits: codes, uint8 rows x cols, and exps, uint8 rows x ceil(cols / 32) (see lqsgd_packed8)."""

    __slots__ = ("codes", "exps")

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor):
        dev = codes.get_device()
        _matrix(codes, "codes", dev, torch.uint8)
        _matrix(exps, "exps", dev, torch.uint8, (codes.shape[0], (codes.shape[1] + GROUP - 1) // GROUP))
        self.codes, self.exps = codes, exps

    @staticmethod
    def empty(rows: int, cols: int, device) -> "Packed8":
        """Uninitialised; rows of codes start on 16-byte boundaries."""
        p = object.__new__(Packed8)
        ld = (cols + 15) & -16
        codes = torch.empty((rows, ld), dtype=torch.uint8, device=device)
        p.codes = codes if ld == cols else codes[:, :cols]
        p.exps = torch.empty((rows, (cols + GROUP - 1) // GROUP), dtype=torch.uint8, device=device)
        return p

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def fields(self) -> tuple:
        return self.codes.data_ptr(), _ld(self.codes), self.exps.data_ptr(), _ld(self.exps)


def pack8(x: torch.Tensor, out: Optional[Packed8] = None) -> Packed8:
    """The 8-bit form of a matrix (bfloat16, float16 or float32)."""
    dev = x.get_device()
    _matrix(x, "x", dev)
    dt = _dtype(x, "x")
    rows, cols = x.shape
    with _On(dev) as stream:
        if out is None:
            out = Packed8.empty(rows, cols, x.device)
        else:
            _matrix(out.codes, "out", dev, torch.uint8, (rows, cols))
        rc = _library().lqsgd_pack8(x.data_ptr(), _ld(x), dt, rows, cols, _PACKED8.pack(*out.fields()), stream)
    if rc:
        B._check(rc)
    return out


def unpack8(p: Packed8, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values an 8-bit form stands for: exact in bfloat16 and float32 (float16: within its range)."""
    rows, cols = p.codes.shape
    dev = p.codes.get_device()
    if dtype not in DTYPES:
        raise ValueError(f"dtype must be one of {list(DTYPES)}")
    with _On(dev) as stream:
        if out is None:
            out = torch.empty((rows, cols), dtype=dtype, device=p.codes.device)
        else:
            _matrix(out, "out", dev, dtype, (rows, cols))
        rc = _library().lqsgd_unpack8(_PACKED8.pack(*p.fields()), rows, cols, out.data_ptr(), _ld(out), DTYPES[dtype], stream)
    if rc:
        B._check(rc)
    return out


def act_grad(dy: torch.Tensor, z8: Optional[Packed8], act: str = "none", bias_grad: bool = True,
             out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(dz, db): dz = dy act'(z) with z from its 8-bit form, db its column sums in float32 (None without bias_grad).
    With act "none" dz is dy itself.  `out` may be dy."""
    dev = dy.get_device()
    _matrix(dy, "dy", dev)
    dt, a = _dtype(dy, "dy"), _act(act)
    rows, cols = dy.shape
    if a == 0:
        if not bias_grad:
            return dy, None
    elif z8 is None:
        raise ValueError("z8 must be the 8-bit form of the pre-activation")
    else:
        _matrix(z8.codes, "z8", dev, torch.uint8, (rows, cols))
    lib = _library()
    with _On(dev) as stream:
        dz, dz_ptr, ld_dz, zf = dy, 0, 0, None
        if a:
            dz = torch.empty((rows, cols), dtype=dy.dtype, device=dy.device) if out is None else _matrix(out, "out", dev, dy.dtype, (rows, cols))
            dz_ptr, ld_dz, zf = dz.data_ptr(), _ld(dz), _PACKED8.pack(*z8.fields())
        db, db_ptr = None, 0
        if bias_grad:
            db = torch.empty(cols, dtype=torch.float32, device=dy.device)
            db_ptr = db.data_ptr()
        rc = lib.lqsgd_act_grad(dy.data_ptr(), _ld(dy), zf, a, dt, rows, cols, dz_ptr, ld_dz, db_ptr, 0, 0, stream)
        if rc == B.ERR_WORKSPACE_TOO_SMALL:
            need = C.c_size_t(0)
            B._check(lib.lqsgd_act_grad_workspace_bytes(rows, cols, C.byref(need)))
            ws = torch.empty(need.value, dtype=torch.uint8, device=dy.device)
            rc = lib.lqsgd_act_grad(dy.data_ptr(), _ld(dy), zf, a, dt, rows, cols, dz_ptr, ld_dz, db_ptr, ws.data_ptr(), need.value, stream)
    if rc:
        B._check(rc)
    return dz, db


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
    _matrix(x, "x", dev)
    dt, code = _dtype(x, "x", True), _act(act)
    _matrix(w, "w", dev, x.dtype)
    rows, cin = x.shape
    cout = w.shape[0]
    if w.shape[1] != cin:
        raise ValueError(f"w must have {cin} columns, not {w.shape[1]}")
    bias_ptr = 0 if bias is None else _vector(bias, "bias", dev, cout)
    res_ptr = ld_res = 0
    if residual is not None:
        _matrix(residual, "residual", dev, x.dtype, (rows, cout))
        res_ptr, ld_res = residual.data_ptr(), _ld(residual)
    lib = _library()
    with _On(dev) as stream:
        y = torch.empty((rows, cout), dtype=x.dtype, device=x.device) if out is None else _matrix(out, "out", dev, x.dtype, (rows, cout))
        z8 = Packed8.empty(rows, cout, x.device) if save_z8 else None
        y8 = Packed8.empty(rows, cout, x.device) if save_y8 else None
        args = (_LINEAR.size, dt, code, 0, rows, cin, cout, x.data_ptr(), _ld(x), w.data_ptr(), _ld(w), 0, 0, bias_ptr, res_ptr, ld_res,
                y.data_ptr(), _ld(y), *_NONE8, *(z8.fields() if save_z8 else _NONE8), *(y8.fields() if save_y8 else _NONE8),
                _status_word(x.device))
        _call(lib.lqsgd_linear_forward, args, _LINEAR, lib.lqsgd_linear_workspace_bytes, FORWARD, x.device, stream)
    return LinearOut(y, z8, y8)


def linear_grad_input(dz: torch.Tensor, w: torch.Tensor, residual: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx = dz w + residual (the gradient that came down the skip connection).  `out` may be the residual."""
    dev = dz.get_device()
    _matrix(dz, "dz", dev)
    dt = _dtype(dz, "dz", True)
    _matrix(w, "w", dev, dz.dtype)
    rows, cout = dz.shape
    cin = w.shape[1]
    if w.shape[0] != cout:
        raise ValueError(f"w must have {cout} rows, not {w.shape[0]}")
    res_ptr = ld_res = 0
    if residual is not None:
        _matrix(residual, "residual", dev, dz.dtype, (rows, cin))
        res_ptr, ld_res = residual.data_ptr(), _ld(residual)
    lib = _library()
    with _On(dev) as stream:
        dx = torch.empty((rows, cin), dtype=dz.dtype, device=dz.device) if out is None else _matrix(out, "out", dev, dz.dtype, (rows, cin))
        args = (_LINEAR.size, dt, 0, 0, rows, cin, cout, 0, 0, w.data_ptr(), _ld(w), dz.data_ptr(), _ld(dz), 0, res_ptr, ld_res,
                dx.data_ptr(), _ld(dx), *_NONE8, *_NONE8, *_NONE8, _status_word(dz.device))
        _call(lib.lqsgd_linear_grad_input, args, _LINEAR, lib.lqsgd_linear_workspace_bytes, GRAD_INPUT, dz.device, stream)
    return dx


def linear_grad_weight(dz: torch.Tensor, x: Union[torch.Tensor, Packed8], out: Optional[torch.Tensor] = None,
                       accumulate: bool = False) -> torch.Tensor:
    """dw = dz^T x in float32, out x in: the gradient a round takes.  x is a matrix of dz's type or its 8-bit form.
    accumulate adds to `out` (a gradient over several micro-batches)."""
    dev = dz.get_device()
    _matrix(dz, "dz", dev)
    dt = _dtype(dz, "dz", True)
    rows, cout = dz.shape
    packed = isinstance(x, Packed8)
    if packed:
        _matrix(x.codes, "x", dev, torch.uint8)
        x_ptr, ld_x, xf = 0, 0, x.fields()
    else:
        _matrix(x, "x", dev, dz.dtype)
        x_ptr, ld_x, xf = x.data_ptr(), _ld(x), _NONE8
    if x.shape[0] != rows:
        raise ValueError(f"x must have {rows} rows, not {x.shape[0]}")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    cin = x.shape[1]
    lib = _library()
    with _On(dev) as stream:
        dw = torch.empty((cout, cin), dtype=torch.float32, device=dz.device) if out is None else _matrix(out, "out", dev, torch.float32, (cout, cin))
        args = (_LINEAR.size, dt, 0, int(accumulate), rows, cin, cout, x_ptr, ld_x, 0, 0, dz.data_ptr(), _ld(dz), 0, 0, 0,
                dw.data_ptr(), _ld(dw), *xf, *_NONE8, *_NONE8, _status_word(dz.device))
        _call(lib.lqsgd_linear_grad_weight, args, _LINEAR, lib.lqsgd_linear_workspace_bytes, GRAD_WEIGHT, dz.device, stream)
    return dw


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
    n, hw, c, ld, sample = _pixels(x, "x")
    dt, code, dev = _dtype(x, "x"), _act(act), x.get_device()
    gamma_ptr, beta_ptr = _vector(gamma, "gamma", dev, c), _vector(beta, "beta", dev, c)
    lib = _library()
    with _On(dev) as stream:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        stats = torch.empty((2, n, max(1, groups)), dtype=torch.float32, device=x.device)
        mean, rstd = stats.unbind(0)
        x8 = Packed8.empty(n * hw, c, x.device) if save_x8 else None
        y8 = Packed8.empty(n * hw, c, x.device) if save_y8 else None
        args = (_NORM.size, dt, code, groups, n, hw, c, eps, x.data_ptr(), ld, sample, 0, 0, 0, y.data_ptr(), c, hw * c,
                gamma_ptr, beta_ptr, mean.data_ptr(), rstd.data_ptr(), 0, 0,
                *(x8.fields() if save_x8 else _NONE8), *(y8.fields() if save_y8 else _NONE8))
        _call(lib.lqsgd_group_norm_forward, args, _NORM, lib.lqsgd_group_norm_workspace_bytes, 0, x.device, stream)
    return GroupNormOut(y, mean, rstd, x8, y8)


def group_norm_grad(dy: torch.Tensor, x: Union[torch.Tensor, Packed8], groups: int, gamma: torch.Tensor, beta: torch.Tensor,
                    mean: torch.Tensor, rstd: torch.Tensor, act: str = "none") -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dgamma, dbeta) of group_norm; x as the forward call had it, or its 8-bit form; mean and rstd as it returned them."""
    n, hw, c, ld, sample = _pixels(dy, "dy")
    dt, code, dev = _dtype(dy, "dy"), _act(act), dy.get_device()
    vectors = (_vector(gamma, "gamma", dev, c), _vector(beta, "beta", dev, c), _vector(mean, "mean", dev, n * groups),
               _vector(rstd, "rstd", dev, n * groups))
    if isinstance(x, Packed8):
        _matrix(x.codes, "x", dev, torch.uint8, (n * hw, c))
        x_ptr, ld_x, sample_x, xf = 0, 0, 0, x.fields()
    else:
        if x.dtype != dy.dtype or x.shape != dy.shape or x.get_device() != dev:
            raise ValueError("x must have dy's type, shape and device")
        _, _, _, ld_x, sample_x = _pixels(x, "x")
        x_ptr, xf = x.data_ptr(), _NONE8
    lib = _library()
    with _On(dev) as stream:
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        dparam = torch.empty((2, c), dtype=torch.float32, device=dy.device)
        dgamma, dbeta = dparam.unbind(0)
        args = (_NORM.size, dt, code, groups, n, hw, c, 1.0, x_ptr, ld_x, sample_x, dy.data_ptr(), ld, sample, dx.data_ptr(), c, hw * c,
                *vectors, dgamma.data_ptr(), dbeta.data_ptr(), *xf, *_NONE8)
        _call(lib.lqsgd_group_norm_backward, args, _NORM, lib.lqsgd_group_norm_workspace_bytes, 1, dy.device, stream)
    return dx, dgamma, dbeta


# ------------------------------------------------------------------------------------- differentiable layers, 8 bits in between

class _LinearLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act, x8):
        w = weight.to(x.dtype)
        r = linear(x, w, bias, act, residual, save_z8=act != "none")
        x8 = pack8(x) if x8 is None else x8
        saved = [w, x8.codes, x8.exps] + ([r.z8.codes, r.z8.exps] if r.z8 is not None else [])
        ctx.save_for_backward(*saved)
        ctx.act, ctx.has_bias, ctx.has_residual = act, bias is not None, residual is not None
        return r.y

    @staticmethod
    def backward(ctx, dy):
        w, xc, xe, *z = ctx.saved_tensors
        dy = dy if dy.stride(-1) == 1 else dy.contiguous()
        dz, db = act_grad(dy, Packed8(*z) if z else None, ctx.act, bias_grad=ctx.has_bias and ctx.needs_input_grad[2])
        dx = linear_grad_input(dz, w) if ctx.needs_input_grad[0] else None
        dw = linear_grad_weight(dz, Packed8(xc, xe)) if ctx.needs_input_grad[1] else None
        return dx, dw, db, (dy if ctx.has_residual else None), None, None


def linear_layer(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
                 residual: Optional[torch.Tensor] = None, x8: Optional[Packed8] = None) -> torch.Tensor:
    """linear() as a differentiable function: weight and bias float32 (the weights a round updates; the products run in x's
    type), x and the pre-activation kept in 8 bits, the weight gradient float32.  x8: x's 8-bit form where it exists
    already (norm_layer and other producers can hand it on)."""
    return _LinearLayer.apply(x, weight, bias, residual, act, x8)


class _NormLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, groups, eps, act, keep):
        r = group_norm(x, groups, gamma, beta, eps, act, save_x8=True, save_y8=keep is not None)
        ctx.save_for_backward(r.x8.codes, r.x8.exps, gamma, beta, r.mean, r.rstd)
        ctx.groups, ctx.act = groups, act
        if keep is not None:
            keep.append(r.y8)
        return r.y

    @staticmethod
    def backward(ctx, dy):
        codes, exps, gamma, beta, mean, rstd = ctx.saved_tensors
        dx, dgamma, dbeta = group_norm_grad(dy.contiguous(), Packed8(codes, exps), ctx.groups, gamma, beta, mean, rstd, ctx.act)
        return dx, dgamma, dbeta, None, None, None, None


def norm_layer(x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, groups: int, eps: float = 1e-5, act: str = "none",
               keep: Optional[list] = None) -> torch.Tensor:
    """group_norm() as a differentiable function with x kept in 8 bits.  `keep`, a list, receives the output's 8-bit form
    (for the linear layer that follows)."""
    return _NormLayer.apply(x, gamma, beta, groups, eps, act, keep)
