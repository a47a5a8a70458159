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
from typing import NamedTuple, Optional, Tuple, Union

import torch

from . import binding as B

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
GROUP = 32
FORWARD, GRAD_INPUT, GRAD_WEIGHT = 0, 1, 2


class CPacked8(C.Structure):
    _fields_ = [("dev_codes", C.c_void_p), ("ld_codes", C.c_int64), ("dev_exps", C.c_void_p), ("ld_exps", C.c_int64)]


class CLinear(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("act", C.c_int32), ("accumulate", C.c_int32),
                ("rows", C.c_int64), ("in_", C.c_int32), ("out", C.c_int32),
                ("dev_x", C.c_void_p), ("ld_x", C.c_int64), ("dev_w", C.c_void_p), ("ld_w", C.c_int64),
                ("dev_dz", C.c_void_p), ("ld_dz", C.c_int64), ("dev_bias", C.c_void_p),
                ("dev_residual", C.c_void_p), ("ld_residual", C.c_int64), ("dev_out", C.c_void_p), ("ld_out", C.c_int64),
                ("x8", CPacked8), ("z8", CPacked8), ("y8", CPacked8),
                ("dev_status", C.c_void_p), ("dev_workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class CGroupNorm(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("act", C.c_int32), ("groups", C.c_int32),
                ("n", C.c_int32), ("hw", C.c_int32), ("c", C.c_int32), ("eps", C.c_float),
                ("dev_x", C.c_void_p), ("ld_x", C.c_int64), ("sample_x", C.c_int64),
                ("dev_dy", C.c_void_p), ("ld_dy", C.c_int64), ("sample_dy", C.c_int64),
                ("dev_out", C.c_void_p), ("ld_out", C.c_int64), ("sample_out", C.c_int64),
                ("dev_gamma", C.c_void_p), ("dev_beta", C.c_void_p), ("dev_mean", C.c_void_p), ("dev_rstd", C.c_void_p),
                ("dev_dgamma", C.c_void_p), ("dev_dbeta", C.c_void_p),
                ("x8", CPacked8), ("y8", CPacked8), ("dev_workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


_lib = None


def _library() -> C.CDLL:
    global _lib
    if _lib is None:
        lib = B.load_library()
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        lib.lqsgd_pack8.argtypes = [vp, i64, i32, i64, i32, C.POINTER(CPacked8), vp]
        lib.lqsgd_unpack8.argtypes = [C.POINTER(CPacked8), i64, i32, vp, i64, i32, vp]
        lib.lqsgd_act_grad_workspace_bytes.argtypes = [i64, i32, C.POINTER(sz)]
        lib.lqsgd_act_grad.argtypes = [vp, i64, C.POINTER(CPacked8), i32, i32, i64, i32, vp, i64, vp, vp, sz, vp]
        lib.lqsgd_linear_workspace_bytes.argtypes = [i32, C.POINTER(CLinear), C.POINTER(sz)]
        for f in (lib.lqsgd_linear_forward, lib.lqsgd_linear_grad_input, lib.lqsgd_linear_grad_weight):
            f.argtypes = [C.POINTER(CLinear), vp]
        lib.lqsgd_group_norm_workspace_bytes.argtypes = [i32, C.POINTER(CGroupNorm), C.POINTER(sz)]
        for f in (lib.lqsgd_group_norm_forward, lib.lqsgd_group_norm_backward):
            f.argtypes = [C.POINTER(CGroupNorm), vp]
        _lib = lib
    return _lib


def _need(ok: bool, text: str) -> None:
    if not ok:
        raise ValueError(text)


def _act(name: str) -> int:
    _need(name in ACTS, f"act must be one of {sorted(ACTS)}, not {name!r}")
    return ACTS[name]


def _matrix(t: torch.Tensor, what: str, dtype: Optional[torch.dtype] = None, shape=None) -> torch.Tensor:
    _need(t.is_cuda, f"{what} must be a CUDA tensor")
    _need(t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1), f"{what} must be a matrix with unit stride along its rows")
    _need(dtype is None or t.dtype == dtype, f"{what} must be {dtype}, not {t.dtype}")
    _need(shape is None or tuple(t.shape) == tuple(shape), f"{what} must have shape {shape}, not {tuple(t.shape)}")
    return t


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _vector(t: torch.Tensor, what: str, n: int) -> torch.Tensor:
    _need(t.is_cuda and t.dtype == torch.float32 and t.numel() == n and t.is_contiguous(),
          f"{what} must be a contiguous float32 CUDA vector of {n}")
    return t


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


class _On:
    """The tensors' device made current for a call (a no-op when it already is), and its current stream."""

    def __init__(self, device: torch.device, *others: Optional[torch.Tensor]):
        for t in others:
            _need(t is None or t.device == device, "all tensors must be on one device")
        self.guard = None if torch.cuda.current_device() == device.index else torch.cuda.device(device)
        self.device = device

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return C.c_void_p(torch.cuda.current_stream(self.device).cuda_stream)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _workspace(nbytes: int, device: torch.device) -> Optional[torch.Tensor]:
    # from PyTorch's allocator, on the current stream: its memory is not handed out again before the call's kernels are done
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


_status = {}


def _status_word(device: torch.device) -> Optional[torch.Tensor]:
    word = _status.get(device.index)
    if word is None and not torch.cuda.is_current_stream_capturing():
        word = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.current_stream(device).synchronize()
        _status[device.index] = word
    return word


def status(device: Union[str, int, torch.device] = "cuda:0") -> int:
    """Status bits (binding.STATUS_TIMEOUT) that the linear layers' kernels have raised on a device so far; synchronises."""
    word = _status.get(torch.device(device).index or 0)
    return 0 if word is None else int(word.item())


# ------------------------------------------------------------------------------------------------ activations in 8 bits

class Packed8:
    """A matrix kept in 8 bits: codes, uint8 rows x cols, and exps, uint8 rows x ceil(cols / 32) (see lqsgd_packed8)."""

    __slots__ = ("codes", "exps")

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor):
        _matrix(codes, "codes", torch.uint8)
        _matrix(exps, "exps", torch.uint8, (codes.shape[0], (codes.shape[1] + GROUP - 1) // GROUP))
        self.codes, self.exps = codes, exps

    @staticmethod
    def empty(rows: int, cols: int, device) -> "Packed8":
        """Uninitialised; rows start on 16-byte boundaries."""
        wide = torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.uint8, device=device)
        return Packed8(wide[:, :cols], torch.empty((rows, (cols + GROUP - 1) // GROUP), dtype=torch.uint8, device=device))

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def c(self) -> CPacked8:
        return CPacked8(self.codes.data_ptr(), _ld(self.codes), self.exps.data_ptr(), _ld(self.exps))


def pack8(x: torch.Tensor, out: Optional[Packed8] = None) -> Packed8:
    """The 8-bit form of a matrix (bfloat16, float16 or float32)."""
    _matrix(x, "x")
    _need(x.dtype in DTYPES, f"x must be one of {list(DTYPES)}")
    if out is None:
        out = Packed8.empty(x.shape[0], x.shape[1], x.device)
    _need(tuple(out.shape) == tuple(x.shape), "out must have x's shape")
    with _On(x.device, out.codes, out.exps) as stream:
        B._check(_library().lqsgd_pack8(_ptr(x), _ld(x), DTYPES[x.dtype], x.shape[0], x.shape[1], C.byref(out.c()), stream))
    return out


def unpack8(p: Packed8, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values an 8-bit form stands for: exact in bfloat16 and float32 (float16: within its range)."""
    _need(dtype in DTYPES, f"dtype must be one of {list(DTYPES)}")
    if out is None:
        out = torch.empty(tuple(p.shape), dtype=dtype, device=p.device)
    _matrix(out, "out", dtype, p.shape)
    with _On(p.device, out) as stream:
        B._check(_library().lqsgd_unpack8(C.byref(p.c()), p.shape[0], p.shape[1], _ptr(out), _ld(out), DTYPES[dtype], stream))
    return out


def act_grad(dy: torch.Tensor, z8: Optional[Packed8], act: str = "none", bias_grad: bool = True,
             out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(dz, db): dz = dy act'(z) with z from its 8-bit form, db its column sums in float32 (None without bias_grad).
    With act "none" dz is dy itself.  `out` may be dy."""
    _matrix(dy, "dy")
    _need(dy.dtype in DTYPES, f"dy must be one of {list(DTYPES)}")
    a = _act(act)
    if a == 0:
        if not bias_grad:
            return dy, None
        dz, zc = None, None
    else:
        _need(z8 is not None and tuple(z8.shape) == tuple(dy.shape), "z8 must be the 8-bit form of a matrix of dy's shape")
        dz = torch.empty(tuple(dy.shape), dtype=dy.dtype, device=dy.device) if out is None else _matrix(out, "out", dy.dtype, dy.shape)
        zc = C.byref(z8.c())
    rows, cols = dy.shape
    lib = _library()
    with _On(dy.device, dz, z8.codes if a else None) as stream:
        db = torch.empty(cols, dtype=torch.float32, device=dy.device) if bias_grad else None
        need = C.c_size_t(0)
        if bias_grad:
            B._check(lib.lqsgd_act_grad_workspace_bytes(rows, cols, C.byref(need)))
        ws = _workspace(need.value, dy.device)
        B._check(lib.lqsgd_act_grad(_ptr(dy), _ld(dy), zc, a, DTYPES[dy.dtype], rows, cols, _ptr(dz), _ld(dz) if dz is not None else 0,
                                    _ptr(db), _ptr(ws), need.value, stream))
    return (dy if dz is None else dz), db


# -------------------------------------------------------------------------------------------------------- linear layers

class LinearOut(NamedTuple):
    y: torch.Tensor
    z8: Optional[Packed8]
    y8: Optional[Packed8]


def _linear_call(product: int, a: CLinear, device: torch.device, stream) -> None:
    lib = _library()
    a.struct_size = C.sizeof(CLinear)
    a.dev_status = _ptr(_status_word(device))
    need = C.c_size_t(0)
    B._check(lib.lqsgd_linear_workspace_bytes(product, C.byref(a), C.byref(need)))
    ws = _workspace(need.value, device)
    a.dev_workspace, a.workspace_bytes = _ptr(ws), need.value
    B._check((lib.lqsgd_linear_forward, lib.lqsgd_linear_grad_input, lib.lqsgd_linear_grad_weight)[product](C.byref(a), stream))


def linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
           residual: Optional[torch.Tensor] = None, save_z8: bool = False, save_y8: bool = False,
           out: Optional[torch.Tensor] = None) -> LinearOut:
    """y = act(x w^T + bias) + residual, x rows x in and w out x in, bfloat16 or float16; bias float32.
    save_z8 / save_y8 also return the 8-bit form of the pre-activation x w^T + bias / of y.  `out` may be the residual."""
    _matrix(x, "x")
    _need(x.dtype in (torch.bfloat16, torch.float16), "x must be bfloat16 or float16")
    rows, cin = x.shape
    _matrix(w, "w", x.dtype)
    cout = w.shape[0]
    _need(w.shape[1] == cin, f"w must have {cin} columns, not {w.shape[1]}")
    if bias is not None:
        _vector(bias, "bias", cout)
    if residual is not None:
        _matrix(residual, "residual", x.dtype, (rows, cout))
    code = _act(act)
    with _On(x.device, w, bias, residual, out) as stream:
        y = torch.empty((rows, cout), dtype=x.dtype, device=x.device) if out is None else _matrix(out, "out", x.dtype, (rows, cout))
        z8 = Packed8.empty(rows, cout, x.device) if save_z8 else None
        y8 = Packed8.empty(rows, cout, x.device) if save_y8 else None
        a = CLinear(dtype=DTYPES[x.dtype], act=code, rows=rows, in_=cin, out=cout, dev_x=_ptr(x), ld_x=_ld(x), dev_w=_ptr(w), ld_w=_ld(w),
                    dev_bias=_ptr(bias), dev_residual=_ptr(residual), ld_residual=0 if residual is None else _ld(residual),
                    dev_out=_ptr(y), ld_out=_ld(y))
        if z8 is not None:
            a.z8 = z8.c()
        if y8 is not None:
            a.y8 = y8.c()
        _linear_call(FORWARD, a, x.device, stream)
    return LinearOut(y, z8, y8)


def linear_grad_input(dz: torch.Tensor, w: torch.Tensor, residual: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx = dz w + residual (the gradient that came down the skip connection).  `out` may be the residual."""
    _matrix(dz, "dz")
    _need(dz.dtype in (torch.bfloat16, torch.float16), "dz must be bfloat16 or float16")
    rows, cout = dz.shape
    _matrix(w, "w", dz.dtype)
    _need(w.shape[0] == cout, f"w must have {cout} rows, not {w.shape[0]}")
    cin = w.shape[1]
    if residual is not None:
        _matrix(residual, "residual", dz.dtype, (rows, cin))
    with _On(dz.device, w, residual, out) as stream:
        dx = torch.empty((rows, cin), dtype=dz.dtype, device=dz.device) if out is None else _matrix(out, "out", dz.dtype, (rows, cin))
        a = CLinear(dtype=DTYPES[dz.dtype], rows=rows, in_=cin, out=cout, dev_dz=_ptr(dz), ld_dz=_ld(dz), dev_w=_ptr(w), ld_w=_ld(w),
                    dev_residual=_ptr(residual), ld_residual=0 if residual is None else _ld(residual), dev_out=_ptr(dx), ld_out=_ld(dx))
        _linear_call(GRAD_INPUT, a, dz.device, stream)
    return dx


def linear_grad_weight(dz: torch.Tensor, x: Union[torch.Tensor, Packed8], out: Optional[torch.Tensor] = None,
                       accumulate: bool = False) -> torch.Tensor:
    """dw = dz^T x in float32, out x in: the gradient a round takes.  x is a matrix of dz's type or its 8-bit form.
    accumulate adds to `out` (a gradient over several micro-batches)."""
    _matrix(dz, "dz")
    _need(dz.dtype in (torch.bfloat16, torch.float16), "dz must be bfloat16 or float16")
    rows, cout = dz.shape
    packed = isinstance(x, Packed8)
    if not packed:
        _matrix(x, "x", dz.dtype)
    _need(x.shape[0] == rows, f"x must have {rows} rows, not {x.shape[0]}")
    cin = x.shape[1]
    _need(not accumulate or out is not None, "accumulate needs out")
    with _On(dz.device, x.codes if packed else x, out) as stream:
        dw = torch.empty((cout, cin), dtype=torch.float32, device=dz.device) if out is None else _matrix(out, "out", torch.float32, (cout, cin))
        a = CLinear(dtype=DTYPES[dz.dtype], accumulate=int(accumulate), rows=rows, in_=cin, out=cout, dev_dz=_ptr(dz), ld_dz=_ld(dz),
                    dev_out=_ptr(dw), ld_out=_ld(dw))
        if packed:
            a.x8 = x.c()
        else:
            a.dev_x, a.ld_x = _ptr(x), _ld(x)
        _linear_call(GRAD_WEIGHT, a, dz.device, stream)
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
    _need(t.is_cuda, f"{what} must be a CUDA tensor")
    _need(t.dim() >= 2 and (t.shape[-1] <= 1 or t.stride(-1) == 1), f"{what} must be samples x ... x channels, channels with unit stride")
    n, c = t.shape[0], t.shape[-1]
    hw, ld = 1, None
    for d in range(t.dim() - 2, 0, -1):                     # the pixel dimensions must fold into one with a fixed distance
        if t.shape[d] == 1:
            continue
        if ld is None:
            ld = t.stride(d)
        else:
            _need(t.stride(d) == ld * hw, f"{what}'s pixel dimensions must be contiguous with one another")
        hw *= t.shape[d]
    ld = c if ld is None else ld
    return n, hw, c, ld, (t.stride(0) if n > 1 else hw * ld)


def group_norm(x: torch.Tensor, groups: int, gamma: torch.Tensor, beta: torch.Tensor, eps: float = 1e-5, act: str = "none",
               save_x8: bool = False, save_y8: bool = False) -> GroupNormOut:
    """y = act(gamma (x - mean) rstd + beta) over `groups` groups of channels of each sample; x is samples x ... x channels,
    bfloat16, float16 or float32, gamma and beta float32.  save_x8 / save_y8 also return 8-bit forms (rows = pixels)."""
    n, hw, c, ld, sample = _pixels(x, "x")
    _need(x.dtype in DTYPES, f"x must be one of {list(DTYPES)}")
    _vector(gamma, "gamma", c), _vector(beta, "beta", c)
    code, lib = _act(act), _library()
    with _On(x.device, gamma, beta) as stream:
        y = torch.empty(tuple(x.shape), dtype=x.dtype, device=x.device)
        mean = torch.empty((n, max(1, groups)), dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
        x8 = Packed8.empty(n * hw, c, x.device) if save_x8 else None
        y8 = Packed8.empty(n * hw, c, x.device) if save_y8 else None
        a = CGroupNorm(struct_size=C.sizeof(CGroupNorm), dtype=DTYPES[x.dtype], act=code, groups=groups, n=n, hw=hw, c=c, eps=eps,
                       dev_x=_ptr(x), ld_x=ld, sample_x=sample, dev_out=_ptr(y), ld_out=c, sample_out=hw * c,
                       dev_gamma=_ptr(gamma), dev_beta=_ptr(beta), dev_mean=_ptr(mean), dev_rstd=_ptr(rstd))
        if x8 is not None:
            a.x8 = x8.c()
        if y8 is not None:
            a.y8 = y8.c()
        need = C.c_size_t(0)
        B._check(lib.lqsgd_group_norm_workspace_bytes(0, C.byref(a), C.byref(need)))
        ws = _workspace(need.value, x.device)
        a.dev_workspace, a.workspace_bytes = _ptr(ws), need.value
        B._check(lib.lqsgd_group_norm_forward(C.byref(a), stream))
    return GroupNormOut(y, mean, rstd, x8, y8)


def group_norm_grad(dy: torch.Tensor, x: Union[torch.Tensor, Packed8], groups: int, gamma: torch.Tensor, beta: torch.Tensor,
                    mean: torch.Tensor, rstd: torch.Tensor, act: str = "none") -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dgamma, dbeta) of group_norm; x as the forward call had it, or its 8-bit form; mean and rstd as it returned them."""
    n, hw, c, ld, sample = _pixels(dy, "dy")
    _need(dy.dtype in DTYPES, f"dy must be one of {list(DTYPES)}")
    _vector(gamma, "gamma", c), _vector(beta, "beta", c)
    _vector(mean, "mean", n * groups), _vector(rstd, "rstd", n * groups)
    packed = isinstance(x, Packed8)
    if packed:
        _need(tuple(x.shape) == (n * hw, c), f"x must be the 8-bit form of {n * hw} x {c} values")
    else:
        _need(x.dtype == dy.dtype and tuple(x.shape) == tuple(dy.shape), "x must have dy's type and shape")
    code, lib = _act(act), _library()
    with _On(dy.device, x.codes if packed else x, gamma, beta, mean, rstd) as stream:
        dx = torch.empty(tuple(dy.shape), dtype=dy.dtype, device=dy.device)
        dgamma = torch.empty(c, dtype=torch.float32, device=dy.device)
        dbeta = torch.empty(c, dtype=torch.float32, device=dy.device)
        a = CGroupNorm(struct_size=C.sizeof(CGroupNorm), dtype=DTYPES[dy.dtype], act=code, groups=groups, n=n, hw=hw, c=c, eps=1.0,
                       dev_dy=_ptr(dy), ld_dy=ld, sample_dy=sample, dev_out=_ptr(dx), ld_out=c, sample_out=hw * c,
                       dev_gamma=_ptr(gamma), dev_beta=_ptr(beta), dev_mean=_ptr(mean), dev_rstd=_ptr(rstd),
                       dev_dgamma=_ptr(dgamma), dev_dbeta=_ptr(dbeta))
        if packed:
            a.x8 = x.c()
        else:
            _, _, _, a.ld_x, a.sample_x = _pixels(x, "x")
            a.dev_x = _ptr(x)
        need = C.c_size_t(0)
        B._check(lib.lqsgd_group_norm_workspace_bytes(1, C.byref(a), C.byref(need)))
        ws = _workspace(need.value, dy.device)
        a.dev_workspace, a.workspace_bytes = _ptr(ws), need.value
        B._check(lib.lqsgd_group_norm_backward(C.byref(a), stream))
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
