"""Host-side checks of the RMS norm, dropout and the products of 8-bit rows that need no GPU: struct layouts, refusals, workspace sizes,
and the test oracles' own generator against its published answers.  Every refused call returns before it touches a device."""
import ctypes as C

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from paper_2506_17974_b200 import binding as B
from paper_2506_17974_b200 import training as tr
import rows_oracle as ro

I32, I64, U32, U64, PTR, SIZE = C.c_int32, C.c_int64, C.c_uint32, C.c_uint64, C.c_void_p, C.c_size_t
BF16, F16, F32 = 0, 1, 2
AT = 0x7f0000000000                                             # an aligned address that nothing reads


class Packed8(C.Structure):
    _fields_ = [("codes", PTR), ("ld_codes", I64), ("exps", PTR), ("ld_exps", I64)]


class Rows8(C.Structure):
    _fields_ = [("codes", PTR), ("ld_codes", I64), ("scales", PTR)]


class Drop(C.Structure):
    _fields_ = [("p", C.c_float), ("reserved", U32), ("seed", U64), ("offset", U64), ("dev_seed", PTR)]


class Rms(C.Structure):
    _fields_ = [("struct_size", U32), ("dtype", I32), ("rows", I64), ("cols", I32), ("eps", C.c_float), ("drop", Drop),
                ("x", PTR), ("ld_x", I64), ("residual", PTR), ("ld_residual", I64), ("dy", PTR), ("ld_dy", I64), ("skip", PTR), ("ld_skip", I64),
                ("h", PTR), ("ld_h", I64), ("y", PTR), ("ld_y", I64), ("dx", PTR), ("ld_dx", I64), ("dresidual", PTR), ("ld_dresidual", I64),
                ("gamma", PTR), ("rstd", PTR), ("dgamma", PTR), ("h8", Packed8), ("y8", Packed8), ("rows8", Rows8), ("workspace", PTR), ("workspace_bytes", SIZE)]


class Linear8(C.Structure):
    _fields_ = [("struct_size", U32), ("dtype", I32), ("act", I32), ("reserved", U32), ("rows", I64), ("cin", I32), ("cout", I32), ("x", Rows8), ("w", Rows8),
                ("bias", PTR), ("residual", PTR), ("ld_residual", I64), ("out", PTR), ("ld_out", I64), ("z8", Packed8), ("y8", Packed8),
                ("status", PTR), ("workspace", PTR), ("workspace_bytes", SIZE)]


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return tr._library()


def rms(**kw):
    a = Rms(struct_size=C.sizeof(Rms), rows=64, cols=128, eps=1e-6, x=AT, ld_x=128, residual=AT, ld_residual=128, dy=AT, ld_dy=128, h=AT, ld_h=128, y=AT, ld_y=128,
            dx=AT, ld_dx=128, gamma=AT, rstd=AT, dgamma=AT)
    for k, v in kw.items():
        if k in ("p", "reserved", "dev_seed"):
            setattr(a.drop, k, v)
        else:
            setattr(a, k, v)
    return a


def linear8(**kw):
    a = Linear8(struct_size=C.sizeof(Linear8), rows=64, cin=128, cout=96, x=Rows8(AT, 128, AT), w=Rows8(AT, 128, AT), out=AT, ld_out=96)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def packed(codes=AT, ld_codes=128, exps=AT, ld_exps=4):
    return Packed8(codes, ld_codes, exps, ld_exps)


def test_struct_sizes():
    assert C.sizeof(Rows8) == tr._ROWS8.size == 24
    assert C.sizeof(Drop) == tr._DROP.size == 32
    assert C.sizeof(Rms) == tr._RMS.size
    assert C.sizeof(Linear8) == tr._LINEAR8.size


def test_generator_gives_the_published_answers():
    """Philox4x32-10 of all zeros, of all ones, and of digits of pi (the vectors published with the generator)."""
    ones = (1 << 32) - 1
    assert ro.philox((0, 0, 0, 0), (0, 0)) == (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)
    assert ro.philox((ones,) * 4, (ones,) * 2) == (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)
    assert ro.philox((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)


def test_mask_follows_the_single_counters():
    """The oracle's whole mask against the generator called once per run of 8."""
    seed, offset, rows, cols, p = 0x123456789abcdef0, 0xfedcba9876543210, 3, 21, 0.3
    keep = ro.kept(rows, cols, p, seed, offset)
    t = round(65536 * p)
    for r in range(rows):
        for c in range(cols):
            b = r * 3 + c // 8
            w = ro.philox((b & 0xffffffff, b >> 32, offset & 0xffffffff, offset >> 32), (seed & 0xffffffff, seed >> 32))[(c % 8) // 2]
            assert keep[r, c] == ((w >> (16 * (c % 2))) & 0xffff >= t)


def test_gradient_formula_against_differences():
    """The oracle's gradients of the norm against central differences in 64 bits."""
    g = np.random.default_rng(3)
    h, gamma, dy, skip = g.normal(size=(3, 11)), g.normal(size=11) + 1, g.normal(size=(3, 11)), g.normal(size=(3, 11))
    eps, step = 1e-3, 1e-6

    def loss(h, gamma):
        return (dy * h * gamma / np.sqrt((h * h).mean(1, keepdims=True) + eps)).sum() + (skip * h).sum()

    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    d, dgamma = ro.rms_grad(dy, h, gamma, rstd, skip)
    for i in range(3):
        for j in range(11):
            e = np.zeros_like(h)
            e[i, j] = step
            assert abs((loss(h + e, gamma) - loss(h - e, gamma)) / (2 * step) - d[i, j]) < 1e-7
    for j in range(11):
        e = np.zeros_like(gamma)
        e[j] = step
        assert abs((loss(h, gamma + e) - loss(h, gamma - e)) / (2 * step) - dgamma[j]) < 1e-7


@pytest.mark.parametrize("change,code", [
    (dict(struct_size=8), B.ERR_INVALID_ARG), (dict(dtype=7), B.ERR_INVALID_ARG), (dict(rows=-1), B.ERR_BAD_SHAPE), (dict(rows=1 << 31), B.ERR_BAD_SHAPE),
    (dict(cols=0), B.ERR_BAD_SHAPE), (dict(cols=(1 << 24) + 1), B.ERR_BAD_SHAPE), (dict(p=1.0), B.ERR_INVALID_ARG), (dict(p=-0.1), B.ERR_INVALID_ARG),
    (dict(p=float("nan")), B.ERR_INVALID_ARG), (dict(reserved=1), B.ERR_INVALID_ARG), (dict(dev_seed=AT + 4), B.ERR_MISALIGNED),
    (dict(gamma=0), B.ERR_INVALID_ARG), (dict(rstd=0), B.ERR_INVALID_ARG), (dict(gamma=AT + 2), B.ERR_MISALIGNED), (dict(rstd=AT + 1), B.ERR_MISALIGNED),
    (dict(h8=packed(ld_codes=127)), B.ERR_INVALID_ARG), (dict(h8=packed(ld_exps=3)), B.ERR_INVALID_ARG)])
def test_norm_refusals_of_both_directions(lib, change, code):
    for fn in (lib.lqsgd_rms_norm_forward, lib.lqsgd_rms_norm_backward):
        assert fn(C.byref(rms(**change)), None) == code, fn


@pytest.mark.parametrize("change,code", [
    (dict(eps=-1.0), B.ERR_INVALID_ARG), (dict(eps=float("nan")), B.ERR_INVALID_ARG), (dict(eps=float("inf")), B.ERR_INVALID_ARG), (dict(x=0), B.ERR_INVALID_ARG),
    (dict(ld_x=127), B.ERR_INVALID_ARG), (dict(x=AT + 1), B.ERR_MISALIGNED), (dict(ld_residual=100), B.ERR_INVALID_ARG), (dict(residual=AT + 1), B.ERR_MISALIGNED),
    (dict(h=0), B.ERR_INVALID_ARG), (dict(h=0, residual=0, p=0.5), B.ERR_INVALID_ARG), (dict(ld_h=127), B.ERR_INVALID_ARG), (dict(y=AT + 1), B.ERR_MISALIGNED),
    (dict(ld_y=127), B.ERR_INVALID_ARG), (dict(y8=packed(exps=0)), B.ERR_INVALID_ARG), (dict(rows8=Rows8(AT, 127, AT)), B.ERR_INVALID_ARG),
    (dict(rows8=Rows8(AT, 128, 0)), B.ERR_INVALID_ARG), (dict(rows8=Rows8(AT, 128, AT + 2)), B.ERR_MISALIGNED)])
def test_norm_forward_refusals(lib, change, code):
    assert lib.lqsgd_rms_norm_forward(C.byref(rms(**change)), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(dx=0, dresidual=0, dgamma=0), B.ERR_INVALID_ARG), (dict(dy=0), B.ERR_INVALID_ARG), (dict(ld_dy=127), B.ERR_INVALID_ARG), (dict(dy=AT + 1), B.ERR_MISALIGNED),
    (dict(skip=AT, ld_skip=127), B.ERR_INVALID_ARG), (dict(skip=AT + 1, ld_skip=128), B.ERR_MISALIGNED), (dict(h=0), B.ERR_INVALID_ARG), (dict(ld_h=3), B.ERR_INVALID_ARG),
    (dict(ld_dx=127), B.ERR_INVALID_ARG), (dict(dresidual=AT + 1, ld_dresidual=128), B.ERR_MISALIGNED), (dict(dgamma=AT + 2), B.ERR_MISALIGNED),
    (dict(workspace=0), B.ERR_WORKSPACE_TOO_SMALL), (dict(workspace=AT + 8, workspace_bytes=1 << 30), B.ERR_MISALIGNED)])
def test_norm_backward_refusals(lib, change, code):
    change.setdefault("rows", 4096)                         # sums over many rows meet in the workspace
    assert lib.lqsgd_rms_norm_backward(C.byref(rms(**change)), None) == code


def test_norm_workspace(lib):
    need = SIZE(99)
    assert lib.lqsgd_rms_norm_workspace_bytes(0, C.byref(rms()), C.byref(need)) == 0 and need.value == 0
    assert lib.lqsgd_rms_norm_workspace_bytes(1, C.byref(rms(rows=8192, cols=4096)), C.byref(need)) == 0 and 0 < need.value <= 16 << 20
    assert lib.lqsgd_rms_norm_workspace_bytes(1, C.byref(rms(rows=0)), C.byref(need)) == 0 and need.value == 0
    assert lib.lqsgd_rms_norm_workspace_bytes(2, C.byref(rms()), C.byref(need)) == B.ERR_INVALID_ARG
    assert lib.lqsgd_rms_norm_workspace_bytes(1, C.byref(rms()), None) == B.ERR_INVALID_ARG
    assert lib.lqsgd_rms_norm_workspace_bytes(1, C.byref(rms(cols=0)), C.byref(need)) == B.ERR_BAD_SHAPE


def test_dropout_refusals(lib):
    def call(x=AT, ld=128, r=None, ld_r=0, dtype=BF16, rows=4, cols=128, p=0.5, out=AT, ld_o=128, reserved=0, dev_seed=None):
        d = Drop(p, reserved, 1, 2, dev_seed)
        return lib.lqsgd_dropout(x, ld, r, ld_r, dtype, rows, cols, C.byref(d), out, ld_o, None)

    assert lib.lqsgd_dropout(AT, 128, None, 0, BF16, 4, 128, None, AT, 128, None) == B.ERR_INVALID_ARG
    for kw in (dict(dtype=3), dict(p=1.0), dict(p=-1.0), dict(p=float("nan")), dict(reserved=3), dict(x=None), dict(out=None), dict(ld=127), dict(ld_o=127),
               dict(r=AT, ld_r=127)):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 24) + 1)):
        assert call(**kw) == B.ERR_BAD_SHAPE, kw
    for kw in (dict(x=AT + 1), dict(out=AT + 1), dict(r=AT + 1, ld_r=128), dict(dev_seed=AT + 4), dict(x=AT + 2, dtype=F32)):
        assert call(**kw) == B.ERR_MISALIGNED, kw
    assert call(rows=0, x=None, out=None) == 0


def test_rows8_refusals(lib):
    for fn in (lib.lqsgd_pack_rows8, lib.lqsgd_unpack_rows8):
        def call(m=AT, ld=128, dtype=BF16, rows=4, cols=128, r=Rows8(AT, 128, AT)):
            pr = None if r is None else C.byref(r)
            if fn is lib.lqsgd_pack_rows8:
                return fn(m, ld, dtype, rows, cols, pr, None)
            return fn(pr, rows, cols, m, ld, dtype, None)
        for kw in (dict(m=None), dict(ld=127), dict(dtype=3), dict(r=None), dict(r=Rows8(None, 128, AT)), dict(r=Rows8(AT, 127, AT)), dict(r=Rows8(AT, 128, None))):
            assert call(**kw) == B.ERR_INVALID_ARG, kw
        for kw in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 24) + 1)):
            assert call(**kw) == B.ERR_BAD_SHAPE, kw
        for kw in (dict(m=AT + 1), dict(r=Rows8(AT, 128, AT + 2))):
            assert call(**kw) == B.ERR_MISALIGNED, kw
        assert call(rows=0, m=None) == 0


@pytest.mark.parametrize("change,code", [
    (dict(struct_size=8), B.ERR_INVALID_ARG), (dict(dtype=F32), B.ERR_INVALID_ARG), (dict(act=4), B.ERR_INVALID_ARG), (dict(act=-1), B.ERR_INVALID_ARG),
    (dict(reserved=1), B.ERR_INVALID_ARG), (dict(rows=-1), B.ERR_BAD_SHAPE), (dict(rows=1 << 31), B.ERR_BAD_SHAPE), (dict(cin=0), B.ERR_BAD_SHAPE),
    (dict(cin=131072), B.ERR_BAD_SHAPE), (dict(cout=0), B.ERR_BAD_SHAPE), (dict(cout=(1 << 24) + 1), B.ERR_BAD_SHAPE), (dict(x=Rows8(None, 128, AT)), B.ERR_INVALID_ARG),
    (dict(x=Rows8(AT, 127, AT)), B.ERR_INVALID_ARG), (dict(x=Rows8(AT, 128, None)), B.ERR_INVALID_ARG), (dict(w=Rows8(AT, 127, AT)), B.ERR_INVALID_ARG),
    (dict(w=Rows8(AT, 128, AT + 1)), B.ERR_MISALIGNED), (dict(out=0), B.ERR_INVALID_ARG), (dict(ld_out=95), B.ERR_INVALID_ARG), (dict(out=AT + 1), B.ERR_MISALIGNED),
    (dict(residual=AT, ld_residual=95), B.ERR_INVALID_ARG), (dict(residual=AT + 1, ld_residual=96), B.ERR_MISALIGNED), (dict(bias=AT + 2), B.ERR_MISALIGNED),
    (dict(status=AT + 2), B.ERR_MISALIGNED), (dict(z8=packed(ld_codes=95)), B.ERR_INVALID_ARG), (dict(y8=packed(ld_exps=2)), B.ERR_INVALID_ARG),
    (dict(x=Rows8(AT + 1, 128, AT)), B.ERR_WORKSPACE_TOO_SMALL)])
def test_linear_rows8_refusals(lib, change, code):
    assert lib.lqsgd_linear_rows8_forward(C.byref(linear8(**change)), None) == code


def test_linear_rows8_workspace(lib):
    need = SIZE(99)
    ask = lambda **kw: lib.lqsgd_linear_rows8_workspace_bytes(C.byref(linear8(**kw)), C.byref(need))      # noqa: E731
    assert ask() == 0 and need.value == 0                                                                 # one tile, one k block
    assert ask(rows=0) == 0 and need.value == 0
    assert ask(x=Rows8(AT, 129, AT)) == 0 and need.value >= 64 * 128                                      # an aligned copy
    assert ask(cin=131072) == B.ERR_BAD_SHAPE
    assert lib.lqsgd_linear_rows8_workspace_bytes(C.byref(linear8()), None) == B.ERR_INVALID_ARG


def test_python_refusals_without_a_gpu():
    x = torch.zeros(2, 8)
    for call in (lambda: tr.dropout(x, 0.1, 0), lambda: tr.pack_rows8(x), lambda: tr.rms_norm(x, torch.ones(8)), lambda: tr.rms_norm_grad(x, x, torch.ones(8), torch.ones(2))):
        with pytest.raises(ValueError):
            call()
