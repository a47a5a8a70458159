"""Host-side checks of the training operators that need no GPU: struct layouts, refusals and workspace sizes of the C
entries.  Every refused call returns before it touches a device, so the addresses here are never read."""
import ctypes as C

import pytest

import __graft_entry__ as entry
from paper_2506_17974_b200 import binding as B
from paper_2506_17974_b200 import training as tr

I32, I64, PTR, SIZE = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t
BF16, F16, F32 = 0, 1, 2
AT = 0x7f0000000000                                             # an aligned address that nothing reads


class Packed8(C.Structure):
    _fields_ = [("codes", PTR), ("ld_codes", I64), ("exps", PTR), ("ld_exps", I64)]


class Linear(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", I32), ("act", I32), ("accumulate", I32), ("rows", I64), ("cin", I32), ("cout", I32),
                ("x", PTR), ("ld_x", I64), ("w", PTR), ("ld_w", I64), ("dz", PTR), ("ld_dz", I64), ("bias", PTR),
                ("residual", PTR), ("ld_residual", I64), ("out", PTR), ("ld_out", I64), ("x8", Packed8), ("z8", Packed8), ("y8", Packed8),
                ("status", PTR), ("workspace", PTR), ("workspace_bytes", SIZE)]


class Norm(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", I32), ("act", I32), ("groups", I32), ("n", I32), ("hw", I32), ("c", I32), ("eps", C.c_float),
                ("x", PTR), ("ld_x", I64), ("sample_x", I64), ("dy", PTR), ("ld_dy", I64), ("sample_dy", I64),
                ("out", PTR), ("ld_out", I64), ("sample_out", I64), ("gamma", PTR), ("beta", PTR), ("mean", PTR), ("rstd", PTR),
                ("dgamma", PTR), ("dbeta", PTR), ("x8", Packed8), ("y8", Packed8), ("workspace", PTR), ("workspace_bytes", SIZE)]


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return B.load_library()


def linear(**kw):
    a = Linear(C.sizeof(Linear), BF16, 0, 0, 64, 128, 96, AT, 128, AT, 128, AT, 96, 0, 0, 0, AT, 128)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def norm(**kw):
    a = Norm(C.sizeof(Norm), BF16, 0, 8, 2, 16, 64, 1e-5, AT, 64, 1024, AT, 64, 1024, AT, 64, 1024, AT, AT, AT, AT, AT, AT)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def packed(codes=AT, ld_codes=128, exps=AT, ld_exps=4):
    return Packed8(codes, ld_codes, exps, ld_exps)


def test_struct_sizes():
    assert C.sizeof(Packed8) == tr._PACKED8.size == 32
    assert C.sizeof(Linear) == tr._LINEAR.size
    assert C.sizeof(Norm) == tr._NORM.size


@pytest.mark.parametrize("change,code", [
    (dict(struct_size=8), B.ERR_INVALID_ARG), (dict(dtype=F32), B.ERR_INVALID_ARG), (dict(dtype=7), B.ERR_INVALID_ARG),
    (dict(act=4), B.ERR_INVALID_ARG), (dict(act=-1), B.ERR_INVALID_ARG), (dict(accumulate=2), B.ERR_INVALID_ARG),
    (dict(rows=-1), B.ERR_BAD_SHAPE), (dict(rows=1 << 31), B.ERR_BAD_SHAPE), (dict(cin=0), B.ERR_BAD_SHAPE),
    (dict(cout=0), B.ERR_BAD_SHAPE), (dict(cin=(1 << 24) + 1), B.ERR_BAD_SHAPE), (dict(cout=(1 << 24) + 1), B.ERR_BAD_SHAPE),
    (dict(out=0), B.ERR_INVALID_ARG), (dict(ld_out=95), B.ERR_INVALID_ARG), (dict(out=AT + 1), B.ERR_MISALIGNED),
    (dict(status=AT + 2), B.ERR_MISALIGNED)])
def test_linear_refusals(lib, change, code):
    for fn in (lib.lqsgd_linear_forward, lib.lqsgd_linear_grad_input, lib.lqsgd_linear_grad_weight):
        assert fn(C.byref(linear(**change)), None) == code, fn


@pytest.mark.parametrize("entry_,change,code", [
    ("forward", dict(x=0), B.ERR_INVALID_ARG), ("forward", dict(w=0), B.ERR_INVALID_ARG), ("forward", dict(ld_x=127), B.ERR_INVALID_ARG),
    ("forward", dict(ld_w=127), B.ERR_INVALID_ARG), ("forward", dict(x=AT + 1), B.ERR_MISALIGNED), ("forward", dict(bias=AT + 2), B.ERR_MISALIGNED),
    ("forward", dict(residual=AT, ld_residual=95), B.ERR_INVALID_ARG), ("forward", dict(residual=AT + 1, ld_residual=96), B.ERR_MISALIGNED),
    ("forward", dict(z8=packed(ld_codes=95)), B.ERR_INVALID_ARG), ("forward", dict(z8=packed(ld_exps=2)), B.ERR_INVALID_ARG),
    ("forward", dict(y8=packed(exps=0)), B.ERR_INVALID_ARG),
    ("grad_input", dict(dz=0), B.ERR_INVALID_ARG), ("grad_input", dict(ld_dz=95), B.ERR_INVALID_ARG), ("grad_input", dict(w=0), B.ERR_INVALID_ARG),
    ("grad_input", dict(dz=AT + 1), B.ERR_MISALIGNED), ("grad_input", dict(residual=AT, ld_residual=127), B.ERR_INVALID_ARG),
    ("grad_weight", dict(dz=0), B.ERR_INVALID_ARG), ("grad_weight", dict(x=0), B.ERR_INVALID_ARG), ("grad_weight", dict(ld_x=127), B.ERR_INVALID_ARG),
    ("grad_weight", dict(out=AT + 2), B.ERR_MISALIGNED), ("grad_weight", dict(x=0, x8=packed(ld_codes=127)), B.ERR_INVALID_ARG)])
def test_linear_operand_refusals(lib, entry_, change, code):
    assert getattr(lib, "lqsgd_linear_" + entry_)(C.byref(linear(**change)), None) == code


def test_linear_null_and_workspace(lib):
    need = SIZE(7)
    assert lib.lqsgd_linear_forward(None, None) == B.ERR_INVALID_ARG
    assert lib.lqsgd_linear_workspace_bytes(0, C.byref(linear()), None) == B.ERR_INVALID_ARG
    assert lib.lqsgd_linear_workspace_bytes(3, C.byref(linear()), C.byref(need)) == B.ERR_INVALID_ARG
    # a sum over many rows for one small tile is cut in pieces that meet in the workspace
    a = linear(rows=65536)
    assert lib.lqsgd_linear_workspace_bytes(2, C.byref(a), C.byref(need)) == 0
    assert need.value > 96 * 128 * 4
    assert lib.lqsgd_linear_grad_weight(C.byref(a), None) == B.ERR_WORKSPACE_TOO_SMALL
    a.workspace, a.workspace_bytes = AT, need.value - 1
    assert lib.lqsgd_linear_grad_weight(C.byref(a), None) == B.ERR_WORKSPACE_TOO_SMALL
    a.workspace, a.workspace_bytes = AT + 8, need.value
    assert lib.lqsgd_linear_grad_weight(C.byref(a), None) == B.ERR_MISALIGNED
    # the 8-bit operand of a weight gradient is decoded there: 16-bit values
    a = linear(x=0, x8=packed())
    assert lib.lqsgd_linear_workspace_bytes(2, C.byref(a), C.byref(need)) == 0 and need.value >= 64 * 128 * 2
    # rows that are not 16-byte aligned are copied there
    a = linear(x=AT + 2, ld_x=129)
    assert lib.lqsgd_linear_workspace_bytes(0, C.byref(a), C.byref(need)) == 0 and need.value >= 64 * 128 * 2
    assert lib.lqsgd_linear_workspace_bytes(0, C.byref(linear(rows=0)), C.byref(need)) == 0 and need.value == 0


def test_linear_without_rows_does_nothing(lib):
    for fn in (lib.lqsgd_linear_forward, lib.lqsgd_linear_grad_input):
        assert fn(C.byref(linear(rows=0, x=0, dz=0, out=0)), None) == 0
    assert lib.lqsgd_linear_grad_weight(C.byref(linear(rows=0, x=0, dz=0, accumulate=1)), None) == 0


def test_pack_refusals(lib):
    p = packed()
    ref = C.byref(p)
    for fn, swap in ((lib.lqsgd_pack8, False), (lib.lqsgd_unpack8, True)):
        def call(x=AT, ld=128, dtype=BF16, rows=4, cols=128, pk=ref):
            head = (pk, I64(rows), I32(cols), PTR(x), I64(ld), I32(dtype)) if swap else (PTR(x), I64(ld), I32(dtype), I64(rows), I32(cols), pk)
            return fn(*head, None)
        assert call(pk=None) == B.ERR_INVALID_ARG
        assert call(dtype=3) == B.ERR_INVALID_ARG
        assert call(rows=-1) == B.ERR_BAD_SHAPE and call(cols=0) == B.ERR_BAD_SHAPE and call(rows=(1 << 40) + 1) == B.ERR_BAD_SHAPE
        assert call(x=0) == B.ERR_INVALID_ARG and call(ld=127) == B.ERR_INVALID_ARG
        assert call(x=AT + 1) == B.ERR_MISALIGNED and call(x=AT + 2, dtype=F32) == B.ERR_MISALIGNED
        assert call(pk=C.byref(packed(codes=0))) == B.ERR_INVALID_ARG and call(pk=C.byref(packed(exps=0))) == B.ERR_INVALID_ARG
        assert call(pk=C.byref(packed(ld_codes=127))) == B.ERR_INVALID_ARG and call(pk=C.byref(packed(ld_exps=3))) == B.ERR_INVALID_ARG
        assert call(rows=0, x=0) == 0


def test_act_grad_refusals(lib):
    need = SIZE(0)

    def call(dy=AT, ld_dy=128, z8=packed(), act=2, dtype=BF16, rows=4096, cols=128, dz=AT, ld_dz=128, db=AT, ws=0, nbytes=0):
        return lib.lqsgd_act_grad(PTR(dy), I64(ld_dy), C.byref(z8) if z8 is not None else None, I32(act), I32(dtype), I64(rows), I32(cols),
                                  PTR(dz), I64(ld_dz), PTR(db), PTR(ws), SIZE(nbytes), None)
    assert call(act=4) == B.ERR_INVALID_ARG and call(dtype=3) == B.ERR_INVALID_ARG
    assert call(rows=-1) == B.ERR_BAD_SHAPE and call(cols=0) == B.ERR_BAD_SHAPE
    assert call(dz=0) == B.ERR_INVALID_ARG and call(dz=0, db=0, act=0) == B.ERR_INVALID_ARG
    assert call(dy=0) == B.ERR_INVALID_ARG and call(ld_dy=127) == B.ERR_INVALID_ARG and call(ld_dz=127) == B.ERR_INVALID_ARG
    assert call(z8=None) == B.ERR_INVALID_ARG and call(z8=packed(ld_codes=64)) == B.ERR_INVALID_ARG
    assert call(dy=AT + 1) == B.ERR_MISALIGNED and call(db=AT + 2) == B.ERR_MISALIGNED
    assert lib.lqsgd_act_grad_workspace_bytes(I64(4096), I32(128), None) == B.ERR_INVALID_ARG
    assert lib.lqsgd_act_grad_workspace_bytes(I64(4096), I32(0), C.byref(need)) == B.ERR_BAD_SHAPE
    assert lib.lqsgd_act_grad_workspace_bytes(I64(4096), I32(128), C.byref(need)) == 0 and need.value > 0
    assert call() == B.ERR_WORKSPACE_TOO_SMALL
    assert call(ws=AT + 8, nbytes=need.value) == B.ERR_MISALIGNED


@pytest.mark.parametrize("change,code", [
    (dict(struct_size=4), B.ERR_INVALID_ARG), (dict(dtype=3), B.ERR_INVALID_ARG), (dict(act=9), B.ERR_INVALID_ARG),
    (dict(n=-1), B.ERR_BAD_SHAPE), (dict(hw=0), B.ERR_BAD_SHAPE), (dict(c=0), B.ERR_BAD_SHAPE), (dict(groups=0), B.ERR_BAD_SHAPE),
    (dict(groups=7), B.ERR_BAD_SHAPE), (dict(c=65544, groups=8), B.ERR_BAD_SHAPE), (dict(out=0), B.ERR_INVALID_ARG),
    (dict(ld_out=63), B.ERR_INVALID_ARG), (dict(sample_out=1023), B.ERR_INVALID_ARG), (dict(out=AT + 1), B.ERR_MISALIGNED),
    (dict(gamma=0), B.ERR_INVALID_ARG), (dict(beta=0), B.ERR_INVALID_ARG), (dict(mean=0), B.ERR_INVALID_ARG), (dict(rstd=0), B.ERR_INVALID_ARG),
    (dict(gamma=AT + 2), B.ERR_MISALIGNED), (dict(rstd=AT + 1), B.ERR_MISALIGNED)])
def test_norm_refusals(lib, change, code):
    for fn in (lib.lqsgd_group_norm_forward, lib.lqsgd_group_norm_backward):
        assert fn(C.byref(norm(**change)), None) == code, fn


def test_norm_operand_refusals(lib):
    fwd, bwd = lib.lqsgd_group_norm_forward, lib.lqsgd_group_norm_backward
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert fwd(C.byref(norm(eps=eps)), None) == B.ERR_INVALID_ARG
    assert fwd(C.byref(norm(x=0)), None) == B.ERR_INVALID_ARG and fwd(C.byref(norm(ld_x=63)), None) == B.ERR_INVALID_ARG
    assert fwd(C.byref(norm(x8=packed(ld_codes=63))), None) == B.ERR_INVALID_ARG
    assert fwd(C.byref(norm(y8=packed(exps=0))), None) == B.ERR_INVALID_ARG
    assert bwd(C.byref(norm(dy=0)), None) == B.ERR_INVALID_ARG and bwd(C.byref(norm(x=0)), None) == B.ERR_INVALID_ARG
    assert bwd(C.byref(norm(dgamma=0)), None) == B.ERR_INVALID_ARG and bwd(C.byref(norm(dbeta=AT + 2)), None) == B.ERR_MISALIGNED
    assert bwd(C.byref(norm(x=0, x8=packed(ld_exps=1))), None) == B.ERR_INVALID_ARG
    need = SIZE(0)
    assert lib.lqsgd_group_norm_workspace_bytes(2, C.byref(norm()), C.byref(need)) == B.ERR_INVALID_ARG
    assert lib.lqsgd_group_norm_workspace_bytes(1, C.byref(norm()), None) == B.ERR_INVALID_ARG
    assert lib.lqsgd_group_norm_workspace_bytes(1, C.byref(norm()), C.byref(need)) == 0 and need.value > 0
    assert bwd(C.byref(norm()), None) == B.ERR_WORKSPACE_TOO_SMALL
    assert bwd(C.byref(norm(workspace=AT + 4, workspace_bytes=need.value)), None) == B.ERR_MISALIGNED
