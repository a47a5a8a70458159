"""Matrices of nearly 2^31 columns: the number of their groups is counted without overflow.  Refused on the host; nothing is read."""
import ctypes as C

import pytest

import test_training_cpu as host
from paper_2506_17974_b200 import binding as B

lib = host.lib
I32, I64, PTR, SIZE = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t


@pytest.mark.parametrize("cols", [(1 << 31) - 1, (1 << 31) - 31])
def test_too_few_exponents_are_refused(lib, cols):
    few = host.packed(ld_codes=cols, ld_exps=(1 << 26) - 1)              # 2^26 groups
    at, ld = PTR(host.AT), I64(cols)
    assert lib.lqsgd_pack8(at, ld, I32(host.BF16), I64(1), I32(cols), C.byref(few), None) == B.ERR_INVALID_ARG
    assert lib.lqsgd_unpack8(C.byref(few), I64(1), I32(cols), at, ld, I32(host.BF16), None) == B.ERR_INVALID_ARG
    assert lib.lqsgd_act_grad(at, ld, C.byref(few), I32(1), I32(host.BF16), I64(1), I32(cols), at, ld, None, None, SIZE(0), None) == B.ERR_INVALID_ARG
