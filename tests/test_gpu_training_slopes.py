"""Slopes of GELU and SiLU in their negative tails, where they are small and 1 minus their mirror image has lost its digits."""
import pytest
import torch

import test_gpu_training as base
from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def every_code(rows):
    """Rows of the 256 codes, steps 2^-3 (up to 15.9 in magnitude), 2^-5 and 2^-8 in turn."""
    exps = torch.tensor([123, 121, 118], dtype=torch.uint8, device=DEV).repeat(rows)[:rows, None].repeat(1, 8).contiguous()
    codes = torch.arange(256, dtype=torch.uint8, device=DEV)[None].repeat(rows, 1).contiguous()
    return tr.Packed8(codes, exps)


# Relative error of the slope below z = -2 (past its zeros at -0.75 and -1.28), in units of 2^-24: the argument of the exponential is
# rounded three times, which moves the exponential by 1.5 z (silu, z to -16: 24) or 1.5 z^2 / 2 (gelu, z to -5.25: 21); exp2 and
# the reciprocal add 4 and 2, the polynomial of the normal tail 27 (1.6e-6); sums and products another 4.  Sums whose terms cancel
# enlarge it by at most 1.6 (gelu at -2).  Together below 100 units, under 2^-17.
BOUND = 2.0 ** -17
LOWEST = {"silu": -16.0, "gelu": -5.25}


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("rows", [6, 600])
def test_negative_tails_keep_their_digits(act, rows):
    p = every_code(rows)
    z = tr.unpack8(p, torch.float32).double()
    dz, _ = tr.act_grad(torch.ones(rows, 256, device=DEV), p, act)
    tail = (z <= -2) & (z >= LOWEST[act])
    want = base.slope64(z[tail], act)
    assert ((dz.double()[tail] - want).abs() <= BOUND * want.abs()).all()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_slope_does_not_depend_on_the_number_of_rows(act, dtype):
    dy = base.randn(600, 256, seed=1, dtype=dtype)
    p = every_code(600)
    many, _ = tr.act_grad(dy, p, act)
    few, _ = tr.act_grad(dy[:6], tr.Packed8(p.codes[:6], p.exps[:6]), act)
    assert torch.equal(many[:6], few)
