"""Sums over many inputs: a layer's output and the gradient of its input are as precise whatever the length of the sum.

The outputs have 16 bits, too few to show it.  So the residual takes the exact result's float16 rounding away again: what is left, at most
2^-12 of the result, is rounded to float16 by at most 2^-11 of itself, and shows the sum to 2^-23."""
import pytest
import torch

import test_gpu_training as base
from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def error(product, exact):
    """Relative 2-norm of the sum's error; product(residual) is the call."""
    near = exact.half()
    got = near.double() + product(-near).double()
    return ((got - exact).norm() / exact.norm()).item()


# An accumulator of the tensor core takes at most 2048 terms in 128 steps.  Each cuts off half a unit on average; a unit is 0.72 x 2^-23 of
# a value on average, and the partial sums are two thirds of the final one on average: 128 x 2^-24 x 0.72 x 2 / 3 < 64 x 2^-24.
# 2^-23 for the residual's way of showing it.
BOUND = 64 * 2.0 ** -24 + 2.0 ** -23


@pytest.mark.parametrize("long", [1024, 4096, 16384, 65536])
@pytest.mark.parametrize("rows,out", [(2304, 2304), (1000, 520), (7, 4096), (130, 128)])
def test_long_sums(rows, out, long):
    g = torch.Generator(DEV).manual_seed(long)
    a, b = (torch.randn(n, long, generator=g, device=DEV).half() for n in (rows, out))
    exact = a.double() @ b.double().t()
    assert error(lambda r: tr.linear(a, b, residual=r).y, exact) <= BOUND
    assert error(lambda r: tr.linear_grad_input(a, b.t().contiguous(), residual=r), exact) <= BOUND


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cin,cout", [(4100, 2500, 4100), (4101, 2504, 4104), (4099, 3401, 4097), (128, 1500, 9000), (127, 1502, 9003)])
def test_everything_behind_several_accumulators(dtype, rows, cin, cout):
    """Bias, activation, residual and 8-bit copies of tiles that several accumulators summed, ragged and aligned, pairs and single SMs."""
    base.test_linear(dtype, rows, cin, cout)
    base.test_linear_grad_input(dtype, rows, cout, cin)
