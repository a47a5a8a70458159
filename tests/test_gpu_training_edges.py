"""Training operators at sizes where a kernel changes its way: rows aligned to 16 but not to 32 bytes in every epilogue, sums longer
than one accumulator takes, pixels of one or two 8-channel pieces, norms too large to stay on the chip.  The checks and their
bounds are those of the operators' own tests."""
import pytest
import torch

import test_gpu_training as base
from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
randn = base.randn


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,cin,cout", [(2300, 64, 2056), (2301, 64, 2056), (2302, 64, 2056), (2300, 70, 2049), (300, 8, 1000), (301, 8, 1000),
                                            (302, 8, 1000), (130, 520, 24), (131, 520, 24), (132, 520, 24)])
def test_linear_rows_of_every_alignment(dtype, rows, cin, cout):
    base.test_linear(dtype, rows, cin, cout)
    base.test_linear_grad_input(dtype, rows, cout, cin)


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("rows,cin,cout", [(1024, 2304, 2304), (1025, 2308, 2304), (2100, 2310, 2300), (3200, 2304, 2310), (1089, 130, 4700)])
def test_weight_gradient_of_several_accumulators(packed, rows, cin, cout):
    base.test_linear_grad_weight(BF, packed, rows, cin, cout)


@pytest.mark.parametrize("rows,cin,cout", [(16384, 2304, 2304), (16384, 512, 256), (65536, 64, 128)])
def test_weight_gradient_keeps_its_precision(rows, cin, cout):
    """However many rows, an accumulator takes 1024 of them: 64 steps, each of which cuts off at most one unit (2^-23), half of it
    on average, of a sum that is below its final size."""
    dz, x = randn(rows, cout, seed=1, dtype=BF), randn(rows, cin, seed=2, dtype=BF)
    want = dz.double().t() @ x.double()
    got = tr.linear_grad_weight(dz, x).double()
    assert ((got - want).norm() / want.norm()).item() <= 64 * 2.0 ** -24


@pytest.mark.parametrize("cin", [2308, 2310])
def test_weight_gradient_adds_to_rows_of_any_alignment(cin):
    dz, x = randn(1500, 2304, seed=1, dtype=BF), randn(1500, cin, seed=2, dtype=BF)
    start = randn(2304, cin, seed=3)
    out = start.clone()
    tr.linear_grad_weight(dz, x, out=out, accumulate=True)
    once = tr.linear_grad_weight(dz, x)
    assert torch.equal(out, start + once)


SMALL = [(40, 700, 8, 1), (3, 2000, 8, 8), (5, 333, 16, 4), (4, 100, 5, 1), (3, 2500, 4, 2), (170, 300, 12, 3), (2, 77, 1, 1), (600, 33, 5, 5),
         (9, 1300, 24, 3)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,hw,c,groups", SMALL + [(33, 3560, 192, 8)])
def test_norm_of_few_channels(dtype, n, hw, c, groups):
    base.test_group_norm(dtype, n, hw, c, groups)


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("n,hw,c,groups", SMALL)
def test_norm_gradient_of_few_channels(packed, n, hw, c, groups):
    base.test_group_norm_grad(BF, packed, n, hw, c, groups)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("c", [5, 8])
def test_norm_keeps_what_is_not_finite_in_its_group(c, bad):
    x = randn(3, 600, c, seed=1)
    gamma, beta = randn(c, seed=4) + 1, randn(c, seed=5)
    clean = tr.group_norm(x, c, gamma, beta)
    x[1, 7, 3] = bad
    dirty = tr.group_norm(x, c, gamma, beta)
    hit = torch.zeros(3, c, dtype=torch.bool, device="cuda")
    hit[1, 3] = True
    assert torch.isnan(dirty.y.transpose(1, 2)[hit]).all() and torch.isnan(dirty.rstd[hit]).all()
    assert torch.equal(dirty.y.transpose(1, 2)[~hit], clean.y.transpose(1, 2)[~hit])
