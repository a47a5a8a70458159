"""Group norm over the longest samples it takes: 2^31 - 4096 pixels of one channel, whose last block of pixels ends past 2^31."""
import pytest
import torch

from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HW = 2 ** 31 - 4096
TAIL = 2_000_000                                             # more than a block of pixels (1,813,760 of them)
# A thread adds up to 7085 values in a row, then 256 threads and 1184 blocks meet; every addition rounds by 2^-24 of the sum of magnitudes.
ADDS = (7085 + 256 + 1184 + 64) * 2.0 ** -24


def sample():
    """Zeros, and at the end 3 and 5 in turn."""
    x = torch.zeros(1, HW, 1, dtype=torch.bfloat16, device=DEV)
    x[0, -TAIL::2, 0] = 3.0
    x[0, -TAIL + 1::2, 0] = 5.0
    mean = 4.0 * TAIL / HW
    rstd = (17.0 * TAIL / HW - mean * mean + 1e-5) ** -0.5
    return x, mean, rstd


def test_forward():
    x, mean, rstd = sample()
    gamma, beta = torch.full((1,), 2.0, device=DEV), torch.full((1,), 0.5, device=DEV)
    r = tr.group_norm(x, 1, gamma, beta)
    assert abs(r.mean.item() - mean) <= 2 * ADDS * mean
    assert abs(r.rstd.item() - rstd) <= 4 * ADDS * rstd
    got, want = r.y[0, -TAIL:, 0].double(), (x[0, -TAIL:, 0].double() - mean) * rstd * 2 + 0.5
    # mean and rstd as above, and the rounding to bfloat16
    assert ((got - want).abs() <= want.abs() * (2.0 ** -8 + 8 * ADDS) + 2 * ADDS).all()
    middle = r.y[0, 1 << 30:(1 << 30) + TAIL, 0].double()
    assert ((middle - (0.5 - mean * rstd * 2)).abs() <= 2.0 ** -8 + 8 * ADDS).all()


def test_backward():
    x, mean, rstd = sample()
    dy = torch.zeros_like(x)
    dy[0, -TAIL:, 0] = 1.0
    gamma, beta = torch.full((1,), 2.0, device=DEV), torch.full((1,), 0.5, device=DEV)
    m, s = (torch.full((1, 1), v, device=DEV) for v in (mean, rstd))
    dx, dgamma, dbeta = tr.group_norm_grad(dy, x, 1, gamma, beta, m, s)
    sums = TAIL * 1.0, TAIL * (4 - mean) * rstd                # of dh, of dh xh
    assert abs(dbeta.item() - sums[0]) <= 2 * ADDS * sums[0]
    assert abs(dgamma.item() - sums[1]) <= 2 * ADDS * sums[1]
    xh = (x[0, -TAIL:, 0].double() - mean) * rstd
    want = rstd * (2.0 - 2 * sums[0] / HW - xh * 2 * sums[1] / HW)
    # the difference's terms are 2, at most 0.002 and at most 2.2
    assert ((dx[0, -TAIL:, 0].double() - want).abs() <= want.abs() * 2.0 ** -8 + rstd * 4.3 * 4 * ADDS).all()
