"""The norm forward and then backward, with the rstd that the forward call supplies, on rows whose squares and their sum fp32 has; and what it
gives past that."""
import numpy as np
import pytest
import torch

import rows_oracle as ro
import test_gpu_training_rows as base

pytestmark = pytest.mark.gpu
tr, U, f64 = base.tr, base.U, base.f64


def check(x, gamma, eps, res=None, p=0.0):
    rows, cols = x.shape
    dtype = x.dtype
    r = tr.rms_norm(x, gamma, eps, res, p, 3, 9, save_h8=True)
    h = f64(r.h)
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    tol = base.terms(cols) / 2 * U + 4 * U                 # half the sum's error; the mean, + eps, the root, the reciprocal
    assert (np.abs(f64(r.rstd) - rstd) <= tol * rstd).all()
    y = h * rstd[:, None] * f64(gamma)
    base.near(r.y, y, dtype, (tol + 2 * U) * np.abs(y))
    # a dy as small as keeps the gradient, which is divided by the row's size, of size 0.01
    dy = (base.matrix(rows, cols, torch.float32, 12) * (0.01 / float(rstd.max()))).to(dtype)
    for kept in (r.h, r.h8):
        hv = f64(tr.unpack8(kept, torch.float32)) if isinstance(kept, tr.Packed8) else h
        dx, _, dgamma = tr.rms_norm_grad(dy, kept, gamma, r.rstd)
        d, dg = ro.rms_grad(f64(dy), hv, f64(gamma), f64(r.rstd))
        xh, u = np.abs(hv * f64(r.rstd)[:, None]), np.abs(f64(dy) * f64(gamma))
        slack = U * (f64(r.rstd)[:, None] * (3 * u + xh * (base.terms(cols) + 6) * (u * xh).mean(1, keepdims=True)) + 2 * np.abs(d))
        base.near(dx, d, dtype, slack)
        base.near(dgamma, dg, torch.float32, U * (rows + 4) * (np.abs(f64(dy)) * xh).sum(0))


@pytest.mark.parametrize("size,eps", [(1e16, 0.0), (1e16, 1e30), (1e-16, 0.0), (1e-16, 1e-30), (1e-30, 1e-6)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [3, 40, 250, 1024, 1100, 4099, 9000, 16400, 35000])
def test_forward_then_backward(cols, dtype, size, eps):
    """1e16: 35000 squares of up to 25e32 add up to 9e37 at most.  1e-16: squares of 1e-32, of which 2^-150, the smallest rounding, is 2^-43."""
    gamma = base.matrix(1, cols, torch.float32, 6)[0] * 0.2 + 1
    for pad, shift in ((0, 0), (3, 1)):
        check(base.matrix(5, cols, dtype, cols, pad, shift) * size, gamma, eps)
    check(base.matrix(5, cols, dtype, cols) * size, gamma, eps, base.matrix(5, cols, dtype, 8) * size, 0.1)


@pytest.mark.parametrize("cols", [40, 3000, 30000])
def test_past_the_range(cols):
    """Squares that add up past the range give rstd 0, y 0 and no gradient but the skip's; squares that vanish, without eps, rstd infinity."""
    x = torch.full((3, cols), 1e20, device="cuda")
    x[1], x[2] = 1e-25, 0.0
    gamma, dy, skip = torch.ones(cols, device="cuda"), torch.ones(3, cols, device="cuda"), base.matrix(3, cols, torch.float32, 1)
    r = tr.rms_norm(x, gamma, 0.0)
    assert r.rstd[0] == 0 and (r.y[0] == 0).all() and (r.rstd[1:] == float("inf")).all()
    dx, _, dgamma = tr.rms_norm_grad(dy[:1], x[:1], gamma, r.rstd[:1], skip[:1])
    assert dx.equal(skip[:1]) and (dgamma == 0).all()
    r = tr.rms_norm(x, gamma, 1e-6)
    assert ((r.rstd[1:] - 1000).abs() < 1e-3).all() and (r.y[2] == 0).all()
