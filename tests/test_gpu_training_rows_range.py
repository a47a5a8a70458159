"""Rows of signed codes of a norm's output at the ends of fp32's range: where products h gamma are 0 or have a few digits left and rstd carries
them up, codes stay within half a step of y; where they pass the range the row counts as not finite."""
import numpy as np
import pytest
import torch

import test_gpu_training_rows as base

pytestmark = pytest.mark.gpu
tr, U, f64 = base.tr, base.U, base.f64


def check(x, gamma, eps, res=None, p=0.0):
    rows, cols = x.shape
    r = tr.rms_norm(x, gamma, eps, res, p, 3, 9, save_rows8=True)
    h = f64(r.h)
    rstd = 1 / np.sqrt((h * h).mean(1) + eps) if eps or (h != 0).any(1).all() else None
    y = h * rstd[:, None] * f64(gamma)
    tol = base.terms(cols) / 2 * U + 6 * U                    # rstd's, and two products
    top, scales = np.abs(y).max(1), f64(r.rows8.scales)
    least, most = (np.maximum(t / 127, 2.0 ** -120) for t in (top, top + 1.5 * 2.0 ** -148 * rstd))     # the product's rounding, and what is added
    assert (scales >= least * (1 - tol - 2 * U)).all() and (scales <= most * (1 + tol + 3 * U)).all()
    back = f64(r.rows8.codes) * scales[:, None]
    assert (np.abs(back - y) <= scales[:, None] / 2 + (2 * tol + 4 * U) * np.abs(y)).all()
    alone = tr.rms_norm(x, gamma, eps, res, p, 3, 9, want_y=False, save_rows8=True)
    assert alone.rows8.codes.equal(r.rows8.codes) and alone.rows8.scales.equal(r.rows8.scales)


# size of h, of gamma, eps
@pytest.mark.parametrize("size,weight,eps", [(1e-15, 1e-28, 0.0), (1e-15, 1e-30, 0.0), (1e-15, 1e-32, 0.0), (1e-17, 1e-27, 1e-34), (1e-15, 1e-20, 0.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [3, 40, 250, 1024, 1100, 4099, 9000, 16400, 35000])
def test_products_with_few_digits(cols, dtype, size, weight, eps):
    gamma = base.matrix(1, cols, torch.float32, 6)[0] * (0.2 * weight) + weight
    for pad, shift in ((0, 0), (3, 1)):
        check(base.matrix(5, cols, dtype, cols, pad, shift) * size, gamma, eps)
    check(base.matrix(5, cols, dtype, cols) * size, gamma, eps, base.matrix(5, cols, dtype, 8) * size, 0.1)


@pytest.mark.parametrize("cols", [33, 3000, 30000])
def test_products_past_the_range(cols):
    x = base.matrix(4, cols, torch.float32, 2)
    x[1] *= 1e-20
    gamma = torch.full((cols,), 1e30, device="cuda")
    r = tr.rms_norm(x * 1e12, gamma, save_rows8=True)
    assert torch.isfinite(r.y).all()
    assert (torch.isnan(r.rows8.scales) == torch.tensor([True, False, True, True], device="cuda")).all()
    assert (r.rows8.codes[[0, 2, 3]] == 0).all() and r.rows8.codes[1].abs().max() == 127


def test_rows_that_are_not_finite_are_not_here():
    for cols in (40, 3000, 30000):
        x = torch.ones(3, cols, device="cuda")
        x[0, 1], x[1, 2] = float("inf"), float("nan")
        for gamma in (1e-44, 1.0, 1e30):
            r = tr.rms_norm(x, torch.full((cols,), gamma, device="cuda"), save_rows8=True)
            assert torch.isnan(r.rows8.scales[:2]).all() and (r.rows8.codes[:2] == 0).all() and torch.isfinite(r.rows8.scales[2])
        weights = torch.ones(cols, device="cuda")
        weights[5] = float("inf")
        r = tr.rms_norm(x, weights, save_rows8=True)
        assert torch.isnan(r.rows8.scales).all() and (r.rows8.codes == 0).all()
