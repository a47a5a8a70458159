"""Tensors given as `out` are written in place: autograd has to learn of it, and the result has to be there."""
import pytest
import torch

from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


def test_backward_sees_that_a_saved_tensor_was_overwritten():
    x, w = randn(32, 64, seed=1, dtype=BF), randn(64, 64, seed=2, dtype=BF)
    a = randn(32, 64, seed=3, dtype=BF).requires_grad_(True)
    h = a * 2
    loss = (h * h).sum()
    with torch.no_grad():
        tr.linear(x, w, residual=h, out=h)
    with pytest.raises(RuntimeError, match="in-?place"):
        loss.backward()


def test_every_out_counts_as_a_write():
    x, w, dz = randn(32, 64, seed=1, dtype=BF), randn(48, 64, seed=2, dtype=BF), randn(32, 48, seed=3, dtype=BF)
    p = tr.pack8(x)
    calls = [(lambda out: tr.linear(x, w, out=out), torch.zeros(32, 48, dtype=BF, device=DEV)),
             (lambda out: tr.linear_grad_input(dz, w, out=out), torch.zeros(32, 64, dtype=BF, device=DEV)),
             (lambda out: tr.linear_grad_weight(dz, x, out=out), torch.zeros(48, 64, device=DEV)),
             (lambda out: tr.linear_grad_weight(dz, p, out=out, accumulate=True), torch.zeros(48, 64, device=DEV)),
             (lambda out: tr.act_grad(x, p, "gelu", out=out), torch.zeros(32, 64, dtype=BF, device=DEV)),
             (lambda out: tr.unpack8(p, BF, out=out), torch.zeros(32, 64, dtype=BF, device=DEV))]
    for call, out in calls:
        view, before = out[:, :], out._version
        call(view)
        assert out._version > before and float(out.abs().max()) > 0
    before = p.codes._version, p.exps._version
    tr.pack8(x, out=p)
    assert p.codes._version > before[0] and p.exps._version > before[1]


def test_out_under_inference_mode():
    with torch.inference_mode():
        x, w = randn(32, 64, seed=1, dtype=BF), randn(64, 64, seed=2, dtype=BF)
        out = torch.empty(32, 64, dtype=BF, device=DEV)
        assert torch.equal(tr.linear(x, w, out=out).y, tr.linear(x, w).y)


@pytest.mark.parametrize("bias_grad", [False, True])
@pytest.mark.parametrize("cols", [64, 67])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_act_grad_without_an_activation_fills_out(bias_grad, cols, dtype):
    dy = randn(33, cols, seed=1, dtype=dtype)
    out = torch.zeros_like(dy)
    dz, db = tr.act_grad(dy, None, "none", bias_grad=bias_grad, out=out)
    assert dz.data_ptr() == out.data_ptr() and torch.equal(out, dy)
    assert (db is None) == (not bias_grad)
    if bias_grad:
        assert torch.equal(db, tr.act_grad(dy, None, "none")[1])
    with pytest.raises(ValueError):
        tr.act_grad(dy, None, "none", out=torch.zeros(33, cols + 1, dtype=dtype, device=DEV))
