"""The differentiable layers can be differentiated once: a loss with a gradient penalty raises instead of losing the penalty's part."""
import pytest
import torch

from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


def linear_inputs():
    return randn(32, 64, seed=1, dtype=BF).requires_grad_(True), randn(64, 64, seed=2).mul_(0.1).requires_grad_(True), torch.zeros(64, device=DEV, requires_grad=True)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("skip", [False, True])
def test_second_derivative_of_a_linear_layer_is_refused(act, skip):
    x, w, b = linear_inputs()
    y = tr.linear_layer(x, w, b, act=act, residual=x if skip else None)
    loss = y.float().pow(2).sum()
    gx, gw = torch.autograd.grad(loss, [x, w], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + gx.float().pow(2).sum() + gw.pow(2).sum()).backward()


def test_second_derivative_of_a_norm_layer_is_refused():
    x = randn(2, 30, 32, seed=1, dtype=BF).requires_grad_(True)
    g, b = torch.ones(32, device=DEV, requires_grad=True), torch.zeros(32, device=DEV, requires_grad=True)
    y = tr.norm_layer(x, g, b, 4, act="silu")
    loss = y.float().pow(2).sum()
    gx, gg = torch.autograd.grad(loss, [x, g], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + gx.float().pow(2).sum() + gg.pow(2).sum()).backward()
