"""Differentiable layers given tensors whose rows are one row (stride 0), as sums over rows and expanded inputs make them."""
import pytest
import torch

from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def parameters(c, out):
    g = torch.Generator(DEV).manual_seed(1)
    return [(torch.randn(out, c, generator=g, device=DEV) / c ** 0.5).requires_grad_(True), torch.zeros(out, device=DEV, requires_grad=True)]


@pytest.mark.parametrize("act", ["none", "gelu"])
def test_linear_layer_with_a_gradient_shared_by_all_rows(act):
    g = torch.Generator(DEV).manual_seed(2)
    x, v = (torch.randn(n, 40, generator=g, device=DEV).bfloat16() for n in (64, 1))
    w, b = parameters(40, 40)
    got = torch.autograd.grad((tr.linear_layer(x, w, b, act=act).sum(0, keepdim=True) * v).sum(), [w, b])
    want = torch.autograd.grad(tr.linear_layer(x, w, b, act=act), [w, b], v.repeat(64, 1))
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_layers_with_expanded_inputs():
    g = torch.Generator(DEV).manual_seed(3)
    row, res = (torch.randn(1, 48, generator=g, device=DEV).bfloat16().requires_grad_(True) for _ in range(2))
    w, b = parameters(48, 48)
    up = torch.randn(20, 48, generator=g, device=DEV).bfloat16()
    ga, be = torch.ones(48, device=DEV), torch.zeros(48, device=DEV)

    def run(x, r):
        h = tr.norm_layer(x.view(1, 20, 48) if x.is_contiguous() else x[None], ga, be, 4, act="silu")
        return tr.linear_layer(x, w, b, residual=r) + h[0]
    got = run(row.expand(20, 48), res.expand(20, 48))
    want = run(row.repeat(20, 1), res.repeat(20, 1))
    assert torch.equal(got, want)
    for p, q in zip(torch.autograd.grad(got, [w, b, row, res], up), torch.autograd.grad(want, [w, b, row, res], up)):
        assert torch.allclose(p.float(), q.float(), rtol=2 ** -7, atol=2 ** -7 * q.abs().max().item())
