"""The example's pre-norm network: it runs, repeats, and its gradients are those of the same network in 64 bits."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_residual.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_residual", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_prenorm_network_trains(example):
    """Every step gives a finite loss; the same seed the same losses, bit for bit."""
    first, second = (example.train(steps=4, workers=2, seed=5, prenorm=True, dropout=0.1)[0] for _ in range(2))
    assert first == second and all(0 < v < 20 for v in first)


def test_prenorm_gradients(example):
    """Against the network in 64 bits (no dropout: masks are tested with the operator).  What rounds on the way: activations to bfloat16, kept
    ones to 8 bits, the products' operands to codes.  Each is off by at most 1/254 of a row's or group's largest value, 0.02 of the norm where that
    is 5 times the root mean square; 2 blocks of 6 such roundings, independent of one another, and back: below 0.02 sqrt(24) = 0.1; twice
    that for the gradients' own roundings."""
    net = example.PreNormNet(64, 2, 8, "cuda:0", seed=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    images, label = torch.randn(16, 3, 8, 8, generator=g, device="cuda"), torch.randint(10, (16,), generator=g, device="cuda")
    loss = F.cross_entropy(net.forward(images.bfloat16()).float(), label)
    grads = torch.autograd.grad(loss, net.weights)
    w = [t.detach().double().requires_grad_(True) for t in net.weights]
    x = F.unfold(images.bfloat16().double(), 3, padding=1).transpose(1, 2).reshape(-1, 27)
    norm = lambda h, gamma: h * gamma / (h.square().mean(1, keepdim=True) + 1e-6).sqrt()           # noqa: E731
    h = x @ w[0].t() + w[1]
    for k in range(2):
        gamma, w1, b1, w2, b2 = w[2 + 5 * k:7 + 5 * k]
        h = h + F.gelu(norm(h, gamma) @ w1.t() + b1) @ w2.t() + b2
    pooled = norm(h, w[12]).view(16, 64, -1).mean(1)
    want = torch.autograd.grad(F.cross_entropy(pooled @ w[13].t() + w[14], label), w)
    for a, b in zip(grads, want):
        assert (a.double() - b).norm() < 0.2 * b.norm()
