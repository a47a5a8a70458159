"""The differentiable layers keep what the wanted gradients need, and make nothing else."""
import pytest
import torch

from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.fixture
def made(monkeypatch):
    """Names of the 8-bit copies that calls make."""
    seen = []
    for name in ("pack8", "linear", "group_norm"):
        def spy(*a, _f=getattr(tr, name), _name=name, **k):
            seen.extend([_name] if _name == "pack8" else [what for what in ("save_z8", "save_x8", "save_y8") if k.get(what)])
            return _f(*a, **k)
        monkeypatch.setattr(tr, name, spy)
    return seen


def layer(wants, act="gelu"):
    """Inputs of a linear layer, of which those in `wants` ask for a gradient."""
    t = dict(x=randn(96, 64, seed=1, dtype=BF), weight=randn(48, 64, seed=2).mul_(0.1), bias=randn(48, seed=3), residual=randn(96, 48, seed=4, dtype=BF))
    return {k: v.requires_grad_(k in wants) for k, v in t.items()}


@pytest.mark.parametrize("act,wants,copies", [
    ("gelu", "x weight bias residual", ["save_z8", "pack8"]), ("none", "x weight bias residual", ["pack8"]), ("gelu", "x", ["save_z8"]),
    ("gelu", "bias", ["save_z8"]), ("gelu", "weight", ["save_z8", "pack8"]), ("none", "x bias", []), ("silu", "residual", []), ("gelu", "", [])])
def test_linear_layer_keeps_what_its_gradients_need(made, act, wants, copies):
    full, some = layer("x weight bias residual".split()), layer(wants.split())
    dy = randn(96, 48, seed=5, dtype=BF)
    want = tr.linear_layer(full["x"], full["weight"], full["bias"], act, full["residual"])
    want.backward(dy)
    del made[:]
    y = tr.linear_layer(some["x"], some["weight"], some["bias"], act, some["residual"])
    assert sorted(made) == sorted(copies)
    assert torch.equal(y, want) and y.requires_grad == bool(wants)
    if wants:
        y.backward(dy)
    for k in some:
        assert torch.equal(some[k].grad, full[k].grad) if k in wants.split() else some[k].grad is None


def test_layers_keep_nothing_without_recording(made):
    t = layer("x weight bias residual".split())
    g, b = torch.ones(64, device=DEV, requires_grad=True), torch.zeros(64, device=DEV, requires_grad=True)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            tr.linear_layer(t["x"], t["weight"], t["bias"], "gelu", t["residual"])
            tr.norm_layer(t["x"].view(2, 48, 64), g, b, 8, act="silu")
            assert made == []
            keep = []
            tr.norm_layer(t["x"].view(2, 48, 64), g, b, 8, act="silu", keep=keep)
            assert made == ["save_y8"] and keep[0].shape == (96, 64)
            del made[:]


@pytest.mark.parametrize("wants", ["x gamma beta", "x", "gamma", "beta"])
def test_norm_layer_with_some_gradients(made, wants):
    def inputs(names):
        t = dict(x=randn(2, 48, 64, seed=1, dtype=BF), gamma=randn(64, seed=2) + 1, beta=randn(64, seed=3))
        return {k: v.requires_grad_(k in names) for k, v in t.items()}
    full, some = inputs(["x", "gamma", "beta"]), inputs(wants.split())
    dy = randn(2, 48, 64, seed=5, dtype=BF)
    tr.norm_layer(full["x"], full["gamma"], full["beta"], 8, act="silu").backward(dy)
    tr.norm_layer(some["x"], some["gamma"], some["beta"], 8, act="silu").backward(dy)
    for k in some:
        assert torch.equal(some[k].grad, full[k].grad) if k in wants.split() else some[k].grad is None
