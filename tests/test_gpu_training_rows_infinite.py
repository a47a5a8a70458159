"""Products of rows of codes whose sums leave fp32's range or are NaN, through every activation."""
import pytest
import torch

pytestmark = pytest.mark.gpu
tr = pytest.importorskip("paper_2506_17974_b200.training")
ACTS = ["none", "relu", "gelu", "silu"]


@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("rows,cin", [(1, 64), (2, 64), (3, 64), (40, 64), (600, 64), (1, 16384), (40, 16384), (100, 131071)])
def test_infinite_sums_through_every_activation(rows, cin, copies):
    """plus infinity passes; z cdf(z) and z logistic(z) of minus infinity are infinity times 0, as in products of 16 bits and in PyTorch."""
    w = torch.ones(300, cin, dtype=torch.int8, device="cuda")
    w[::2] = -1
    w8 = tr.Rows8(w, torch.full((300,), 1e30, device="cuda"))
    x8 = tr.Rows8(torch.ones(rows, cin, dtype=torch.int8, device="cuda"), torch.full((rows,), 1e30, device="cuda"))
    for act in ACTS:
        y = tr.linear_rows8(x8, w8, act=act, save_z8=copies).y
        assert (y[:, 1::2] == float("inf")).all(), act
        down = y[:, ::2]
        assert {"none": down == -float("inf"), "relu": down == 0, "gelu": torch.isnan(down), "silu": torch.isnan(down)}[act].all(), act
    z = torch.full((rows, 64), 1.0, device="cuda", dtype=torch.bfloat16)
    half = tr.linear(z, torch.full((8, 64), -3e38, device="cuda", dtype=torch.bfloat16), act="gelu").y
    assert torch.isnan(half).all()


def test_nan_sums_stay():
    x8 = tr.Rows8(torch.ones(3, 64, dtype=torch.int8, device="cuda"), torch.full((3,), float("nan"), device="cuda"))
    w8 = tr.pack_rows8(torch.ones(40, 64, device="cuda"))
    for act in ACTS:
        for n in (1, 3):
            assert torch.isnan(tr.linear_rows8(tr.Rows8(x8.codes[:n], x8.scales[:n]), w8, act=act).y).all()
