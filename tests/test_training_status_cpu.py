"""training.status() asks the device it is given; "cuda" is the current one."""
import torch

from paper_2506_17974_b200 import training as tr


def test_status_of_the_current_device(monkeypatch):
    monkeypatch.setattr(tr, "_status", {0: torch.tensor([0]), 1: torch.tensor([16])})
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    assert tr.status("cuda") == 16 and tr.status("cuda:1") == 16 and tr.status(1) == 16
    assert tr.status() == 0 and tr.status("cuda:0") == 0 and tr.status("cuda:2") == 0
