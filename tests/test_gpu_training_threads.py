"""Workspaces that calls keep belong to their host thread and go with it."""
import threading

import pytest
import torch

from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_thread_takes_its_workspaces_along():
    g = torch.Generator(DEV).manual_seed(1)
    dy, x = (torch.randn(4096, c, generator=g, device=DEV).bfloat16() for c in (512, 256))
    want = tr.act_grad(dy, None)[1], tr.linear_grad_weight(dy, x)
    torch.cuda.synchronize()
    results, held = [], []

    def work():
        results.append((tr.act_grad(dy, None)[1], tr.linear_grad_weight(dy, x)))
        torch.cuda.current_stream().synchronize()
        held.append(torch.cuda.memory_allocated())

    before = torch.cuda.memory_allocated()
    for _ in range(3):
        t = threading.Thread(target=work)
        t.start()
        t.join()
        got = results.pop()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        del got
        assert torch.cuda.memory_allocated() == before
    assert min(held) - before >= 1 << 20                       # a thread at work does keep one


def test_threads_on_one_stream_do_not_share_a_workspace():
    g = torch.Generator(DEV).manual_seed(2)
    dys = [torch.randn(20000 + 512 * i, 96, generator=g, device=DEV).bfloat16() for i in range(4)]
    want = [tr.act_grad(d, None)[1] for d in dys]
    bad = []

    def work(i):
        for _ in range(50):
            if not torch.equal(tr.act_grad(dys[i], None)[1], want[i]):
                bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
