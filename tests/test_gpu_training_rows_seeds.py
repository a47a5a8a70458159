"""A dropout's seed on the device in every kernel that drops: the mask and the results of the same whole numbers, bit for bit."""
import pytest
import torch

import test_gpu_training_rows as base

pytestmark = pytest.mark.gpu
tr = base.tr
# rows of a few lanes, of a warp, of a block, walked in steps; strips of dropout of every width
COLS = [5, 96, 300, 600, 1100, 4099, 8200, 9000, 16400, 25087]
SEEDS = [(77, 1000, 5), (2 ** 63 - 3, 2 ** 32 - 2, 9), (-5, 2 ** 62, 2 ** 32 - 1), (2 ** 33 + 1, -3, 2)]        # seed, what is added, offset: sums that carry


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_same_results(cols, dtype, pad, shift):
    rows = 3 if cols > 8000 else 21
    x, res = base.matrix(rows, cols, dtype, 1, pad, shift), base.matrix(rows, cols, dtype, 2, pad, shift)
    dy, gamma = base.matrix(rows, cols, dtype, 3, pad, shift), base.matrix(1, cols, torch.float32, 4)[0] + 1
    for key, add, offset in SEEDS:
        seed, total = torch.tensor([key, add], dtype=torch.int64, device="cuda"), (offset + add) % 2 ** 64
        for r in (None, res):
            assert tr.dropout(x, 0.3, seed, offset, residual=r).equal(tr.dropout(x, 0.3, key, total, residual=r))
        a, b = (tr.rms_norm(x, gamma, residual=res, p=0.3, seed=s, offset=o, save_h8=True, save_y8=True, save_rows8=True) for s, o in ((seed, offset), (key, total)))
        for s, t in ((a.y, b.y), (a.h, b.h), (a.rstd, b.rstd), (a.h8.codes, b.h8.codes), (a.y8.codes, b.y8.codes), (a.rows8.codes, b.rows8.codes)):
            assert s.equal(t)
        for h in (a.h, a.h8):
            got, want = (tr.rms_norm_grad(dy, h, gamma, a.rstd, res, 0.3, s, o) for s, o in ((seed, offset), (key, total)))
            assert all(s.equal(t) for s, t in zip(got, want))


@pytest.mark.parametrize("cols", [40, 1100, 16400])
def test_layers(cols):
    gamma = torch.ones(cols, device="cuda", requires_grad=True)
    x, res = (base.matrix(7, cols, torch.bfloat16, s).requires_grad_(True) for s in (1, 2))
    seed = torch.tensor([11, 2 ** 32 - 1], dtype=torch.int64, device="cuda")
    for layer in (lambda s, o: tr.add_rms_norm_layer(x, res, gamma, p=0.4, seed=s, offset=o), lambda s, o: (tr.dropout_layer(x, 0.4, s, o, residual=res),)):
        outs = [layer(s, o) for s, o in ((seed, 3), (11, 2 ** 32 + 2))]
        grads = [torch.autograd.grad([t for t in out], [x, res], [torch.ones_like(t) for t in out]) for out in outs]
        assert all(a.equal(b) for a, b in zip(*outs)) and all(a.equal(b) for a, b in zip(*grads))


def test_many_rows():
    """Blocks that take several rows each, forward and backward."""
    for rows, cols in ((5000, 40), (2500, 1030), (700, 4096), (300, 9000)):
        x, gamma = base.matrix(rows, cols, torch.bfloat16, 1), torch.ones(cols, device="cuda")
        seed = torch.tensor([5, 6], dtype=torch.int64, device="cuda")
        r = tr.rms_norm(x, gamma, p=0.2, seed=seed, offset=7)
        assert r.h.equal(tr.dropout(x, 0.2, 5, 13))
        got, want = (tr.rms_norm_grad(x, r.h, gamma, r.rstd, p=0.2, seed=s, offset=o) for s, o in ((seed, 7), (5, 13)))
        assert all(s.equal(t) for s, t in zip(got, want))
