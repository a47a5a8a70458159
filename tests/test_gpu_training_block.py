"""The pre-norm residual block in training: dropout, the residual's addition, RMS norm and products in 8 bits as differentiable layers,
together with the layers that were there, against the same steps in 64 bits.

Where a step rounds (to bfloat16, to 8 bits) the 64-bit form takes the rounded values that the layer itself kept or returned, so that
only the roundings inside a step count: see each tolerance."""
import numpy as np
import pytest
import torch

import rows_oracle as ro

pytestmark = pytest.mark.gpu
tr = pytest.importorskip("paper_2506_17974_b200.training")


def f64(t):
    return t.detach().double().cpu().numpy()


def leaf(*shape, seed, scale=1.0, dtype=torch.float32, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale + mean).to(dtype).cuda().requires_grad_(True)


def rel(got, want):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def test_dropout_layer():
    x, res = leaf(37, 100, seed=1, dtype=torch.bfloat16), leaf(37, 100, seed=2, dtype=torch.bfloat16)
    seed = torch.tensor([3, 0], device="cuda")
    for s in (3, seed):
        y = tr.dropout_layer(x, 0.4, s, 5, residual=res)
        assert y.equal(tr.dropout(x.detach(), 0.4, 3, 5, residual=res.detach()))
        dy = torch.randn_like(y)
        dx, dres = torch.autograd.grad(y, (x, res), dy)
        assert dx.equal(tr.dropout(dy, 0.4, 3, 5)) and dres.equal(dy)
    (dx,) = torch.autograd.grad(tr.dropout_layer(x, 0.4, 3, 5).sum(), x)                    # the gradient of a sum: expanded
    assert ((f64(dx) != 0) == ro.kept(37, 100, 0.4, 3, 5)).all()
    y = tr.dropout_layer(x, 0.4, seed, 5)
    seed += 1                                                                               # another mask by the time of the backward pass
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        torch.autograd.grad(y.float().sum(), x)


@pytest.mark.parametrize("rows,cols", [(9, 96), (33, 1000), (5, 4100)])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_add_rms_norm_layer(rows, cols, p):
    """Gradients of a scalar of both outputs, of either alone, and of none."""
    x, res, gamma = leaf(rows, cols, seed=1, dtype=torch.bfloat16), leaf(rows, cols, seed=2, dtype=torch.bfloat16), leaf(cols, seed=3, scale=0.2, mean=1.0)
    keep, rows8 = [], []
    y, h = tr.add_rms_norm_layer(x, res, gamma, 1e-6, p, 7, 8, keep, rows8)
    want = tr.rms_norm(x.detach(), gamma.detach(), residual=res.detach(), p=p, seed=7, offset=8, save_h8=True, save_rows8=True)
    assert y.equal(want.y) and h.equal(want.h) and rows8[0].codes.equal(want.rows8.codes) and keep[0].codes.equal(tr.pack8(want.y).codes)
    gy, gh = torch.randn_like(y), torch.randn_like(h)
    for a, b in ((gy, gh), (gy, None), (None, gh)):
        outs = [(t, g) for t, g in ((y, a), (h, b)) if g is not None]
        dx, dres, dgamma = torch.autograd.grad([t for t, _ in outs], (x, res, gamma), [g for _, g in outs], retain_graph=True, allow_unused=True)
        if a is None:
            assert dgamma is None and dres.equal(b) and dx.equal(tr.dropout(b, p, 7, 8) if p else b)
            continue
        wx, wres, wgamma = tr.rms_norm_grad(a, want.h8, gamma.detach(), want.rstd, b, p, 7, 8)
        assert dx.equal(wx) and dres.equal(wres) and dgamma.equal(wgamma)
    (dgamma,) = torch.autograd.grad(y, gamma, gy)
    assert dgamma.equal(tr.rms_norm_grad(gy, want.h8, gamma.detach(), want.rstd, None, p, 7, 8)[2])
    with torch.no_grad():
        y, h = tr.add_rms_norm_layer(x, res, gamma, 1e-6, p, 7, 8)
        assert not y.requires_grad and y.equal(want.y)


def test_rms_norm_layer_and_second_derivative():
    x, gamma = leaf(12, 64, seed=1, dtype=torch.float16), leaf(64, seed=3, scale=0.2, mean=1.0)
    y = tr.rms_norm_layer(x, gamma)
    dx, dgamma = torch.autograd.grad(y.sum(), (x, gamma), create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dx.float().sum(), x)
    want = tr.rms_norm_grad(torch.ones_like(y), tr.pack8(x.detach()), gamma.detach(), tr.rms_norm(x.detach(), gamma.detach()).rstd)
    assert dx.equal(want[0]) and dgamma.equal(want[2])
    y = tr.rms_norm_layer(x.t().contiguous().t(), gamma)                                    # rows that do not lie along memory
    assert torch.autograd.grad(y.sum(), gamma)[0].equal(dgamma)


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("given", [False, True])
def test_linear_rows8_layer(act, given):
    """Straight through the rounding: dz w, dz^T x of what was multiplied, dz's column sums, dz = dy act'(z) with z in 8 bits."""
    x, w, b, res = leaf(70, 130, seed=1, dtype=torch.bfloat16), leaf(50, 130, seed=2, scale=130 ** -0.5), leaf(50, seed=3), leaf(70, 50, seed=4, dtype=torch.bfloat16)
    x8, w8 = tr.pack_rows8(x.detach()), tr.pack_rows8(w.detach())
    y = tr.linear_rows8_layer(x, w, b, act, res, x8 if given else None, w8 if given else None)
    want = tr.linear_rows8(x8, w8, b.detach(), act, res.detach(), save_z8=True)
    assert y.equal(want.y)
    dy = torch.randn_like(y)
    dx, dw, db, dres = torch.autograd.grad(y, (x, w, b, res), dy)
    dz, wb = tr.act_grad(dy, want.z8, act)
    assert dres.equal(dy) and db.equal(wb)
    z = f64(dz)
    assert rel(dx, z @ f64(w.detach().bfloat16())) < 2.0 ** -8                              # one rounding to bfloat16
    assert rel(dw, z.T @ f64(tr.unpack_rows8(x8, torch.bfloat16))) < 3e-6                   # fp32 sums
    with pytest.raises(ValueError):
        tr.linear_rows8_layer(x.float(), w)


def block(x, h, weights, p, seed):
    """h + dropout(x), normed, through a feed-forward of two layers: the first in 8-bit rows, the second in 16 bits."""
    gamma, w1, b1, w2, b2 = weights
    rows8 = []
    y, h = tr.add_rms_norm_layer(x, h, gamma, p=p, seed=seed, offset=0, keep_rows8=rows8)
    a = tr.linear_rows8_layer(y, w1, b1, act="gelu", rows8=rows8[0])
    return tr.linear_layer(a, w2, b2), h, rows8[0]


@pytest.mark.parametrize("rows,c,hid,p", [(1, 64, 256, 0.0), (65, 96, 200, 0.2), (300, 520, 1000, 0.1)])
def test_block_in_training(rows, c, hid, p):
    """Forward and gradients of the whole block against 64 bits, the roundings of the path among them.

    Relative 2-norms, a rounding to bfloat16 at most 2^-8 of each value, to kept 8 bits or rows of codes at most 1/2 step of 1/127 (2^-7) of
    the group's or the row's largest, which is at most 5 times the values' root mean square: 5/254 = 0.02 of the norm.  The output passes rows of x
    and w1 in codes (0.02 each) and four roundings to bfloat16: below 0.06.  The gradients pass kept h, z and activations as well: three more
    times 0.02, below 0.12."""
    x, h0 = leaf(rows, c, seed=1, dtype=torch.bfloat16), leaf(rows, c, seed=2, dtype=torch.bfloat16)
    weights = [leaf(c, seed=3, scale=0.1, mean=1.0), leaf(hid, c, seed=4, scale=c ** -0.5), leaf(hid, seed=5, scale=0.1), leaf(c, hid, seed=6, scale=hid ** -0.5),
               leaf(c, seed=7, scale=0.1)]
    out, h, _ = block(x, h0, weights, p, 11)
    final = tr.dropout_layer(out, p, 11, 1, residual=h)
    dy = torch.randn_like(final)
    got = torch.autograd.grad(final, [x, h0] + weights, dy)

    d = [t.detach().double().requires_grad_(True) for t in [x, h0] + weights]
    mask = lambda off: torch.from_numpy(ro.kept(rows, c, p, 11, off)).cuda() * (65536 / (65536 - ro.threshold(p)))      # noqa: E731
    hd = d[1] + d[0] * mask(0)
    y = hd * d[2] / (hd.square().mean(1, keepdim=True) + 1e-6).sqrt()
    z = y @ d[3].t() + d[4]
    want = hd + (z * 0.5 * torch.erfc(-z / 2 ** 0.5) @ d[5].t() + d[6]) * mask(1)
    assert rel(final, f64(want)) < 0.06
    for name, g, w in zip(("x", "h", "gamma", "w1", "b1", "w2", "b2"), got, torch.autograd.grad(want, d, dy.double())):
        assert rel(g, f64(w)) < 0.12, name
    assert tr.status() == 0


def test_block_captured_as_a_step():
    """A step with its backward pass in a graph, the seed on the device: replays draw new masks and give the eager step's bits."""
    c, hid, rows = 128, 384, 50
    x = leaf(rows, c, seed=1, dtype=torch.bfloat16)
    h0 = leaf(rows, c, seed=2, dtype=torch.bfloat16)
    weights = [leaf(c, seed=3, scale=0.1, mean=1.0), leaf(hid, c, seed=4, scale=c ** -0.5), leaf(hid, seed=5), leaf(c, hid, seed=6, scale=hid ** -0.5), leaf(c, seed=7)]
    seed = torch.tensor([11, 0], device="cuda")

    def step():
        out, h, _ = block(x, h0, weights, 0.2, seed)
        return torch.autograd.grad((tr.dropout_layer(out, 0.2, seed, 1, residual=h).float() ** 2).mean(), [x, h0] + weights)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = step()
    side.synchronize()
    seen = []
    for k in range(3):
        seed.copy_(torch.tensor([11, 10 * k]))
        graph.replay()
        torch.cuda.synchronize()
        seen.append([t.clone() for t in held])
        for a, b in zip(held, step()):
            assert a.equal(b)
    assert not seen[0][0].equal(seen[1][0])
