"""RMS norm, dropout, rows of signed 8-bit codes and their products on the GPU, against plain forms in 64 bits (rows_oracle.py).

Tolerances count roundings: half a step of an output's type (HALF), 2^-24 per fp32 operation.  A sum of n terms taken in a tree of threads'
sums is off by at most (terms per thread + levels of the tree) 2^-24 of the sum of magnitudes; TERMS bounds that for rows of up to `cols`."""
import numpy as np
import pytest
import torch

import rows_oracle as ro

pytestmark = pytest.mark.gpu
tr = pytest.importorskip("paper_2506_17974_b200.training")
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}      # half the smallest step
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16, torch.float32]
# lengths around the changes of kernel: lanes of a warp, a warp, blocks of one to eight runs a thread, rows read twice
LENGTHS = [1, 7, 8, 31, 33, 64, 100, 129, 250, 256, 577, 1000, 1024, 1025, 4096, 4099, 8200, 16384, 16400, 25087, 33000]


def terms(cols):
    """fp32 additions that one term of a row's sum passes: a thread's (8 a run, runs of 4 to 512 threads), two trees of warps."""
    return 8 * max(8, -(-cols // 4096)) + 12


def matrix(rows, cols, dtype, seed, pad=0, shift=0, scale=1.0, device="cuda"):
    """Normal values; rows `cols + pad` apart, the first `shift` elements into its buffer."""
    g = torch.Generator(device=device).manual_seed(seed)
    flat = torch.randn(shift + rows * (cols + pad), generator=g, device=device).mul_(scale).to(dtype)
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def f64(t):
    return t.detach().double().cpu().numpy()


def near(got, want, dtype, slack=0.0):
    """Within half a step of its type, and `slack` (absolute), of the value in 64 bits; a result computed in fp32 is rounded once more."""
    got, want = f64(got), np.asarray(want)
    # past the type's largest value by half a step a result is infinite (65536 x is, in float16, for every |x| >= 1)
    over = np.isinf(got) & (np.abs(want) >= torch.finfo(dtype).max) & (np.sign(got) == np.sign(want))
    got = np.where(over, want, got)
    tol = (HALF[dtype] + 2 * U) * np.abs(want) + LEAST[dtype] + slack
    worst = np.abs(got - want) - tol
    assert (worst <= 0).all(), (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


# -------------------------------------------------------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 0, 0), (5, 100, 28, 0), (4, 100, 1, 3), (2, 129, 0, 0), (33, 257, 0, 1), (7, 264, 0, 0),
                                                 (64, 4096, 0, 0), (9, 4096, 8, 4), (1, 25087, 0, 0), (3, 25087, 1, 0), (700, 40, 0, 0)])
def test_dropout(dtype, rows, cols, pad, shift):
    x, res = matrix(rows, cols, dtype, 1, pad, shift), matrix(rows, cols, dtype, 2)
    for p, seed, offset, r in ((0.37, 5, 0, None), (0.1, 2 ** 63 + 11, 2 ** 40 + 3, res), (0.0, 1, 1, res), (0.99999, -4, 7, None)):
        want = ro.dropped(f64(x), p, seed, offset, None if r is None else f64(r))
        y = tr.dropout(x, p, seed, offset, residual=r)
        near(y, want, dtype)
        if r is None:
            assert ((f64(y) == 0) == ((want == 0) | (np.abs(want) <= LEAST[dtype]))).all()       # dropped values are exactly 0


def test_dropout_does_not_depend_on_layout():
    """One mask for every type, stride and alignment, alone and inside the norm; and its share is p's."""
    rows, cols, p, seed, offset = 37, 1003, 0.25, 99, 12
    keep = ro.kept(rows, cols, p, seed, offset)
    assert abs(keep.mean() - 0.75) < 5 * (0.25 * 0.75 / keep.size) ** 0.5
    for dtype in TYPES:
        for pad, shift in ((0, 0), (5, 0), (5, 8), (0, 1)):
            ones = torch.ones(shift + rows * (cols + pad), device="cuda", dtype=dtype)[shift:].view(rows, cols + pad)[:, :cols]
            assert ((f64(tr.dropout(ones, p, seed, offset)) != 0) == keep).all()
            assert ((f64(tr.rms_norm(ones, torch.ones(cols, device="cuda"), p=p, seed=seed, offset=offset).h) != 0) == keep).all()


@pytest.mark.parametrize("cols", [96, 1001, 4096])
def test_dropout_in_place_and_dropped_infinities(cols):
    x, res = matrix(6, cols, torch.float16, 3), matrix(6, cols, torch.float16, 4)
    want = tr.dropout(x, 0.5, 8, residual=res)
    for out in (x.clone(), res.clone()):
        a, b = (out, res) if out.equal(x) else (x, out)
        assert tr.dropout(a, 0.5, 8, residual=b, out=out) is out and out.equal(want)
    keep = torch.from_numpy(ro.kept(6, cols, 0.5, 8, 0)).cuda()
    bad = torch.where(keep, x, torch.tensor(float("nan"), dtype=x.dtype, device="cuda"))
    bad[:, ::3] = torch.where(keep[:, ::3], bad[:, ::3], torch.tensor(float("inf"), dtype=x.dtype, device="cuda"))
    assert tr.dropout(bad, 0.5, 8).equal(tr.dropout(x, 0.5, 8))


def test_seed_on_the_device_and_replays():
    """A seed on the device gives the mask of the same numbers; a captured call reads it anew at every replay."""
    x = matrix(20, 300, torch.bfloat16, 5)
    gamma = torch.ones(300, device="cuda")
    seed = torch.tensor([77, 1000], dtype=torch.int64, device="cuda")
    assert tr.dropout(x, 0.3, seed, 5).equal(tr.dropout(x, 0.3, 77, 1005))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = tr.dropout(x, 0.3, seed, 5)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = tr.dropout(x, 0.3, seed, 5)
            r = tr.rms_norm(x, gamma, p=0.3, seed=seed, offset=6)
            dx, _, dgamma = tr.rms_norm_grad(r.y, r.h, gamma, r.rstd, p=0.3, seed=seed, offset=6)
            seed[1] += 16
    torch.cuda.current_stream().wait_stream(side)
    start = int(seed[1])
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        off = start + 16 * k
        assert y.equal(tr.dropout(x, 0.3, 77, off + 5))
        want = tr.rms_norm(x, gamma, p=0.3, seed=77, offset=off + 6)
        assert r.y.equal(want.y) and r.h.equal(want.h)
        wx, _, wg = tr.rms_norm_grad(want.y, want.h, gamma, want.rstd, p=0.3, seed=77, offset=off + 6)
        assert dx.equal(wx) and dgamma.equal(wg)


# ------------------------------------------------------------------------------------------------- rows of signed codes

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", LENGTHS)
def test_rows8(dtype, cols):
    rows = 5 if cols > 4000 else 37
    for pad, shift in ((0, 0), (3, 1)):
        x = matrix(rows, cols, dtype, cols, pad, shift) * torch.logspace(-6, 4, rows, device="cuda").to(dtype)[:, None]
        x = torch.nn.functional.pad(x, (0, pad))[:, :cols]
        codes, scales = ro.rows8(x.float().cpu().numpy())
        r = tr.pack_rows8(x)
        assert (r.scales.cpu().numpy() == scales).all() and (r.codes.cpu().numpy() == codes).all()
        given = tr.Rows8(torch.full((rows, cols + 7), 9, dtype=torch.int8, device="cuda")[:, :cols], torch.empty(rows, device="cuda"))
        tr.pack_rows8(x, out=given)
        assert given.codes.equal(r.codes) and (given.codes.as_strided((rows, 7), (cols + 7, 1), cols) == 9).all()
        for to in TYPES:
            want = torch.from_numpy(codes.astype(np.float32) * scales[:, None]).to(to)
            assert tr.unpack_rows8(r, to).cpu().equal(want)
            wide = torch.full((rows, cols + 5), 3.0, dtype=to, device="cuda")
            tr.unpack_rows8(given, to, out=wide[:, 3:cols + 3])
            assert wide[:, 3:cols + 3].cpu().equal(want) and (wide[:, :3] == 3).all() and (wide[:, cols + 3:] == 3).all()


@pytest.mark.parametrize("cols", [5, 200, 2000, 40000])
def test_rows8_of_special_rows(cols):
    x = torch.zeros(8, cols, device="cuda")
    x[1], x[2, -1] = 2.0 ** -149, float("inf")
    x[3, 0], x[4] = float("nan"), torch.finfo(torch.float32).max
    x[5, cols // 2] = -1e-36
    x[6] = -2.0 ** -119
    x[7, 0], x[7, -1] = 1.0, -1.0
    codes, scales = ro.rows8(x.cpu().numpy())
    r = tr.pack_rows8(x)
    assert (r.codes.cpu().numpy() == codes).all() and np.array_equal(r.scales.cpu().numpy(), scales, equal_nan=True)
    y = tr.unpack_rows8(r, torch.float32)
    assert torch.isnan(y[2:4]).all() and torch.isfinite(y[4:]).all() and (y[:2] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [16385, 28672, 28673, 57344, 57352])
def test_rows8_of_long_rows(dtype, cols):
    """Around the lengths up to which a block has a row in shared memory."""
    for pad in (0, 1):
        x = matrix(2, cols, dtype, cols, pad)
        codes, scales = ro.rows8(x.float().cpu().numpy())
        r = tr.pack_rows8(x)
        assert (r.codes.cpu().numpy() == codes).all() and (r.scales.cpu().numpy() == scales).all()


# ------------------------------------------------------------------------------------------------------------- the norm

def check_forward(x, res, gamma, p, eps=1e-6, seed=3, offset=9):
    rows, cols = x.shape
    dtype = x.dtype
    r = tr.rms_norm(x, gamma, eps, res, p, seed, offset, save_h8=True, save_y8=True, save_rows8=True)
    if res is None and p == 0:
        assert r.h is x
    else:
        near(r.h, ro.dropped(f64(x), p, seed, offset, None if res is None else f64(res)), dtype)
        assert r.h.equal(tr.dropout(x, p, seed, offset, residual=res))
    h = f64(r.h)
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    tol = terms(cols) / 2 * U + 4 * U                         # half the sum's error; the mean, + eps, the root, the reciprocal
    assert (np.abs(f64(r.rstd) - rstd) <= tol * rstd).all()
    y = h * rstd[:, None] * f64(gamma)
    near(r.y, y, dtype, (tol + 2 * U) * np.abs(y))
    for kept, of in ((r.h8, r.h), (r.y8, r.y)):
        want = tr.pack8(of)
        assert kept.codes.equal(want.codes) and kept.exps.equal(want.exps)
    top = np.abs(y).max(1)
    scales = f64(r.rows8.scales)
    assert (np.abs(scales - np.maximum(top / 127, 2.0 ** -120)) <= (tol + 4 * U) * np.maximum(top / 127, 2.0 ** -120)).all()
    back = f64(r.rows8.codes) * scales[:, None]
    assert (np.abs(back - y) <= scales[:, None] / 2 + (2 * tol + 8 * U) * np.abs(y)).all()
    few = tr.rms_norm(x, gamma, eps, res, p, seed, offset, want_y=False, save_rows8=True)
    assert few.y is None and few.h8 is None and few.rows8.codes.equal(r.rows8.codes) and few.rstd.equal(r.rstd)
    return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", LENGTHS)
def test_rms_norm(dtype, cols):
    rows = 3 if cols > 4000 else 19
    gamma = matrix(1, cols, torch.float32, 6)[0] * 0.2 + 1
    res = matrix(rows, cols, dtype, 8, scale=1.5)
    check_forward(matrix(rows, cols, dtype, 7), res, gamma, 0.1)
    check_forward(matrix(rows, cols, dtype, 7, pad=3, shift=1), None, gamma, 0.0)
    check_forward(matrix(1, cols, dtype, 9), matrix(1, cols, dtype, 10, shift=1), matrix(1, cols, torch.float32, 6, shift=1)[0], 0.0)


def test_rms_norm_of_special_rows():
    """Rows of zeros, of equal values, of tiny values, with an infinity, with a NaN, and whose squares pass fp32's range."""
    for cols in (40, 600, 3000, 35000):
        x = torch.zeros(6, cols, device="cuda")
        x[1], x[2] = 1.0, 1e-30
        x[3, 5], x[4, 7], x[5] = float("inf"), float("nan"), 1e25
        r = tr.rms_norm(x, torch.ones(cols, device="cuda"), save_rows8=True, save_y8=True)
        assert (r.y[0] == 0).all() and (r.rows8.codes[0] == 0).all() and r.rows8.scales[0] == 2.0 ** -120
        assert ((r.y[1] - 1).abs() < 1e-6).all() and (r.rows8.codes[1] == 127).all()
        assert ((r.y[2] / 1e-27 - 1).abs() < 1e-6).all()
        assert r.rstd[3] == 0 and torch.isnan(r.y[3, 5]) and torch.isnan(r.rows8.scales[3]) and (r.rows8.codes[3] == 0).all()
        assert torch.isnan(r.y[4]).all() and torch.isnan(r.rows8.scales[4]) and torch.isnan(r.rstd[4])
        assert r.rstd[5] == 0 and (r.y[5] == 0).all()


def check_backward(dy, h, gamma, rstd, skip, p, seed=4, offset=2):
    rows, cols = dy.shape
    dtype = dy.dtype
    hv = f64(tr.unpack8(h, torch.float32) if isinstance(h, tr.Packed8) else h)
    g, r, dyv, sk = f64(gamma), f64(rstd), f64(dy), None if skip is None else f64(skip)
    d, dgamma = ro.rms_grad(dyv, hv, g, r, sk)
    dx, dres, dg = tr.rms_norm_grad(dy, h, gamma, rstd, skip, p, seed, offset)
    # u, xh, their product's mean, the difference, + skip: each 2^-24 of its own size; the mean as a sum of magnitudes
    xh, u = np.abs(hv * r[:, None]), np.abs(dyv * g)
    slack = U * (r[:, None] * (3 * u + xh * (terms(cols) + 6) * (u * xh).mean(1, keepdims=True)) + (0 if sk is None else np.abs(sk)) + 2 * np.abs(d))
    near(dres, d, dtype, slack)
    if p > 0:
        scale = 65536 / (65536 - ro.threshold(p))
        near(dx, ro.dropped(d, p, seed, offset), dtype, slack * scale + 2 * U * np.abs(d) * scale)
        assert ((f64(dx) != 0) <= ro.kept(rows, cols, p, seed, offset)).all()
    else:
        assert dx is dres
    # a row's term, then sums of at most `rows` of them in some order
    near(dg, dgamma, torch.float32, U * (rows + 4) * (np.abs(dyv) * xh).sum(0))
    alone = tr.rms_norm_grad(dy, h, gamma, rstd, skip, p, seed, offset, gamma_grad=False)
    assert alone[2] is None and alone[0].equal(dx) and alone[1].equal(dres)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [6657, 10241, 13313, 28679, 57352])
def test_rms_norm_of_long_rows(dtype, cols):
    """Steps of every width: the last one full, nearly empty, or with lanes left over."""
    gamma = matrix(1, cols, torch.float32, 6)[0] * 0.2 + 1
    check_forward(matrix(2, cols, dtype, 7), matrix(2, cols, dtype, 8, scale=1.5), gamma, 0.1)
    check_forward(matrix(2, cols, dtype, 7, pad=3, shift=1), None, gamma, 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", LENGTHS)
def test_rms_norm_grad(dtype, cols):
    rows = 3 if cols > 4000 else 23
    gamma = matrix(1, cols, torch.float32, 6)[0] * 0.2 + 1
    h = matrix(rows, cols, dtype, 11, scale=1.5)
    dy, skip = matrix(rows, cols, dtype, 12, scale=0.05), matrix(rows, cols, dtype, 13, scale=0.05)
    fwd = tr.rms_norm(h, gamma, save_h8=True)
    check_backward(dy, fwd.h8, gamma, fwd.rstd, skip, 0.1)
    check_backward(dy, h, gamma, fwd.rstd, None, 0.0)
    odd = matrix(rows, cols, dtype, 12, pad=3, shift=1, scale=0.05)
    check_backward(odd, matrix(rows, cols, dtype, 11, pad=1, scale=1.5), gamma, fwd.rstd, matrix(rows, cols, dtype, 13, shift=1), 0.37)


@pytest.mark.parametrize("rows,cols", [(1, 64), (5000, 40), (3001, 520), (2500, 1030), (700, 4096), (200, 20000)])
def test_rms_norm_grad_over_many_rows(rows, cols):
    """Every block has several rows, and their sums meet; repeated calls give the same bits."""
    gamma = matrix(1, cols, torch.float32, 6)[0] * 0.2 + 1
    h, dy = matrix(rows, cols, torch.bfloat16, 14), matrix(rows, cols, torch.bfloat16, 15)
    rstd = tr.rms_norm(h, gamma).rstd
    check_backward(dy, h, gamma, rstd, None, 0.1)
    a, b = (tr.rms_norm_grad(dy, h, gamma, rstd, p=0.1, seed=1) for _ in range(2))
    assert all(s.equal(t) for s, t in zip(a, b))


def test_empty_batches():
    gamma, x = torch.ones(48, device="cuda"), torch.empty(0, 48, device="cuda", dtype=torch.bfloat16)
    r = tr.rms_norm(x, gamma, residual=x, p=0.1, save_h8=True, save_y8=True, save_rows8=True)
    assert r.y.shape == r.h.shape == r.h8.shape == r.rows8.shape == (0, 48) and r.rstd.shape == (0,)
    dx, _, dgamma = tr.rms_norm_grad(x, x, gamma, r.rstd)
    assert dx.shape == (0, 48) and (dgamma == 0).all()
    assert tr.dropout(x, 0.5, 1).shape == (0, 48) and tr.pack_rows8(x).shape == (0, 48)
    w = tr.pack_rows8(torch.ones(9, 48, device="cuda"))
    assert tr.linear_rows8(r.rows8, w, save_z8=True).y.shape == (0, 9)


# ------------------------------------------------------------------------------------------ products of rows of codes

def check_product(rows, cin, cout, dtype, act, bias, residual, seed=0, x_pad=0, w_pad=0, out_pad=0, extreme=False, copies=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    def codes(r, pad):                                                                         # noqa: E306
        if extreme:
            return torch.full((r, cin), -128, dtype=torch.int8, device="cuda")
        wide = (cin + 15) // 16 * 16 if pad == 0 else cin + pad
        return torch.randint(-127, 128, (r, wide), generator=g, device="cuda", dtype=torch.int8)[:, :cin]
    xc, wc = codes(rows, x_pad), codes(cout, w_pad)
    size = 2.0 ** -30 if extreme else 1 / (73 * 73 * cin ** 0.5)                               # sums of size about 1
    sx = torch.rand(rows, generator=g, device="cuda") * 2 + 0.1
    sw = (torch.rand(cout, generator=g, device="cuda") + 0.5) * size
    b = torch.randn(cout, generator=g, device="cuda") if bias else None
    res = matrix(rows, cout, dtype, seed + 1, out_pad) if residual else None
    out = torch.full((rows, cout + out_pad), 5.0, device="cuda", dtype=dtype)
    acc = (xc.double() @ wc.double().t()).cpu().numpy()                                        # exact: below 2^53
    r = tr.linear_rows8(tr.Rows8(xc, sx), tr.Rows8(wc, sw), b, act, res, dtype, save_z8=copies, save_y8=copies, out=out[:, :cout] if out_pad else None)
    product = acc * f64(sx)[:, None] * f64(sw)
    z = product + (0 if b is None else f64(b))
    z_off = 3 * U * np.abs(product) + U * np.abs(z)                                            # the integer's rounding and two scales; the bias
    zt = torch.from_numpy(z)
    y = {"none": zt, "relu": zt.clamp(min=0), "gelu": zt * 0.5 * torch.erfc(-zt / 2 ** 0.5), "silu": zt * torch.sigmoid(zt)}[act].numpy()
    # slopes are at most 1.13; the activations' own fp32 error is that of linear()'s tests: 2^-21 of |z| covers it
    slack = 1.13 * z_off + (0 if act in ("none", "relu") else 2.0 ** -21 * np.abs(z))
    if res is not None:
        y = y + f64(res)
        slack = slack + U * np.abs(y)
    near(r.y, y, dtype, slack)
    assert (f64(out)[:, cout:] == 5).all() and tr.status() == 0
    if not copies:
        return
    z8 = f64(tr.unpack8(r.z8, torch.float32))
    groups = np.abs(np.pad(z, ((0, 0), (0, -cout % 32)))).reshape(rows, -1, 32).max(2)
    step = np.exp2(np.maximum(np.ceil(np.log2(np.maximum(groups * (1 + 8 * U), 1e-300) / 127.5)), -126))
    step = np.repeat(step, 32, 1)[:, :cout]
    assert (np.abs(z8 - z) <= step / 2 + z_off * 2).all()
    want = tr.pack8(r.y)
    assert r.y8.codes.equal(want.codes) and r.y8.exps.equal(want.exps)


@pytest.mark.parametrize("rows,cin,cout", [
    (1, 1, 1), (1, 16, 10), (1, 4096, 300), (2, 31, 7), (3, 128, 128), (7, 129, 100), (8, 127, 33), (16, 1000, 257), (17, 257, 512), (31, 4097, 130),
    (64, 512, 1000), (128, 128, 128), (129, 640, 129), (250, 3136, 512), (255, 96, 4100), (300, 2000, 40), (1000, 577, 577), (1, 16384, 64), (5, 70000, 12),
    (1500, 300, 2600), (2048, 512, 4096), (4096, 256, 2300)])
def test_linear_rows8(rows, cin, cout):
    check_product(rows, cin, cout, torch.bfloat16, "gelu", True, True, seed=rows)
    check_product(rows, cin, cout, torch.float16, "silu", False, False, seed=cin)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cin,cout", [(3, 300, 70), (200, 160, 260), (1200, 200, 2500)])
def test_linear_rows8_layouts(act, rows, cin, cout):
    """Rows of codes and of the output at every alignment."""
    for x_pad, w_pad, out_pad in ((1, 0, 1), (0, 3, 2), (4, 5, 8)):
        check_product(rows, cin, cout, torch.float16, act, True, out_pad != 2, x_pad + 10 * w_pad, x_pad, w_pad, out_pad)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("cin,cout", [(1, 1), (15, 3), (16, 4), (17, 33), (496, 5), (512, 1001), (4100, 7), (4096, 130), (40000, 9), (131071, 2), (520, 40000)])
def test_linear_rows8_of_few_rows(rows, cin, cout):
    """Without copies in 8 bits a few rows take a kernel of their own."""
    check_product(rows, cin, cout, torch.bfloat16, "silu", True, rows != 2, seed=cin, copies=False)
    check_product(rows, cin, cout, torch.float16, "none", rows == 3, False, seed=cout, out_pad=rows - 1, copies=False)


def test_longest_and_largest_sums():
    """131071 products of 128 by 128: one short of leaving 32 bits."""
    check_product(3, 131071, 5, torch.bfloat16, "none", False, False, extreme=True)
    check_product(3, 131071, 5, torch.bfloat16, "none", False, False, extreme=True, copies=False)
    check_product(300, 131071, 140, torch.float16, "none", True, False)


def test_rows_that_are_not_finite():
    x = matrix(40, 256, torch.bfloat16, 1)
    x[3, 5], x[9, 0] = float("nan"), float("inf")
    w = tr.pack_rows8(matrix(70, 256, torch.float32, 2))
    r = tr.linear_rows8(tr.pack_rows8(x), w, act="gelu", save_z8=True)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 9]] = True
    assert torch.isnan(r.y[bad]).all() and torch.isfinite(r.y[~bad]).all()
    assert (r.z8.exps[bad] == 255).all()


@pytest.mark.parametrize("rows", [1, 40, 600])
def test_sums_that_leave_the_range(rows):
    """Scales that carry a sum past fp32's range: infinity through every activation, nothing through those that cut negative values."""
    codes = torch.ones(rows, 64, dtype=torch.int8, device="cuda")
    w = torch.ones(300, 64, dtype=torch.int8, device="cuda")
    w[::2] = -1
    x8, w8 = tr.Rows8(codes, torch.full((rows,), 1e30, device="cuda")), tr.Rows8(w, torch.full((300,), 1e30, device="cuda"))
    for act in ("none", "relu", "gelu", "silu"):
        y = tr.linear_rows8(x8, w8, act=act).y
        assert (y[:, 1::2] == float("inf")).all()
        if act in ("relu", "none"):
            assert (y[:, ::2] == (0 if act == "relu" else -float("inf"))).all()


def test_product_of_kept_rows_is_near_the_real_one():
    """x and w to codes and their product, against the product of the values that the codes stand for."""
    x, w = matrix(65, 700, torch.bfloat16, 1), matrix(90, 700, torch.float32, 2, scale=700 ** -0.5)
    x8, w8 = tr.pack_rows8(x), tr.pack_rows8(w)
    want = (f64(x8.codes) * f64(x8.scales)[:, None]) @ (f64(w8.codes) * f64(w8.scales)[:, None]).T
    near(tr.linear_rows8(x8, w8, dtype=torch.float16).y, want, torch.float16, 4 * U * np.abs(want))


# ----------------------------------------------------------------------------------------------------- calls and refusals

def test_matrices_of_more_than_2_to_the_31_values():
    """Rows whose offsets pass 32 bits: the last rows of a large matrix against the same rows by themselves."""
    rows, cols = 53700, 40001                                   # 2.148e9 values; every row starts elsewhere in 16 bytes
    x = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
    x.copy_(torch.randn(1, cols, device="cuda") * torch.linspace(1, 2, rows, device="cuda")[:, None])
    last, gamma = x[-3:].clone(), torch.ones(cols, device="cuda")
    y = tr.dropout(x, 0.5, 3)
    assert ((f64(y[-3:]) != 0) == (ro.kept(3, cols, 0.5, 3, 0, rows - 3) & (f64(last) != 0))).all()
    del y
    r, want = tr.rms_norm(x, gamma), tr.rms_norm(last, gamma)
    assert r.y[-3:].equal(want.y) and r.rstd[-3:].equal(want.rstd)
    dx, _, dgamma = tr.rms_norm_grad(r.y, x, gamma, r.rstd)
    assert dx[-3:].equal(tr.rms_norm_grad(want.y, last, gamma, want.rstd)[0])
    xh = x[::4000].double() * r.rstd[::4000].double()[:, None]   # gamma = 1: dgamma = the sum over rows of y xh, rows nearly alike
    assert ((dgamma.double() / rows - (xh * xh).mean(0)).abs() <= 0.02 * (xh * xh).mean(0) + 1e-6).all()
    del r, dx
    p, want = tr.pack_rows8(x), tr.pack_rows8(last)
    assert p.codes[-3:].equal(want.codes) and p.scales[-3:].equal(want.scales)
    assert tr.unpack_rows8(p)[-3:].equal(tr.unpack_rows8(want))


def test_largest_kept_values():
    """h near the end of fp32's range, kept in 8 bits: the gradient reads what unpack8 gives in bfloat16."""
    h = torch.zeros(2, 96, device="cuda")
    h[0, :40], h[1, 50] = torch.finfo(torch.float32).max, -3e38
    h8, gamma, rstd = tr.pack8(h), torch.ones(96, device="cuda"), torch.full((2,), 1e-38, device="cuda")
    dy = matrix(2, 96, torch.float32, 1)
    got, want = (tr.rms_norm_grad(dy, t, gamma, rstd) for t in (h8, tr.unpack8(h8, torch.bfloat16).float()))
    # a sum of such rows' products may pass fp32's range (then NaN in both); xh = h rstd, of size 1, and dgamma do not
    assert all(torch.allclose(a, b, rtol=0, atol=0, equal_nan=True) for a, b in zip(got, want)) and torch.isfinite(got[2]).all()


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e15, 1e30])
@pytest.mark.parametrize("cols", [40, 1100, 9000])
def test_rms_norm_grad_of_rows_of_any_size(size, cols):
    """Without eps the norm does not see a row's size, and its gradient is divided by it."""
    h, dy, gamma = matrix(4, cols, torch.float32, 1), matrix(4, cols, torch.float32, 2), torch.ones(cols, device="cuda")
    rstd = (1 / h.double().square().mean(1).sqrt()).float()
    dx, _, dgamma = tr.rms_norm_grad(dy, h * size, gamma, rstd / size)
    want, wantg = ro.rms_grad(f64(dy), f64(h * size), np.ones(cols), f64(rstd / size))
    assert np.linalg.norm(f64(dx) - want) < 1e-5 * np.linalg.norm(want) and np.linalg.norm(f64(dgamma) - wantg) < 1e-5 * np.linalg.norm(wantg)


def test_refusals():
    x, gamma = matrix(4, 64, torch.bfloat16, 1), torch.ones(64, device="cuda")
    x8, w8 = tr.pack_rows8(x), tr.pack_rows8(matrix(8, 64, torch.float32, 2))
    seed = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: tr.dropout(x, 0.1, seed), lambda: tr.dropout(x, 0.1, seed.cuda().float()), lambda: tr.dropout(x, 0.1, seed.cuda()[:1]),
                 lambda: tr.dropout(x, 0.1, 0, residual=x[:3]), lambda: tr.dropout(x, 0.1, 0, residual=x.float()), lambda: tr.dropout(x.t(), 0.1, 0),
                 lambda: tr.dropout(x.double(), 0.1, 0), lambda: tr.rms_norm(x, gamma[:63]), lambda: tr.rms_norm(x, gamma.bfloat16()),
                 lambda: tr.rms_norm(x, gamma, residual=x.half()), lambda: tr.rms_norm(x[0], gamma), lambda: tr.rms_norm_grad(x, x, gamma, gamma),
                 lambda: tr.rms_norm_grad(x, tr.pack8(x[:3]), gamma, gamma[:4]), lambda: tr.linear_rows8(x8, w8, dtype=torch.float32),
                 lambda: tr.linear_rows8(x, w8), lambda: tr.linear_rows8(x8, tr.pack_rows8(x[:, :32])), lambda: tr.linear_rows8(x8, w8, act="tanh"),
                 lambda: tr.linear_rows8(x8, w8, bias=gamma), lambda: tr.linear_rows8(x8, w8, residual=x), lambda: tr.Rows8(x8.codes, x8.scales[:3]),
                 lambda: tr.Rows8(x8.codes.view(torch.uint8), x8.scales), lambda: tr.pack_rows8(x, out=w8), lambda: tr.unpack_rows8(x8, torch.int8)):
        with pytest.raises(ValueError):
            call()
    from paper_2506_17974_b200 import binding as B
    for call in (lambda: tr.dropout(x, 1.0, 0), lambda: tr.dropout(x, -0.1, 0), lambda: tr.rms_norm(x, gamma, p=float("nan"), residual=x),
                 lambda: tr.rms_norm(x, gamma, eps=-1.0)):
        with pytest.raises(B.LqsgdError) as e:
            call()
        assert e.value.code == B.ERR_INVALID_ARG
        del e                                                 # with its traceback it would keep this frame, and the tensors, until a collection


def test_other_stream_and_capture():
    """The whole block on a side stream and from a graph: the same bits as on the default stream."""
    x, res = matrix(130, 512, torch.bfloat16, 1), matrix(130, 512, torch.bfloat16, 2)
    gamma, w8 = torch.ones(512, device="cuda"), tr.pack_rows8(matrix(1000, 512, torch.float32, 3, scale=0.05))

    def block():
        r = tr.rms_norm(x, gamma, residual=res, p=0.2, seed=5, want_y=False, save_rows8=True)
        return r.h, tr.linear_rows8(r.rows8, w8, act="silu").y

    want = block()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = block()
        side.synchronize()
        assert all(a.equal(b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = block()
        for t in held:
            t.zero_()
        graph.replay()
    side.synchronize()
    assert all(a.equal(b) for a, b in zip(held, want))
