"""The training operators against their formulas in 64 bits: linear layers, activations in 8 bits, group norm.

Error bounds are derived, not fitted.  u(T) = 2^-p, p the significant bits of T, is half a unit in the last place, relative: 2^-8 (bf16),
2^-11 (fp16), 2^-24 (fp32).  A sum of K products accumulated in fp32 is off by at most c * 2^-23 * sum |a||b| with c the
number of additions a partial sum goes through (the tensor core may truncate instead of rounding, hence 2^-23)."""
import math

import pytest
import torch

from paper_2506_17974_b200 import binding as B
from paper_2506_17974_b200 import training as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF: 2.0 ** -133, HF: 2.0 ** -25, F32: 2.0 ** -149}        # half the smallest subnormal number


def randn(*shape, seed=0, dtype=F32, scale=1.0, pad=0):
    g = torch.Generator(DEV).manual_seed(seed)
    wide = (torch.randn(*shape[:-1], shape[-1] + pad, generator=g, device=DEV) * scale).to(dtype)
    return wide[..., :shape[-1]]


def assert_within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    assert torch.isfinite(got).all(), what
    over = ((got - want).abs() - bound).max().item()
    worst = ((got - want).abs() / torch.as_tensor(bound, device=got.device).clamp(min=1e-300)).max().item()
    assert over <= 0, f"{what}: {worst:.2f} x the bound"


# ------------------------------------------------------------------------------------------------------------- 8-bit form

def power64(e):
    """2^e in 64 bits, exactly (pow and exp2 need not be)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def reference_pack(x):
    """Codes and exponent bytes from the definition, in 64 bits."""
    rows, cols = x.shape
    pad = -cols % 32
    v = torch.nn.functional.pad(x.double(), (0, pad)).view(rows, -1, 32)
    top = v.abs().amax(2)
    bad = ~torch.isfinite(top)
    top = torch.where(bad, torch.zeros_like(top), top)
    e = torch.full_like(top, -126)
    for k in range(-126, 124):                       # the smallest e with rint(top / 2^e) <= 127
        too_big = torch.round(top * power64(-e)) > 127
        e = torch.where(too_big, torch.full_like(e, k + 1), e)
    mag = torch.round(v.abs() * power64(-e)[..., None]).nan_to_num(0, 0, 0)
    code = mag.to(torch.int64) + 128 * torch.signbit(v)
    exps = torch.where(bad, torch.full_like(e, 255), e + 126).to(torch.int64)
    value = torch.where(bad[..., None], torch.full_like(v, math.nan), torch.where(torch.signbit(v), -mag, mag) * power64(e)[..., None])
    return code.view(rows, -1)[:, :cols], exps, value.view(rows, -1)[:, :cols]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 31, 0), (5, 32, 0), (7, 33, 2), (64, 64, 0), (9, 100, 1), (33, 257, 0), (2, 1000, 8), (300, 96, 32)])
def test_pack8_is_the_definition_bit_for_bit(dtype, rows, cols, pad):
    x = randn(rows, cols, seed=rows * cols, scale=3.0, pad=pad).to(dtype)
    x = (x * torch.exp2(torch.randint(-12, 12, (rows, 1), device=DEV).float())).to(dtype)
    wide = torch.zeros(rows, cols + pad, dtype=dtype, device=DEV)
    wide[:, :cols] = x
    x = wide[:, :cols]
    p = tr.pack8(x)
    code, exps, value = reference_pack(x)
    finite = (exps != 255).repeat_interleave(32, 1)[:, :cols]
    assert torch.equal(p.exps.long(), exps)
    assert torch.equal(p.codes.long()[finite], code[finite])
    back = tr.unpack8(p, F32).double()
    assert torch.equal(back[finite], value[finite])
    assert torch.equal(tr.unpack8(p, BF).double()[finite], value[finite])


def test_pack8_edges():
    rows = [
        [0.0] * 32, [-0.0] * 32,
        [127.5] + [1.0] * 31,                            # rounds to 128: the next exponent
        [127.49] + [0.5, 1.5, 2.5, -0.5, -1.5] + [0.0] * 26,   # halves to even
        [3.4028234663852886e38] + [-1e38] * 31,
        [1e-45, 1e-40, -3e-39] + [0.0] * 29,             # below the smallest step
        [2.0 ** -120, 2.0 ** -121] + [0.0] * 30,
        [math.inf] + [1.0] * 31, [1.0] * 31 + [-math.inf], [math.nan] + [1.0] * 31,
    ]
    x = torch.tensor(rows, dtype=F32, device=DEV)
    p = tr.pack8(x)
    code, exps, value = reference_pack(x)
    assert torch.equal(p.exps.long(), exps)
    ok = exps[:, 0] != 255
    assert torch.equal(p.codes.long()[ok], code[ok])
    back = tr.unpack8(p, F32)
    assert torch.isnan(back[~ok]).all()
    big = torch.finfo(F32).max
    assert torch.equal(back[ok].double(), value[ok].clamp(-big, big))
    assert torch.isnan(tr.unpack8(p, HF)[~ok]).all()
    assert tr.unpack8(p, HF)[4].abs().max().item() == 65504.0        # saturates
    assert tr.unpack8(p, BF)[4].abs().max().item() == torch.finfo(BF).max


def test_pack8_rows_past_2_to_31_bytes():
    """Offsets that pass 32 bits: the last rows of a matrix of 2^31 + bytes of codes."""
    rows, cols = 70001, 32768
    x = torch.zeros(rows, cols, dtype=BF, device=DEV)
    x[-3:] = randn(3, cols, seed=5, dtype=BF)
    p = tr.pack8(x)
    code, exps, value = reference_pack(x[-3:])
    assert torch.equal(p.codes[-3:].long(), code) and torch.equal(p.exps[-3:].long(), exps)
    assert int(p.codes[:-3].max()) == 0
    assert torch.equal(tr.unpack8(p, BF)[-3:].double(), value)


def kept(rows, cols, seed, dtype=F32, scale=1.0):
    """An 8-bit matrix and the values it stands for."""
    p = tr.pack8(randn(rows, cols, seed=seed, dtype=dtype, scale=scale))
    return p, tr.unpack8(p, F32).double()


def act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z),
            "gelu": lambda: 0.5 * z * torch.special.erfc(-z / math.sqrt(2))}[act]()


def slope64(z, act):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: s + z * s * (1 - s),
            "gelu": lambda: 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[act]()


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 300, 0), (5, 33, 3), (129, 64, 0), (1000, 40, 0), (257, 1025, 7), (2048, 512, 0)])
def test_act_grad(dtype, act, rows, cols, pad):
    dy = randn(rows, cols, seed=1, dtype=dtype, pad=pad)
    z8, z = kept(rows, cols, 2, scale=2.0)
    dz, db = tr.act_grad(dy, z8 if act != "none" else None, act)
    want = dy.double() * slope64(z, act)
    # the slope in fp32: functions of a few units in the last place, values up to 1.13, absolute error below 2^-20
    part = dy.double().abs() * 2.0 ** -20
    if act == "none":
        assert dz is dy
    else:
        assert_within(dz, want, want.abs() * U[dtype] * 1.01 + part + TINY[dtype], "dz")
    adds = rows / 8 + 64
    assert_within(db, want.sum(0), (part + adds * 2.0 ** -24 * want.abs()).sum(0) + 1e-30, "db")


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_act_grad_over_the_whole_range_of_steps(act):
    """One column of groups per exponent, magnitudes 0 .. 127, both signs."""
    exps = torch.arange(0, 249, dtype=torch.uint8, device=DEV)[:, None].repeat(1, 8)
    codes = torch.arange(256, dtype=torch.uint8, device=DEV)[None].repeat(249, 1).contiguous()
    p = tr.Packed8(codes, exps)
    z = tr.unpack8(p, F32).double()
    dz, _ = tr.act_grad(torch.ones(249, 256, device=DEV), p, act)
    assert_within(dz, slope64(z, act), 2.0 ** -20, "slope")


def test_act_grad_may_write_over_dy_and_keeps_nan():
    dy = randn(64, 96, seed=1, dtype=BF)
    z8, z = kept(64, 96, 2)
    want, _ = tr.act_grad(dy, z8, "gelu")
    again = dy.clone()
    got, _ = tr.act_grad(again, z8, "gelu", out=again)
    assert got.data_ptr() == again.data_ptr() and torch.equal(got, want)
    z8.exps[3, 1] = 255
    for act in ("relu", "gelu", "silu"):
        bad, db = tr.act_grad(dy, z8, act)
        assert torch.isnan(bad[3, 32:64]).all() and torch.isfinite(bad[:3]).all()
        assert torch.isnan(db[32:64]).all() and torch.isfinite(db[:32]).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_act_grad_against_differences(act):
    z8, z = kept(40, 70, 3)
    dy = randn(40, 70, seed=4)
    dz, _ = tr.act_grad(dy, z8, act)
    v = randn(40, 70, seed=5).double()
    h = 1e-4
    diff = ((act64(z + h * v, act) - act64(z - h * v, act)) * dy.double()).sum() / (2 * h)
    # truncation h^2 / 6 * f''' (|f'''| < 2) per element, rounding of dz 2^-20
    bound = ((h * h / 3 * v.abs() ** 3 + 2.0 ** -20 * v.abs()) * dy.double().abs()).sum()
    assert abs(((dz.double() * v).sum() - diff).item()) <= bound.item()


# ----------------------------------------------------------------------------------------------------------- linear layers

def product_bound(a, b, k, extra=16):
    """|error| of fp32-accumulated a b^T (a: m x k, b: n x k, in 64 bits)."""
    return (k / 16 + extra) * 2.0 ** -23 * (a.abs() @ b.abs().t())


SIZES = [  # rows, in, out
    (1, 1, 1), (1, 512, 10), (2, 25, 32), (7, 300, 130), (16, 64, 64), (17, 4096, 128), (31, 100, 257), (33, 128, 256), (64, 1000, 96),
    (65, 72, 40), (128, 64, 128), (129, 65, 129), (250, 3136, 512), (257, 512, 100), (1000, 136, 264), (2048, 1024, 512), (515, 2304, 1030),
    (4100, 256, 512), (8192, 64, 128),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_linear(dtype, rows, cin, cout):
    act = ["none", "relu", "gelu", "silu"][(rows + cout) % 4]
    pad = [0, 3, 8][(rows + cin) % 3]
    x = randn(rows, cin, seed=1, dtype=dtype, pad=pad)
    w = randn(cout, cin, seed=2, dtype=dtype, scale=cin ** -0.5)
    bias = randn(cout, seed=3, scale=0.3)
    res = randn(rows, cout, seed=4, dtype=dtype, pad=pad)
    r = tr.linear(x, w, bias, act=act, residual=res, save_z8=True, save_y8=True)
    z = x.double() @ w.double().t() + bias.double()
    dz = product_bound(x.double(), w.double(), cin) + 2.0 ** -23 * z.abs()
    y = act64(z, act) + res.double()
    assert_within(r.y, y, y.abs() * U[dtype] * 1.01 + 1.2 * dz + 2.0 ** -20 * (1 + z.abs()) + TINY[dtype], "y")
    # 8-bit forms: half a step, a step being at most 1/63.5 of the group's largest
    top = torch.nn.functional.pad(z.abs() + dz, (0, -cout % 32)).view(rows, -1, 32).amax(2).repeat_interleave(32, 1)[:, :cout]
    assert_within(tr.unpack8(r.z8, F32), z, top / 127 * 1.0001 + dz + 2.0 ** -127, "z8")
    y8 = tr.pack8(r.y)
    assert torch.equal(r.y8.codes, y8.codes) and torch.equal(r.y8.exps, y8.exps)      # of y as stored
    plain = tr.linear(x, w).y
    zz = x.double() @ w.double().t()
    assert_within(plain, zz, zz.abs() * U[dtype] * 1.01 + dz + TINY[dtype], "x w^T")
    assert tr.status(DEV) == 0


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_linear_grad_input(dtype, rows, cin, cout):
    pad = [0, 3, 8][(rows + cin) % 3]
    dz = randn(rows, cout, seed=1, dtype=dtype, pad=pad)
    w = randn(cout, cin, seed=2, dtype=dtype, scale=cout ** -0.5)
    res = randn(rows, cin, seed=3, dtype=dtype, pad=pad)
    want = dz.double() @ w.double()
    bound = product_bound(dz.double(), w.double().t().contiguous(), cout)
    assert_within(tr.linear_grad_input(dz, w), want, want.abs() * U[dtype] * 1.01 + bound + TINY[dtype], "dx")
    want = want + res.double()
    for inplace in (False, True):
        got = tr.linear_grad_input(dz, w, residual=res, out=res if inplace else None)
        assert_within(got, want, want.abs() * U[dtype] * 1.01 + bound + 2.0 ** -23 * want.abs() + TINY[dtype], "dx + residual")
    assert tr.status(DEV) == 0


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,cin,cout", SIZES + [(70000, 64, 40)])
def test_linear_grad_weight(dtype, packed, rows, cin, cout):
    pad = [0, 3, 8][(rows + cin) % 3]
    dz = randn(rows, cout, seed=1, dtype=dtype, pad=pad)
    x = randn(rows, cin, seed=2, dtype=dtype)
    if packed:
        p = tr.pack8(x)
        if pad == 3:                                     # codes without any alignment
            p = tr.Packed8(p.codes.contiguous(), p.exps.contiguous())
        x64, arg = tr.unpack8(p, F32).double(), p
    else:
        x64, arg = x.double(), x
    want = dz.double().t() @ x64
    bound = product_bound(dz.double().t().contiguous(), x64.t().contiguous(), rows) + 1e-30
    dw = tr.linear_grad_weight(dz, arg)
    assert_within(dw, want, bound, "dw")
    wide = torch.full((cout, cin + 5), 2.0, device=DEV)
    got = tr.linear_grad_weight(dz, arg, out=wide[:, :cin], accumulate=True)
    assert_within(got, want + 2.0, bound + 2.0 ** -23 * (want.abs() + 2), "2 + dw")
    assert (wide[:, cin:] == 2.0).all()
    assert torch.equal(dw, tr.linear_grad_weight(dz, arg))           # the same bits again
    assert tr.status(DEV) == 0


def test_linear_grad_weight_decodes_every_step():
    """Rows of x with steps from the smallest to the largest that the operand type holds, dz picking rows out one by one."""
    for dtype, lo, hi in ((BF, 0, 248), (HF, 90, 136)):
        n = hi - lo + 1
        exps = torch.arange(lo, hi + 1, dtype=torch.uint8, device=DEV)[:, None].repeat(1, 8)
        codes = torch.arange(256, dtype=torch.uint8, device=DEV)[None].repeat(n, 1).contiguous()
        p = tr.Packed8(codes, exps)
        want = tr.unpack8(p, dtype).float()
        dz = torch.eye(n, dtype=dtype, device=DEV)
        assert torch.equal(tr.linear_grad_weight(dz, p), want)
    p.exps[5, 2] = 255
    dw = tr.linear_grad_weight(dz, p)
    assert torch.isnan(dw[:, 64:96]).all() and torch.isfinite(dw[:, :64]).all() and torch.isfinite(dw[:, 96:]).all()


def test_linear_large_tiles_and_long_rows():
    """Sizes that take the widest tile, ragged on every side, and a result whose offsets pass 32 bits."""
    rows, cin, cout = 3333, 1111, 2777
    x, w = randn(rows, cin, seed=1, dtype=BF), randn(cout, cin, seed=2, dtype=BF, scale=cin ** -0.5)
    z = x.double() @ w.double().t()
    assert_within(tr.linear(x, w).y, z, z.abs() * U[BF] * 1.01 + product_bound(x.double(), w.double(), cin), "y")
    dz = randn(rows, cout, seed=3, dtype=BF)
    dx = dz.double() @ w.double()
    assert_within(tr.linear_grad_input(dz, w), dx, dx.abs() * U[BF] * 1.01 + product_bound(dz.double(), w.double().t().contiguous(), cout), "dx")
    rows, cin, cout = 140000, 64, 16384                    # 2.3e9 values
    x, w = randn(rows, cin, seed=1, dtype=BF), randn(cout, cin, seed=2, dtype=BF, scale=0.125)
    r = tr.linear(x, w, save_z8=True)
    for part in (slice(0, 300), slice(rows - 300, rows)):
        z = x[part].double() @ w.double().t()
        assert_within(r.y[part], z, z.abs() * U[BF] * 1.01 + product_bound(x[part].double(), w.double(), cin), "y")
    last = tr.Packed8(r.z8.codes[-300:], r.z8.exps[-300:])
    top = (z.abs() * 1.001).view(300, -1, 32).amax(2).repeat_interleave(32, 1)
    assert_within(tr.unpack8(last, F32), z, top / 127 + 1e-5, "z8")


def test_linear_propagates_infinities_and_nan_only_where_they_belong():
    x, w = randn(130, 96, seed=1, dtype=BF), randn(70, 96, seed=2, dtype=BF)
    clean = tr.linear(x, w).y
    x[5, 7] = math.nan
    y = tr.linear(x, w, save_z8=True)
    assert torch.isnan(y.y[5]).all() and (y.z8.exps[5] == 255).all()
    keep = [i for i in range(130) if i != 5]
    assert torch.equal(y.y[keep], clean[keep]) and (y.z8.exps[keep] != 255).all()


def test_zero_rows():
    x, w = torch.empty(0, 64, dtype=BF, device=DEV), randn(32, 64, seed=1, dtype=BF)
    assert tr.linear(x, w, save_z8=True).y.shape == (0, 32)
    dz = torch.empty(0, 32, dtype=BF, device=DEV)
    assert tr.linear_grad_input(dz, w).shape == (0, 64)
    assert float(tr.linear_grad_weight(dz, x).abs().max()) == 0.0
    assert float(tr.linear_grad_weight(dz, tr.pack8(x), out=torch.ones(32, 64, device=DEV), accumulate=True).min()) == 1.0
    z, db = tr.act_grad(dz, tr.pack8(dz), "gelu")
    assert float(db.abs().max()) == 0.0
    e = torch.empty(0, 9, 64, dtype=BF, device=DEV)
    g, b = torch.ones(64, device=DEV), torch.zeros(64, device=DEV)
    r = tr.group_norm(e, 8, g, b)
    dx, dg, dbeta = tr.group_norm_grad(e, e, 8, g, b, r.mean, r.rstd)
    assert r.y.shape == e.shape and float(dg.abs().max()) == 0.0 and float(dbeta.abs().max()) == 0.0


# ----------------------------------------------------------------------------------------------------------------- group norm

def norm64(x, groups, gamma, beta, eps, act):
    n, hw, c = x.shape
    v = x.double().view(n, hw, groups, c // groups)
    mean, var = v.mean((1, 3)), v.var((1, 3), unbiased=False)
    rstd = 1 / torch.sqrt(var + eps)
    xh = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).view(n, hw, c)
    h = xh * gamma.double() + beta.double()
    return act64(h, act), mean, rstd, xh, h


NORMS = [  # n, hw, c, groups
    (1, 1, 64, 2), (2, 49, 20, 4), (3, 64, 256, 32), (5, 17, 100, 4), (2, 1024, 64, 8), (1, 16384, 32, 1), (7, 9, 33, 1), (4, 3136, 96, 4),
    (300, 16, 8, 8), (2, 100, 768, 3), (1, 30, 5000, 1), (2, 500, 1056, 32), (33, 4, 512, 16), (3, 256, 513, 27),
]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n,hw,c,groups", NORMS)
def test_group_norm(dtype, n, hw, c, groups):
    act = ["none", "relu", "gelu", "silu"][(n + hw + c) % 4]
    pad = [0, 5, 8][(hw + groups) % 3]
    x = randn(n, hw, c, seed=1, dtype=dtype, pad=pad)
    x.mul_(randn(c, seed=2, dtype=dtype)).add_(randn(c, seed=3, dtype=dtype))
    gamma, beta = randn(c, seed=4) + 1, randn(c, seed=5)
    r = tr.group_norm(x, groups, gamma, beta, 1e-5, act, save_x8=True, save_y8=True)
    y, mean, rstd, xh, h = norm64(x, groups, gamma, beta, 1e-5, act)
    spread = torch.nn.functional.pad(x.double().abs(), (0, 0)).view(n, hw, groups, -1).amax((1, 3))
    # sums of at most ~ hw / 8 + 64 terms in fp32, about values of the channel; rstd carries half the variance's error
    adds = (hw / 8 + c / groups + 64) * 2.0 ** -24
    assert_within(r.mean, mean, spread * adds * 2, "mean")
    assert_within(r.rstd, rstd, rstd * adds * 4, "rstd")
    wide = lambda t: t.repeat_interleave(c // groups, 1)[:, None, :]
    err = (xh.abs() * adds * 4 + wide(spread * rstd) * adds * 2 + 2.0 ** -21 * (1 + xh.abs())) * gamma.double().abs() * 1.2 + 2.0 ** -21 * (1 + beta.double().abs())
    assert_within(r.y, y, y.abs() * U[dtype] * 1.01 + err + TINY[dtype], "y")
    for got, src in ((r.x8, x), (r.y8, r.y)):
        want = tr.pack8(src.reshape(n * hw, c))
        assert torch.equal(got.codes, want.codes) and torch.equal(got.exps, want.exps)


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n,hw,c,groups", NORMS[1:])
def test_group_norm_grad(dtype, packed, n, hw, c, groups):
    act = ["none", "relu", "gelu", "silu"][(n + hw + c) % 4]
    pad = [0, 5, 8][(hw + groups) % 3]
    dy = randn(n, hw, c, seed=6, dtype=dtype, pad=pad)
    x = randn(n, hw, c, seed=1, dtype=dtype) * 2 + 0.5
    gamma, beta = randn(c, seed=4) + 1, randn(c, seed=5)
    arg = tr.pack8(x.reshape(n * hw, c)) if packed else x
    x64 = (tr.unpack8(arg, F32).view(n, hw, c) if packed else x).double()
    _, mean, rstd, _, _ = norm64(x64, groups, gamma, beta, 1e-5, act)
    mean, rstd = mean.float(), rstd.float()
    dx, dgamma, dbeta = tr.group_norm_grad(dy, arg, groups, gamma, beta, mean, rstd, act)
    k = c // groups
    wide = lambda t: t.double().repeat_interleave(k, 1)[:, None, :]
    xh = (x64 - wide(mean)) * wide(rstd)
    h = xh * gamma.double() + beta.double()
    dh = dy.double() * slope64(h, act)
    # the slope at an h that is 2^-21 (1 + |h|) off (|act''| < 1.2); relu's jumps where |h| is that small
    dslope = 1.2 * 2.0 ** -21 * (1 + h.abs() + xh.abs()) + 2.0 ** -20
    if act == "relu":
        dslope = dslope + (h.abs() < 2.0 ** -18).double()
    e = dy.double().abs() * dslope + dh.abs() * 2.0 ** -22
    adds = (hw / 8 + n / 8 + 200) * 2.0 ** -24
    exh = 2.0 ** -22 * (xh.abs() + (wide(mean) * wide(rstd)).abs() + 1)
    assert_within(dbeta, dh.sum((0, 1)), (e + adds * dh.abs()).sum((0, 1)) + 1e-30, "dbeta")
    assert_within(dgamma, (dh * xh).sum((0, 1)), (e * xh.abs() + dh.abs() * exh + adds * (dh * xh).abs()).sum((0, 1)) + 1e-30, "dgamma")
    u = dh * gamma.double()
    over = lambda t: wide(t.view(n, hw, groups, k).mean((1, 3)))
    want = wide(rstd) * (u - over(u) - xh * over(u * xh))
    eu = e * gamma.double().abs() + u.abs() * 2.0 ** -22
    bound = wide(rstd) * (eu + over(eu + (adds + k * 2.0 ** -24) * u.abs()) + xh.abs() * over(eu * xh.abs() + u.abs() * exh + (adds + k * 2.0 ** -24) * (u * xh).abs())
                          + exh * over(u * xh).abs() + 2.0 ** -22 * (u.abs() + over(u).abs() + (xh * over(u * xh)).abs()))
    assert_within(dx, want, want.abs() * U[dtype] * 1.01 + bound * 1.01 + TINY[dtype], "dx")


def test_group_norm_of_constant_and_distant_values():
    x = torch.full((2, 100, 64), 3.0, device=DEV)
    g, b = torch.ones(64, device=DEV), torch.full((64,), 0.5, device=DEV)
    r = tr.group_norm(x, 4, g, b)
    assert torch.equal(r.y, torch.full_like(x, 0.5)) and torch.equal(r.mean, torch.full_like(r.mean, 3.0))
    x = randn(2, 4096, 64, seed=1) + 10000.0            # a mean 10^4 deviations away cancels nothing
    r = tr.group_norm(x, 4, g, b)
    y, mean, rstd, xh, _ = norm64(x, 4, g, b, 1e-5, "none")
    assert_within(r.rstd, rstd, rstd * 1e-4, "rstd")
    assert_within(r.y, y, 1e-2, "y")


def test_group_norm_keeps_nan_in_its_group():
    x = randn(3, 50, 64, seed=1)
    x[1, 7, 20] = math.nan
    g, b = torch.ones(64, device=DEV), torch.zeros(64, device=DEV)
    r = tr.group_norm(x, 8, g, b)
    assert torch.isnan(r.y[1, :, 16:24]).all() and torch.isnan(r.mean[1, 2])
    bad = torch.isnan(r.y)
    assert int(bad.sum()) == 50 * 8


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_group_norm_grad_against_differences(act):
    n, hw, c, groups = 2, 30, 24, 3
    x8, x = kept(n * hw, c, 3)
    x = x.view(n, hw, c)
    gamma, beta = randn(c, seed=4) + 1, randn(c, seed=5)
    dy = randn(n, hw, c, seed=6)
    f = lambda x, ga, be: (norm64(x, groups, ga, be, 1e-5, act)[0] * dy.double()).sum()
    _, mean, rstd, _, _ = norm64(x, groups, gamma, beta, 1e-5, act)
    dx, dgamma, dbeta = tr.group_norm_grad(dy, x8, groups, gamma, beta, mean.float().contiguous(), rstd.float().contiguous(), act)
    h = 1e-4
    vx, vg, vb = randn(n, hw, c, seed=7).double(), randn(c, seed=8).double(), randn(c, seed=9).double()
    ga, be = gamma.double(), beta.double()
    for got, diff in (((dx.double() * vx).sum(), (f(x + h * vx, ga, be) - f(x - h * vx, ga, be)) / (2 * h)),
                      ((dgamma.double() * vg).sum(), (f(x, ga + h * vg, be) - f(x, ga - h * vg, be)) / (2 * h)),
                      ((dbeta.double() * vb).sum(), (f(x, ga, be + h * vb) - f(x, ga, be - h * vb)) / (2 * h))):
        assert abs((got - diff).item()) <= 2e-4 * max(1.0, abs(diff.item()), float(dy.double().norm()))


# ------------------------------------------------------------------------------------------------- streams, graphs, refusals

def test_operators_on_another_stream_and_in_a_graph():
    x, w = randn(300, 200, seed=1, dtype=BF), randn(96, 200, seed=2, dtype=BF)
    g, b = torch.ones(96, device=DEV), torch.zeros(96, device=DEV)

    def step(x):
        r = tr.linear(x, w, act="silu", save_z8=True)
        nrm = tr.group_norm(r.y.view(3, 100, 96), 4, g, b, act="gelu", save_x8=True)
        dx, dg, db = tr.group_norm_grad(nrm.y, nrm.x8, 4, g, b, nrm.mean, nrm.rstd, act="gelu")
        dz, dbias = tr.act_grad(dx.view(300, 96), r.z8, "silu")
        return [nrm.y, dg, db, dbias, tr.linear_grad_input(dz, w), tr.linear_grad_weight(dz, tr.pack8(x))]
    want = [t.clone() for t in step(x)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(x)
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip(got, want):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    held = x.clone()
    with torch.cuda.graph(graph):
        out = step(held)
    held.zero_()
    graph.replay()
    held.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    for p, q in zip(out, want):
        assert torch.equal(p, q)


def test_layers_train_and_hand_their_gradients_to_a_round():
    """norm_layer -> linear_layer -> linear_layer + skip: gradients near those of the same net in 64 bits (the 8-bit
    activations are the difference), and one round takes them."""
    torch.manual_seed(0)
    c, hid, n, hw = 64, 128, 4, 64
    x = randn(n, hw, c, seed=1, dtype=BF).requires_grad_(True)
    par = [torch.ones(c, device=DEV), torch.zeros(c, device=DEV), randn(hid, c, seed=2, scale=c ** -0.5), torch.zeros(hid, device=DEV),
           randn(c, hid, seed=3, scale=hid ** -0.5), torch.zeros(c, device=DEV)]
    par = [p.requires_grad_(True) for p in par]
    ga, be, w1, b1, w2, b2 = par
    keep = []
    h = tr.norm_layer(x, ga, be, 8, act="silu", keep=keep)
    a = tr.linear_layer(h.view(n * hw, c), w1, b1, act="gelu", x8=keep[0])
    y = tr.linear_layer(a, w2, b2, residual=x.view(n * hw, c))
    t = randn(n * hw, c, seed=9, dtype=BF)
    (y * t).sum().backward()
    x64 = x.detach().double().requires_grad_(True)
    p64 = [p.detach().double().requires_grad_(True) for p in par]
    hh = norm64_grad(x64, 8, p64[0], p64[1])
    aa = torch.nn.functional.gelu(hh.view(n * hw, c) @ p64[2].t() + p64[3])
    yy = aa @ p64[4].t() + p64[5] + x64.view(n * hw, c)
    (yy * t.double()).sum().backward()
    for got, want in zip([x] + par, [x64] + p64):
        rel = ((got.grad.double() - want.grad).norm() / want.grad.norm()).item()
        assert rel < 0.03, rel
    layers = [tuple(w1.shape), tuple(w2.shape)]
    comp = B.LQSGD(layers, 2, 4)
    ghat = [torch.empty_like(w1), torch.empty_like(w2)]
    comp.step([[w1.grad, w2.grad]], ghat)
    torch.cuda.synchronize()
    assert all(torch.isfinite(g).all() for g in ghat) and comp.status() == [0, 0]


def norm64_grad(x, groups, gamma, beta):
    n, hw, c = x.shape
    v = x.view(n, hw, groups, c // groups)
    mean, var = v.mean((1, 3), keepdim=True), v.var((1, 3), unbiased=False, keepdim=True)
    h = ((v - mean) / torch.sqrt(var + 1e-5)).view(n, hw, c) * gamma + beta
    return h * torch.sigmoid(h)


def test_refusals():
    x, w = randn(8, 16, dtype=BF), randn(4, 16, dtype=BF)
    with pytest.raises(ValueError):
        tr.linear(x.float(), w.float())
    with pytest.raises(ValueError):
        tr.linear(x, w.half())
    with pytest.raises(ValueError):
        tr.linear(x, randn(4, 15, dtype=BF))
    with pytest.raises(ValueError):
        tr.linear(x, w, act="tanh")
    with pytest.raises(ValueError):
        tr.linear(x, w, bias=torch.zeros(4, dtype=BF, device=DEV))
    with pytest.raises(ValueError):
        tr.linear(x.t(), w)
    with pytest.raises(ValueError):
        tr.linear(x.cpu(), w)
    with pytest.raises(ValueError):
        tr.linear_grad_weight(randn(8, 4, dtype=BF), x, accumulate=True)
    with pytest.raises(ValueError):
        tr.act_grad(x, None, "gelu")
    with pytest.raises(ValueError):
        tr.Packed8(torch.zeros(4, 64, dtype=torch.uint8, device=DEV), torch.zeros(4, 3, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        tr.group_norm(randn(2, 4, 4, 8, dtype=BF)[:, :, ::2].transpose(1, 2), 2, torch.ones(8, device=DEV), torch.zeros(8, device=DEV))
    with pytest.raises(B.LqsgdError) as e:
        tr.group_norm(randn(2, 4, 8, dtype=BF), 3, torch.ones(8, device=DEV), torch.zeros(8, device=DEV))
    assert e.value.code == B.ERR_BAD_SHAPE
    with pytest.raises(B.LqsgdError) as e:
        tr.group_norm(randn(2, 4, 8, dtype=BF), 2, torch.ones(8, device=DEV), torch.zeros(8, device=DEV), eps=0.0)
    assert e.value.code == B.ERR_INVALID_ARG
