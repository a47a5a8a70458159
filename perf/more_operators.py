"""What is measured of the operators of a pre-norm residual block: RMS norm, dropout, and linear layers in 8-bit integers.

A block takes the output of its last layer, drops some of it, adds the residual stream, normalises each row (a token) and
multiplies it, in 8 bits, by the next layer's weights.  Every case is one call that such a program makes:

  rms       h = residual + dropout(x), y = gamma h rstd, rstd = 1 / sqrt(mean(h^2) + eps); on request y or h also in the
            8-bit form of kept activations ("y8", "h8"), y also in rows of signed 8-bit codes ("rows8")
  rms_grad  the gradients of x, of the residual and of gamma, h read in its own type or from its 8-bit form
  dropout   residual + dropout(x), the mask from a counter-based generator
  rows8     x to rows of signed 8-bit codes with one scale each, and back
  linear8   y = act((sum over k of x and w's codes) sx sw + bias) + residual; "save" also the pre-activation in 8 bits

Rows of signed codes: top = max |x| of the row, the scale is max(top / 127, 2^-120), a code rint(x min(127 / top, 2^120)), halves to
even.  A row with a value that is not finite has the scale NaN and codes 0.

The 8-bit form of kept activations: each row is cut into groups of 32 columns (the last may be shorter).  A group has one exponent
e, the smallest with rint(max |x| / 2^e) <= 127 and e >= -126, stored as the byte e + 126; a value is a sign bit (128, set for x < 0)
and the magnitude rint(|x| / 2^e), halves to even.  Every value it stands for is exact in bf16.

Dropout: a value is kept where its 16 random bits are at least T = min(rint(65536 p), 65535), and is then multiplied by
65536 / (65536 - T); the others are 0.  The bits of row r, column c: Philox4x32 with 10 rounds (Salmon et al., 2011), the key is the
64-bit seed, the counter's low half r ceil(cols / 8) + c / 8 and its high half the offset; word (c mod 8) / 2, its low half first.
"""
import math

import torch

own = False          # False: the plain forms; True: the framework's operators

GROUP = 32
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # one token between two layers of a network that answers: nothing but latency
        dict(name="rms_token", op="rms", rows=1, cols=4096, residual=True, p=0.0, y=False, y8=False, h8=False, rows8=True, dtype="bf16", pad=0),
        # the same place in training: dropout, the residual stream, the norm, both kept copies
        dict(name="rms_train", op="rms", rows=8192, cols=4096, residual=True, p=0.1, y=True, y8=True, h8=True, rows8=False, dtype="bf16", pad=0),
        # wide flattened features of an odd length, into 8-bit integers
        dict(name="rms_wide_odd", op="rms", rows=1021, cols=25087, residual=False, p=0.0, y=True, y8=False, h8=False, rows8=True, dtype="fp16", pad=1),
        # the backward pass of rms_train
        dict(name="rms_grad_train", op="rms_grad", rows=8192, cols=4096, skip=True, kept=True, p=0.1, dtype="bf16", pad=0),
        # the backward pass of a narrow norm in fp32, an uneven batch
        dict(name="rms_grad_odd", op="rms_grad", rows=250, cols=577, skip=False, kept=False, p=0.0, dtype="fp32", pad=1),
        # dropout on the hidden activations of a large feed-forward block
        dict(name="dropout_large", op="dropout", rows=8192, cols=16384, residual=False, p=0.1, dtype="bf16", pad=0),
        # dropout before the residual's addition on rows that are not 16-byte aligned
        dict(name="dropout_odd", op="dropout", rows=1021, cols=25087, residual=True, p=0.5, dtype="fp32", pad=0),
        # a large layer's fp32 weights into 8-bit integers, once a step
        dict(name="rows8_weights", op="rows8", rows=16384, cols=4096, dtype="fp32", pad=0),
        # a small batch's activations
        dict(name="rows8_small", op="rows8", rows=250, cols=3136, dtype="bf16", pad=0),
        # one token through the first half of a large feed-forward block: the weights' bytes are the cost
        dict(name="linear8_token", op="linear8", rows=1, cin=4096, cout=16384, act="silu", residual=False, save=False, dtype="bf16", pad=0),
        # an uneven batch through an odd layer, with the residual
        dict(name="linear8_uneven", op="linear8", rows=1021, cin=4097, cout=1000, act="none", residual=True, save=False, dtype="fp16", pad=0),
        # the first half of a large feed-forward block in training
        dict(name="linear8_large", op="linear8", rows=8192, cin=4096, cout=16384, act="gelu", residual=False, save=True, dtype="bf16", pad=0),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rms", "rms", "rms_grad", "rms_grad", "dropout", "rows8", "linear8", "linear8", "linear8"])
    case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16"] + ["fp32"] * (op != "linear8")), pad=rng.choice([0, 0, 0, 1, 8]))
    rows = _log_int(rng, 1, 16384)
    if op == "linear8":
        case.update(rows=rows, cin=_log_int(rng, 8, 16384), cout=_log_int(rng, 8, 16384), residual=rng.random() < 0.5,
                    act=rng.choice(["none", "relu", "gelu", "silu"]), save=rng.random() < 0.3)
        if rng.random() < 0.6:               # real layers mostly have round widths, batches any size
            case.update(cin=max(16, case["cin"] // 16 * 16), cout=max(16, case["cout"] // 16 * 16))
        while case["rows"] * case["cin"] * case["cout"] > 8192 * 4096 * 16384:
            case["rows"] = (case["rows"] + 1) // 2
        return case
    case.update(rows=rows, cols=_log_int(rng, 32, 25088))
    if rng.random() < 0.5:
        case["cols"] = case["cols"] // 8 * 8
    most = 8192 * 4096 if op in ("rms", "rms_grad") else 8192 * 8192
    while case["rows"] * case["cols"] > most:
        case["rows"] = (case["rows"] + 1) // 2
    if op == "rms":
        case.update(residual=rng.random() < 0.7, p=rng.choice([0.0, 0.1, 0.37]), y8=rng.random() < 0.3, h8=rng.random() < 0.3, rows8=rng.random() < 0.5)
        case["y"] = not case["rows8"] or case["y8"] or rng.random() < 0.5
    elif op == "rms_grad":
        case.update(skip=rng.random() < 0.7, kept=rng.random() < 0.5, p=rng.choice([0.0, 0.1, 0.37]))
    elif op == "dropout":
        case.update(residual=rng.random() < 0.5, p=rng.choice([0.05, 0.1, 0.37, 0.5]))
    return case


# ------------------------------------------------------------------------------------------------------------ inputs

def _matrix(gen, rows, cols, dtype, scale, pad):
    """rows x cols of N(0, scale^2), as the left part of a wider buffer where pad > 0."""
    wide = torch.randn((rows, cols + pad), generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)
    return wide[:, :cols]


def _vector(gen, n, mean, scale):
    return torch.randn(n, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).add_(mean)


def _power(e):
    """2^e as float32, exactly, for whole -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _to_codes(x):
    """The 8-bit form of kept activations of x (rows x cols) as two byte tensors: the codes and the exponents."""
    rows, cols = x.shape
    groups = (cols + GROUP - 1) // GROUP
    v = torch.zeros((rows, groups * GROUP), device=x.device, dtype=torch.float32)
    v[:, :cols] = x.float()
    v = v.view(rows, groups, GROUP)
    top = v.abs().amax(dim=2, keepdim=True)
    finite = torch.isfinite(top)
    top = torch.where(finite, top, torch.zeros_like(top))
    e = torch.frexp(top)[1] - 7                                   # 64 <= top / 2^e < 128
    e = torch.where(top == 0, torch.full_like(e, -126), e).clamp_(min=-126)
    e = e + (torch.round(top * _power(-e)) > 127)
    mag = torch.round(v.abs() * _power(-e)).to(torch.uint8)
    codes = torch.where(v < 0, mag + 128, mag).view(rows, -1)[:, :cols].contiguous()
    exps = torch.where(finite, e + 126, torch.full_like(e, 255)).to(torch.uint8).view(rows, groups)
    return codes, exps


def _from_codes(codes, exps):
    """The values, fp32, that the 8-bit form of kept activations stands for."""
    rows, cols = codes.shape
    e = exps.to(torch.int32).unsqueeze(2)
    v = torch.nn.functional.pad(codes, (0, -cols % GROUP)).view(rows, -1, GROUP)
    mag = (v & 127).float()
    v = torch.where(v >= 128, -mag, mag) * _power(e.clamp(max=248) - 126)
    v = torch.where(e == 255, torch.full_like(v, math.nan), v)
    return v.view(rows, -1)[:, :cols].contiguous()


def _to_rows8(x):
    """x as rows of signed 8-bit codes: the codes, int8, and the scales, fp32."""
    v = x.float()
    top = v.abs().amax(dim=1)
    finite = torch.isfinite(top)
    inv = torch.clamp(127.0 / top, max=2.0 ** 120)
    scales = torch.where(finite, torch.clamp(top / 127.0, min=2.0 ** -120), torch.full_like(top, math.nan))
    codes = torch.round(torch.where(finite[:, None], v * inv[:, None], torch.zeros_like(v))).to(torch.int8)
    return codes, scales


def _laid_out(codes, pad):
    """Rows of codes as a program keeps them: each starts on a 16-byte boundary (pad 0), or `pad` bytes more lie between them."""
    rows, cols = codes.shape
    wide = torch.zeros((rows, (cols + 15) // 16 * 16 if pad == 0 else cols + pad), device=codes.device, dtype=torch.int8)
    wide[:, :cols] = codes
    return wide[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dt, pad = case["op"], DTYPES[case["dtype"]], case["pad"]
    s = dict(case, dt=dt, seed=(seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 62, offset=seed % 1000)
    if op == "linear8":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        xc, s["sx"] = _to_rows8(_matrix(gen, rows, cin, torch.float32, 1.0, 0))
        wc, s["sw"] = _to_rows8(_matrix(gen, cout, cin, torch.float32, 1 / math.sqrt(cin), 0))
        s["xc"], s["wc"] = _laid_out(xc, pad), _laid_out(wc, 0)
        s["bias"] = _vector(gen, cout, 0.0, 0.1)
        s["res"] = _matrix(gen, rows, cout, dt, 1.0, pad) if case["residual"] else None
        return s
    rows, cols = case["rows"], case["cols"]
    if op == "rms":
        s["x"] = _matrix(gen, rows, cols, dt, 0.7, pad)
        s["res"] = _matrix(gen, rows, cols, dt, 1.5, 0) if case["residual"] else None
        s["gamma"] = _vector(gen, cols, 1.0, 0.2)
    elif op == "rms_grad":
        s["dy"] = _matrix(gen, rows, cols, dt, 0.05, pad)
        s["skip_grad"] = _matrix(gen, rows, cols, dt, 0.05, 0) if case["skip"] else None
        s["gamma"] = _vector(gen, cols, 1.0, 0.2)
        h = _matrix(gen, rows, cols, dt, 1.5, 0)
        if case["kept"]:
            s["codes"], s["exps"] = _to_codes(h)
            h = _from_codes(s["codes"], s["exps"])
        else:
            s["h"] = h
        h = h.float()
        s["rstd"] = 1 / torch.sqrt((h * h).mean(dim=1) + EPS)               # the forward pass's
    elif op == "dropout":
        s["x"] = _matrix(gen, rows, cols, dt, 1.0, pad)
        s["res"] = _matrix(gen, rows, cols, dt, 1.0, 0) if case["residual"] else None
    else:
        t = torch.randn((rows, 1), generator=gen, device="cuda").exp_()      # rows of different size
        s["x"] = torch.cat([_matrix(gen, rows, cols, torch.float32, 1.0, 0) * t, t.expand(rows, pad)], 1).to(dt)[:, :cols]
    return s


# --------------------------------------------------------------------------------------------------------- the plain forms

def _act(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _philox(c0, c1, c2, c3, k0, k1):
    """Ten rounds on words held in int64 (products wrap modulo 2^64, as they should)."""
    low = 0xFFFFFFFF
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _threshold(p):
    return min(int(round(65536 * p)), 65535)


def _factor(s, rows, cols):
    """What dropout multiplies by: 0 or 65536 / (65536 - T)."""
    t = _threshold(s["p"])
    n = torch.arange(rows * ((cols + 7) // 8), device="cuda", dtype=torch.int64)
    off, seed = torch.full_like(n, s["offset"]), s["seed"]
    words = torch.stack(_philox(n & 0xFFFFFFFF, n >> 32, off & 0xFFFFFFFF, off >> 32, seed & 0xFFFFFFFF, seed >> 32), dim=1)
    bits = torch.stack((words & 0xFFFF, words >> 16), dim=2).view(rows, -1)[:, :cols]
    return (bits >= t).to(torch.float32) * (65536 / (65536 - t))


def _plain(s):
    op, dt = s["op"], s["dt"]
    if op == "linear8":
        z = (s["xc"].float() @ s["wc"].float().t()) * s["sx"][:, None] * s["sw"] + s["bias"]
        y = _act(z, s["act"])
        if s["res"] is not None:
            y = y + s["res"].float()
        out = {"y": y.to(dt)}
        if s["save"]:
            out["z8"] = _from_codes(*_to_codes(z)).to(torch.bfloat16)
        return out
    if op == "rows8":
        codes, scales = _to_rows8(s["x"])
        return {"x8": (codes.float() * scales[:, None]).to(torch.bfloat16), "scales": scales}
    rows, cols = s["rows"], s["cols"]
    if op == "dropout":
        y = s["x"].float() * _factor(s, rows, cols)
        if s["res"] is not None:
            y = y + s["res"].float()
        return {"y": y.to(dt)}
    if op == "rms":
        h, out = s["x"].float(), {}
        if s["p"] > 0:
            h = h * _factor(s, rows, cols)
        if s["res"] is not None:
            h = h + s["res"].float()
        if s["p"] > 0 or s["res"] is not None:
            out["h"] = h.to(dt)
            h = out["h"].float()
        out["rstd"] = 1 / torch.sqrt((h * h).mean(dim=1) + EPS)
        y = h * out["rstd"][:, None] * s["gamma"]
        if s["y"]:
            out["y"] = y.to(dt)
        if s["h8"]:
            out["h8"] = _from_codes(*_to_codes(h)).to(torch.bfloat16)
        if s["y8"]:
            out["y8"] = _from_codes(*_to_codes(y.to(dt))).to(torch.bfloat16)
        if s["rows8"]:
            codes, out["scales"] = _to_rows8(y)
            out["rows8"] = (codes.float() * out["scales"][:, None]).to(torch.bfloat16)
        return out
    h = _from_codes(s["codes"], s["exps"]) if s["kept"] else s["h"].float()
    xh, dy = h * s["rstd"][:, None], s["dy"].float()
    g = dy * s["gamma"]
    d = s["rstd"][:, None] * (g - xh * (g * xh).mean(dim=1, keepdim=True))
    if s["skip_grad"] is not None:
        d = d + s["skip_grad"].float()
    out = {"dx": d.to(dt), "dgamma": (dy * xh).sum(dim=0)}
    if s["p"] > 0:
        out["dresidual"] = out["dx"]
        out["dx"] = (d * _factor(s, rows, cols)).to(dt)
    return out


# ------------------------------------------------------------------------------------------------- the framework's operators

def _own(s):
    from paper_2506_17974_b200 import training as tr
    op = s["op"]
    if op == "linear8":
        r = tr.linear_rows8(tr.Rows8(s["xc"], s["sx"]), tr.Rows8(s["wc"], s["sw"]), s["bias"], act=s["act"], residual=s["res"], dtype=s["dt"],
                            save_z8=s["save"])
        return {"y": r.y, "z8": tr.unpack8(r.z8, torch.bfloat16)} if s["save"] else {"y": r.y}
    if op == "rows8":
        r = tr.pack_rows8(s["x"])
        return {"x8": tr.unpack_rows8(r, torch.bfloat16), "scales": r.scales}
    if op == "dropout":
        return {"y": tr.dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s["res"])}
    if op == "rms":
        r = tr.rms_norm(s["x"], s["gamma"], eps=EPS, residual=s["res"], p=s["p"], seed=s["seed"], offset=s["offset"], want_y=s["y"],
                        save_h8=s["h8"], save_y8=s["y8"], save_rows8=s["rows8"])
        out = {"rstd": r.rstd}
        if s["p"] > 0 or s["res"] is not None:
            out["h"] = r.h
        if s["y"]:
            out["y"] = r.y
        if s["h8"]:
            out["h8"] = tr.unpack8(r.h8, torch.bfloat16)
        if s["y8"]:
            out["y8"] = tr.unpack8(r.y8, torch.bfloat16)
        if s["rows8"]:
            out["scales"], out["rows8"] = r.rows8.scales, tr.unpack_rows8(r.rows8, torch.bfloat16)
        return out
    h = tr.Packed8(s["codes"], s["exps"]) if s["kept"] else s["h"]
    dx, dresidual, dgamma = tr.rms_norm_grad(s["dy"], h, s["gamma"], s["rstd"], skip=s["skip_grad"], p=s["p"], seed=s["seed"], offset=s["offset"])
    out = {"dx": dx, "dgamma": dgamma}
    if s["p"] > 0:
        out["dresidual"] = dresidual
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------- costs

def work(case):
    op, b = case["op"], SIZE[case["dtype"]]
    kept = lambda r, c: r * c + r * ((c + GROUP - 1) // GROUP)                     # noqa: E731  bytes of a kept 8-bit form
    if op == "linear8":
        m, k, n = case["rows"], case["cin"], case["cout"]
        by = m * k + n * k + b * m * n * (2 if case["residual"] else 1) + 4 * m + 8 * n + (2 * m * n if case["save"] else 0)
        return {"bytes": by, "flops": 2 * m * n * k}
    m, n = case["rows"], case["cols"]
    if op == "rows8":
        return {"bytes": m * n * (b + 2) + 4 * m, "flops": 4 * m * n}
    if op == "dropout":
        return {"bytes": m * n * b * (3 if case["residual"] else 2), "flops": 2 * m * n}
    if op == "rms":
        summed = case["residual"] or case["p"] > 0
        by = m * n * (b * (1 + case["residual"] + summed + case["y"]) + 2 * (case["y8"] + case["h8"] + case["rows8"])) + 4 * n + 4 * m * (1 + case["rows8"])
        return {"bytes": by, "flops": 8 * m * n}
    by = b * m * n * (2 + case["skip"] + (case["p"] > 0)) + (kept(m, n) if case["kept"] else b * m * n) + 8 * n + 4 * m
    return {"bytes": by, "flops": 10 * m * n}


# --------------------------------------------------------------------------------------------------- the definition in 64 bits

def _act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * (0.5 * torch.special.erfc(-z / math.sqrt(2)))
    return z


def _kept64(x):
    """What the 8-bit form of kept activations of x stands for, every step in 64 bits."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % GROUP)).reshape(rows, -1, GROUP)
    top = v.abs().max(dim=2, keepdim=True).values
    half = torch.frexp(top.clamp(min=1e-300))[1].long() - 1                                # 2^half <= top < 2^(half + 1)
    step = ((half - 6 + 1023) << 52).view(torch.float64)
    step = torch.where(top / step >= 127.5, step * 2, step).clamp(min=2.0 ** -126)
    return (torch.round(v / step) * step).reshape(rows, -1)[:, :cols]


def _decode64(codes, exps):
    e = exps.long().repeat_interleave(GROUP, dim=1)[:, :codes.shape[1]] - 126
    return codes.bitwise_and(127).double() * ((e + 1023) << 52).view(torch.float64) * (1 - 2 * (codes >> 7).double())


def _rows64(x):
    """What rows of signed codes stand for, and their scales, every step in 64 bits."""
    step = (x.double().abs().max(dim=1, keepdim=True).values / 127).clamp(min=2.0 ** -120)
    return torch.round(x.double() / step) * step, step[:, 0]


def _times(a, m):
    """The high and the low word of a m, a in words and m < 2^32, from products of half words."""
    ah, al, mh, ml = a >> 16, a & 0xFFFF, m >> 16, m & 0xFFFF
    low = al * ml
    mid = ah * ml + (low >> 16)
    mid2 = al * mh + (mid & 0xFFFF)
    return ah * mh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)


def _kept_by_dropout(s, rows, cols):
    blocks = (cols + 7) // 8
    block = torch.arange(blocks, device="cuda")[None, :] + blocks * torch.arange(rows, device="cuda")[:, None]
    ctr = [block % 2 ** 32, block // 2 ** 32, torch.full_like(block, s["offset"] % 2 ** 32), torch.full_like(block, s["offset"] // 2 ** 32)]
    for r in range(10):
        key = [(s["seed"] % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32]
        h0, l0 = _times(ctr[0], 0xD2511F53)
        h1, l1 = _times(ctr[2], 0xCD9E8D57)
        ctr = [h1 ^ ctr[1] ^ key[0], l1, h0 ^ ctr[3] ^ key[1], l0]
    keep = torch.empty((rows, 8 * blocks), device="cuda", dtype=torch.bool)
    t = min(round(65536 * s["p"]), 65535)
    for i in range(8):
        keep[:, i::8] = (ctr[i // 2] // 2 ** (16 * (i % 2))) % 65536 >= t
    return keep[:, :cols], 65536 / (65536 - t)


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "linear8":
        z = torch.mm(s["xc"].double(), s["wc"].double().t()).mul_(s["sx"].double()[:, None]).mul_(s["sw"].double()).add_(s["bias"].double())
        out = {"z8": _kept64(z)} if s["save"] else {}
        y = _act64(z, s["act"])
        return {"y": y if s["res"] is None else y.add_(s["res"].double()), **out}
    if op == "rows8":
        x8, scales = _rows64(s["x"])
        return {"x8": x8, "scales": scales}
    rows, cols = s["rows"], s["cols"]
    if s["p"] > 0:
        keep, scale = _kept_by_dropout(s, rows, cols)
        drop = lambda t: torch.where(keep, t * scale, torch.zeros((), dtype=t.dtype, device=t.device))     # noqa: E731
    else:
        drop = lambda t: t                                                                                 # noqa: E731
    if op == "dropout":
        y = drop(s["x"].double())
        return {"y": y if s["res"] is None else y.add_(s["res"].double())}
    if op == "rms":
        h, out = drop(s["x"].double()), {}
        if s["res"] is not None:
            h = h + s["res"].double()
        if s["p"] > 0 or s["res"] is not None:
            out["h"] = h
            h = h.to(s["dt"]).double()                           # the norm is of h as it is returned
        out["rstd"] = (h.square().mean(dim=1) + EPS).rsqrt()
        y = h * out["rstd"][:, None] * s["gamma"].double()
        if s["y"]:
            out["y"] = y
        if s["h8"]:
            out["h8"] = _kept64(h)
        if s["y8"]:
            out["y8"] = _kept64(y.to(s["dt"]))                   # of y as it is returned
        if s["rows8"]:
            out["rows8"], out["scales"] = _rows64(y)
        return out
    h = _decode64(s["codes"], s["exps"]) if s["kept"] else s["h"].double()
    xh, dy, r = h * s["rstd"].double()[:, None], s["dy"].double(), s["rstd"].double()[:, None]
    u = dy * s["gamma"].double()
    d = r * u - r * xh * (torch.einsum("rc,rc->r", u, xh) / cols)[:, None]
    if s["skip_grad"] is not None:
        d = d + s["skip_grad"].double()
    out = {"dx": drop(d), "dgamma": torch.einsum("rc,rc->c", dy, xh)}
    if s["p"] > 0:
        out["dresidual"] = d
    return out
