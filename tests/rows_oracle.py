"""Plain numpy forms, in 64 bits, of the operators on whole rows: dropout's generator, RMS norm, rows of signed 8-bit codes."""
import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = 0xFFFFFFFF


def philox(ctr, key):
    """One call of Philox4x32-10 on Python numbers."""
    c, k = list(ctr), list(key)
    for _ in range(10):
        a, b = M0 * c[0], M1 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & LOW, (a >> 32) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + W0) & LOW, (k[1] + W1) & LOW]
    return tuple(c)


def threshold(p):
    """Of p as the library has it, in 32 bits; halves to even."""
    return min(int(np.rint(65536 * np.float64(np.float32(p)))), 65535)


def kept(rows, cols, p, seed, offset, row0=0):
    """Which values dropout keeps, bool rows x cols, from row row0 on."""
    blocks = (cols + 7) // 8
    b = np.arange(row0 * blocks, (row0 + rows) * blocks, dtype=np.uint64)
    low, seed, offset = np.uint64(LOW), seed % 2 ** 64, offset % 2 ** 64
    c = [b & low, b >> np.uint64(32), np.full_like(b, offset & LOW), np.full_like(b, offset >> 32)]
    k0, k1 = seed & LOW, seed >> 32
    for _ in range(10):
        x, y = np.uint64(M0) * c[0], np.uint64(M1) * c[2]
        c = [(y >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), y & low, (x >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), x & low]
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    words = np.stack(c, 1)
    bits = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 2).reshape(rows, blocks * 8)[:, :cols]
    return bits >= np.uint64(threshold(p))


def dropped(x, p, seed, offset, residual=None):
    """residual + dropout(x) in 64 bits; the factor as the library has it, in 32."""
    x = np.asarray(x, np.float64)
    if p > 0:
        scale = np.float64(np.float32(65536 / (65536 - threshold(p))))
        x = np.where(kept(*x.shape, p, seed, offset), x * scale, 0.0)
    return x if residual is None else x + np.asarray(residual, np.float64)


def rms_grad(dy, h, gamma, rstd, skip=None):
    """(d, dgamma) in 64 bits."""
    xh, u = h * rstd[:, None], dy * gamma
    d = rstd[:, None] * (u - xh * (u * xh).mean(1, keepdims=True))
    return (d if skip is None else d + skip), (dy * xh).sum(0)


def rows8(x):
    """(codes, scales) of float32 x, in float32 as the definition has it."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(1).astype(np.float32)
    fine = np.isfinite(top)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        scale = np.maximum(top / np.float32(127), np.float32(2.0 ** -120))
        inv = np.minimum(np.float32(127) / top, np.float32(2.0 ** 120))
        codes = np.rint(np.where(fine[:, None], x, np.float32(0)) * np.where(fine, inv, np.float32(0))[:, None])
    return codes.astype(np.int8), np.where(fine, scale, np.float32(np.nan)).astype(np.float32)
