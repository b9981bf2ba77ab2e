"""The operators of a training step written out plainly, in numpy and 64 bits: what the tests of conef_dropout_*, conef_norm_* and
conef_mx_* compare with.  Shares nothing with the library."""
import numpy as np

DROP, MX_ROWS, MX_COLS = 0xC0000000, 0xC8000000, 0xD0000000
U32, U16 = 2.0 ** -24, 2.0 ** -8          # largest relative error of a rounding to fp32 (24 significant bits) and to bf16 (8)
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def philox(counter, key):
    """Philox4x32-10 of one counter (four words) under a key (two words), in Python integers."""
    c, k, mask = list(counter), list(key), 0xFFFFFFFF
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & mask, (a >> 32) ^ c[3] ^ k[1], a & mask]
        k = [(k[0] + 0x9E3779B9) & mask, (k[1] + 0xBB67AE85) & mask]
    return c


def draws(rows, cols, word, seed, step):
    """16-bit draw of every element."""
    per = -(-cols // 8)
    c0 = np.arange(rows * per, dtype=np.uint64)
    c = [c0, np.full_like(c0, word), np.full_like(c0, step & 0xFFFFFFFF), np.full_like(c0, step >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    mask, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s) ^ c[1] ^ np.uint64(k[0]), b & mask, (a >> s) ^ c[3] ^ np.uint64(k[1]), a & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    w = np.stack(c, -1)
    halves = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(rows, per * 8)
    return halves[:, :cols].astype(np.int64)


def keep_and_scale(shape, p, seed, site, step):
    t = min(65535, int(np.floor(float(np.float32(p)) * 65536 + 0.5)))
    return draws(*shape, DROP + site, seed, step) >= t, np.float32(65536.0 / (65536 - t))


def bf16(x):
    """fp32 or fp64 values rounded to bf16 (through fp32), as fp32"""
    x = np.asarray(x, np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), r, x)


def rounded(x, is_bf16):
    return bf16(x) if is_bf16 else np.asarray(x, np.float32)


def dropped_sum(x, residual, p, seed, site, step, is_bf16):
    """residual + s keep(x): bits, since every operation is one fp32 rounding"""
    keep, s = keep_and_scale(x.shape, p, seed, site, step)
    v = np.where(keep, np.float32(x) * s, np.float32(0))
    return rounded(v if residual is None else np.float32(residual) + v, is_bf16)


def norm(z, gamma, beta, eps):
    z = z.astype(np.float64)
    mean = z.mean(1)
    rstd = 1.0 / np.sqrt(((z - mean[:, None]) ** 2).mean(1) + eps)
    hat = (z - mean[:, None]) * rstd[:, None]
    return hat * gamma + beta, mean, rstd, hat


def norm_back(dy, z, gamma, mean, rstd):
    """dz without dz_in, dgamma, dbeta, for the given statistics"""
    dy, z, gamma, mean, rstd = (np.asarray(v).astype(np.float64) for v in (dy, z, gamma, mean, rstd))
    hat = (z - mean[:, None]) * rstd[:, None]
    a = dy * gamma
    dz = rstd[:, None] * (a - a.mean(1, keepdims=True) - hat * (a * hat).mean(1, keepdims=True))
    return dz, (dy * hat).sum(0), dy.sum(0), hat, a


def mx_encode(x, u=None):
    """(codes, scale bytes) of x's rows; u: draws, or None for nearest even.  Element by element distances in 64 bits."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :cols] = x
    v = v.reshape(rows, blocks, 32)
    bad = ~np.isfinite(v).all(-1)
    a = np.abs(np.where(bad[..., None], 0.0, v))
    most = a.max(-1)
    e = np.where(most > 0, np.frexp(np.where(most > 0, most, 1.0))[1] - 1, -200)
    b = e - 2
    if u is not None:
        b = np.where(most > 6 * 2.0 ** b, b + 1, b)
    b = np.maximum(b, -127)
    a = a / (2.0 ** b)[..., None]
    low = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 7)
    up = np.minimum(low + 1, 7)
    gap = np.where(up > low, GRID[up] - GRID[low], 1.0)
    f = np.where(up > low, (a - GRID[low]) / gap, 0.0)
    if u is None:
        take = (f > 0.5) | ((f == 0.5) & (low % 2 == 1))
    else:
        full = np.zeros((rows, blocks * 32), np.int64)
        full[:, :cols] = u
        take = np.floor(f * 65536) + full.reshape(rows, blocks, 32) >= 65536
    code = np.where(take, up, low) + 8 * np.signbit(v)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(rows, -1)[:, :cols].astype(np.uint8), np.where(bad, 255, b + 127).astype(np.uint8)


def mx_decode(codes, scales):
    v = GRID[codes & 7] * np.where(codes >= 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, 1)[:, :codes.shape[1]]


def mx_pack(codes, scales):
    """The packed buffers, byte by byte as the format states them (zeros where the operand is filled up)."""
    rows, cols = codes.shape
    r, P = -(-rows // 64) * 64, -(-cols // 128)
    out_c, out_s = np.zeros(r * P * 64, np.uint8), np.zeros(r * P * 4, np.uint8)
    i, j = np.meshgrid(np.arange(rows), np.arange(cols), indexing="ij")
    at = ((i // 16) * P + j // 128) * 1024 + (j // 32 % 4) * 256 + (i % 16) * 16 + (j % 32) // 2
    np.bitwise_or.at(out_c, at, (codes << (4 * (j % 2))).astype(np.uint8))
    i, b = np.meshgrid(np.arange(rows), np.arange(scales.shape[1]), indexing="ij")
    out_s[((i // 64) * P + b // 4) * 256 + (b % 4) * 64 + (i % 16) * 4 + i % 64 // 16] = scales
    return out_c, out_s
