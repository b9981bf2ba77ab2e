"""The operators of a step in 8 bits written out plainly, in numpy and 64 bits: what the tests of conef_q8_*, conef_rms_* and conef_loss_* compare
with.  Shares nothing with the library."""
import numpy as np

from layers_ref import U16, U32, bf16, rounded  # noqa: F401

E4M3, E5M2 = 0, 1
BITS, BIAS, LARGEST = (3, 2), (7, 15), (448.0, 57344.0)


def table(form):
    """what the 256 codes stand for"""
    c = np.arange(256)
    e, m = (c & 127) >> BITS[form], (c & ((1 << BITS[form]) - 1)) / (1 << BITS[form])
    v = np.where(e > 0, (1 + m) * 2.0 ** (e - BIAS[form]), m * 2.0 ** (1 - BIAS[form]))
    return np.where(c > 127, -v, v)


def encode(x, form):
    """(codes, scale bytes) of x's rows, by distances to the two neighbours among the format's values"""
    rows, cols = x.shape
    blocks = -(-cols // 128)
    v = np.zeros((rows, blocks * 128))
    v[:, :cols] = x
    v = v.reshape(rows, blocks, 128)
    bad = ~np.isfinite(v).all(-1)
    a = np.abs(np.where(bad[..., None], 0.0, v))
    most = a.max(-1)
    b = np.full(most.shape, -127)
    for _ in range(400):                                          # the smallest power for which nothing is cut off
        more = most > LARGEST[form] * 2.0 ** b
        if not more.any():
            break
        b = b + more
    a = a / (2.0 ** b.astype(float))[..., None]
    grid = np.unique(table(form)[:128][table(form)[:128] <= LARGEST[form]])
    low = np.clip(np.searchsorted(grid, a, side="right") - 1, 0, len(grid) - 1)
    up = np.minimum(low + 1, len(grid) - 1)
    below, above = a - grid[low], grid[up] - a
    take = (up > low) & ((above < below) | ((above == below) & (low % 2 == 1)))
    code = np.where(take, up, low) + 128 * np.signbit(v)          # (codes are places in the grid)
    return np.where(bad[..., None], 0, code).reshape(rows, -1)[:, :cols].astype(np.uint8), np.where(bad, 255, b + 127).astype(np.uint8)


def decode(codes, scales, form):
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return table(form)[codes] * np.repeat(s, 128, 1)[:, :codes.shape[1]]


def pack(codes, scales):
    """The packed buffers, byte by byte as the format states them (zeros where the operand is filled up)."""
    rows, cols = codes.shape
    R, P = -(-rows // 64) * 64, -(-cols // 128)
    out_c, out_s = np.zeros(R * P * 128, np.uint8), np.zeros(R * P, np.uint8)
    i, j = np.meshgrid(np.arange(rows), np.arange(cols), indexing="ij")
    out_c[((i // 16) * P + j // 128) * 2048 + (j // 16 % 8) * 256 + (i % 16) * 16 + j % 16] = codes
    i, b = np.meshgrid(np.arange(rows), np.arange(P), indexing="ij")
    out_s[b * R + i] = scales
    return out_c, out_s


def rms(z, gamma, eps):
    """(y, rstd) in 64 bits"""
    z = z.astype(np.float64)
    rstd = 1.0 / np.sqrt((z * z).mean(1) + np.float64(np.float32(eps)))
    return z * rstd[:, None] * gamma.astype(np.float64), rstd


def rms_back(dy, z, gamma, rstd):
    """dz without dz_in, dgamma, for the given statistic; hat and a"""
    dy, z, gamma, rstd = (np.asarray(v).astype(np.float64) for v in (dy, z, gamma, rstd))
    hat = z * rstd[:, None]
    a = dy * gamma
    return rstd[:, None] * (a - hat * (a * hat).mean(1, keepdims=True)), (dy * hat).sum(0), hat, a


def loss(x, w, targets, dloss=None):
    """(loss, lse, logits, probabilities, dx, dw) in 64 bits"""
    x, w = x.astype(np.float64), w.astype(np.float64)
    logits = x @ w.T
    most = logits.max(1, keepdims=True)
    lse = most[:, 0] + np.log(np.exp(logits - most).sum(1))
    there = (targets >= 0) & (targets < w.shape[0])
    at = np.where(there, targets, 0)
    rows = np.arange(len(targets))
    p = np.exp(logits - lse[:, None])
    d = p.copy()
    d[rows, at] -= 1.0
    d *= np.where(there, 1.0 if dloss is None else dloss.astype(np.float64), 0.0)[:, None]
    return np.where(there, lse - logits[rows, at], 0.0), lse, logits, p, d @ w, d.T @ x
