"""AdamW with states in 32 or 8 bits in numpy: binary32 with one rounding per operation, and in binary64."""
import numpy as np

BLOCK = 256
# the 127 magnitudes of e4m3, written out from the format: subnormals are multiples of 2^-9, normals (1 + m/8) 2^(e-7)
GRID = np.array([m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1])
F = np.float32


def noise(seed, blocks_before, n):
    """32 random bits for each of n elements of a tensor that `blocks_before` blocks of the list come before."""
    p = np.arange(n, dtype=np.uint64) + np.uint64(blocks_before * BLOCK)
    mask = np.uint64(0xFFFFFFFF)
    h = (p & mask) ^ (((p >> np.uint64(32)) * np.uint64(0x9E3779B9)) & mask) ^ np.uint64(seed & 0xFFFFFFFF)
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x7FEB352D)) & mask
    h = ((h ^ (h >> np.uint64(15))) + np.uint64(seed >> 32)) & mask
    h = (h * np.uint64(0x846CA68B)) & mask
    return h ^ (h >> np.uint64(16))


def decode(codes, scale):
    """Values of codes in blocks of 256, binary32."""
    mag = np.where((codes & 0x7F) == 0x7F, np.nan, GRID[np.minimum(codes & 0x7F, 0x7E)])
    v = np.where(codes & 0x80, -mag, mag).astype(F)
    return v * np.repeat(scale, BLOCK)[: len(codes)]


def encode(x, bits, keep_positive):
    """Codes and scales; `bits`: None (nearest, ties to even) or 16 random bits of every element."""
    n = len(x)
    blocks = -(-n // BLOCK)
    a = np.abs(x)
    padded = np.zeros(blocks * BLOCK, F)
    padded[:n] = np.where(np.isfinite(x), a, 0)
    top = padded.reshape(-1, BLOCK).max(1)
    kept = top >= F(2.0 ** -100)
    inv = np.where(kept, F(448) * (F(1) / np.where(kept, top, F(1))), F(0)).astype(F)
    scale = np.where(kept, top * (F(1) / F(448)), F(0)).astype(F)
    y = (a * np.repeat(inv, BLOCK)[:n]).astype(np.float64)
    y = np.where(np.isinf(a), np.where(np.repeat(kept, BLOCK)[:n], 448.0, 0.0), y)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.nan_to_num(y), 2.0 ** -6))) - 3)
    units = np.rint(y / step) if bits is None else np.floor(y / step + bits.astype(np.float64) / 65536)
    q = np.minimum(units * step, 448.0)
    code = np.searchsorted(GRID, np.nan_to_num(q)).astype(np.int64)
    if keep_positive:
        code = np.where((x > 0) & np.repeat(kept, BLOCK)[:n], np.maximum(code, 1), code)
    code = np.where(np.isnan(x), 0x7F, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8), scale


def step32(w, g, m, v, lr, step, betas, eps, wd, theta=None, lam=None, mu=0.0, grad_scale=None):
    """(w, m, v, sqrt v) in binary32, every operation rounded once."""
    b1, b2 = betas
    g = g.astype(F) * F(1 if grad_scale is None else grad_scale)
    if theta is not None:
        g = (g + F(mu) * (w - theta)) - lam
    m = F(b1) * m + F(1 - b1) * g
    v = F(b2) * v + F(1 - b2) * (g * g)
    r = np.sqrt(v)
    u = m / (r * F(1 / np.sqrt(1 - b2 ** step)) + F(eps))
    return F(1 - lr * wd) * w - F(lr / (1 - b1 ** step)) * u, m, v, r


def step64(w, g, m, v, lr, step, betas, eps, wd, theta=None, lam=None, mu=0.0, grad_scale=None):
    """(w, m, v) from the textbook formula in binary64."""
    w, g, m, v = (np.asarray(t, np.float64) for t in (w, g, m, v))
    g = g * (1.0 if grad_scale is None else grad_scale)
    if theta is not None:
        g = g + mu * (w - theta.astype(np.float64)) - lam.astype(np.float64)
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g ** 2
    return w * (1 - lr * wd) - lr * (m / (1 - betas[0] ** step)) / (np.sqrt(v / (1 - betas[1] ** step)) + eps), m, v
