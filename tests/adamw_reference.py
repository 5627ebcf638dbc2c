"""The optimizer's operators from their formulas in 64 bits (numpy): what the GPU tests compare with."""
import numpy as np

BLOCK = 256
LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8
U = 2.0 ** -24                                              # half a step of fp32, relative


def moments(g, m, v, scale=1.0, beta1=BETA1, beta2=BETA2):
    """new m and v and how far fp32 may be off: the constants, g' and each product are rounded, then the sum"""
    g = g.astype(np.float64) * scale
    m1, m2, v1, v2 = beta1 * m.astype(np.float64), (1.0 - beta1) * g, beta2 * v.astype(np.float64), (1.0 - beta2) * g * g
    # (scale, g', constant, product, sum; the square has the first two twice and a rounding of its own; 2^-149 where they underflow)
    return m1 + m2, v1 + v2, 6 * U * (np.abs(m1) + np.abs(m2)) + 2.0 ** -148, 9 * U * (v1 + v2) + 2.0 ** -148


def step(w, m, v, dm, dv, t, decay=0.0, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, root=None):
    """new w from the new moments, and how far fp32 may be off given that m is within dm, v within dv"""
    w = w.astype(np.float64)
    root = np.sqrt(v) if root is None else root
    c1, c2 = lr / (1.0 - beta1 ** t), 1.0 / np.sqrt(1.0 - beta2 ** t)
    den = root * c2 + eps
    # the root's error: half of v's relative one, or all of it where v is as small as its own error
    droot = np.where(v > 4 * dv, dv / (2.0 * np.sqrt(np.maximum(v - dv, 1e-300))), np.sqrt(v + dv)) + U * root
    low = np.maximum(den - droot * c2 - 8 * U * den, 1e-300)
    u = c1 * m / den
    du = c1 * (np.abs(m) + dm) / low - c1 * np.abs(m) / den + 12 * U * np.abs(u)
    out = (1.0 - lr * decay) * w - u
    return out, 3 * U * (np.abs(w) + np.abs(out)) + du + 2.0 ** -148


def philox(q, t, j, seed):
    """Philox4x32-10 of the counters (q, t, j), as many rows of four words as q has entries"""
    q = q.astype(np.uint64)
    mask = np.uint64(0xFFFFFFFF)
    c = [q & mask, q >> np.uint64(32), np.full_like(q, t & 0xFFFFFFFF), np.full_like(q, j)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & mask, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & mask]
        k = [(k[0] + np.uint64(0x9E3779B9)) & mask, (k[1] + np.uint64(0xBB67AE85)) & mask]
    return np.stack(c, 1)


def code_values():
    """what the 256 codes of e4m3 stand for"""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    x = np.where(e > 0, (1 + f / 8.0) * 2.0 ** (e - 7.0), f * 2.0 ** -9)
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c >> 7, -x, x)


CODES = code_values()


def held(codes, scales):
    """the numbers that codes and scales (one per block) stand for"""
    return CODES[codes] * scales.astype(np.float64)[np.arange(codes.size) // BLOCK]


def largest(x):
    """the largest finite magnitude of each block, 2^-100 at least"""
    n = -(-x.size // BLOCK)
    y = np.zeros(n * BLOCK)
    y[:x.size] = np.where(np.isfinite(x), np.abs(x), 0.0)
    return np.maximum(y.reshape(n, BLOCK).max(1), 2.0 ** -100)


def coded(x, dx, bits, root=False):
    """(code of x, whether it is certain): x within dx, `bits` the 16 random bits of each element"""
    most = largest(x)
    y = np.abs(x) * (448.0 / most)[np.arange(x.size) // BLOCK]
    fine = np.isfinite(x)
    y = np.where(fine, y, 0.0)
    e = np.maximum(np.frexp(np.maximum(y, 2.0 ** -6))[1] - 1, -6)
    spacing = 2.0 ** (e - 3.0)
    at = y / spacing
    whole = np.floor(at)
    rest = (at - whole) * 2.0 ** 20 + bits * 16.0 + 8.0     # (below 2^-6 the spacing is that of 2^-6: whole counts from 0)
    code = np.where(e > -6, (e + 6) * 8 + whole, whole) + (rest >= 2.0 ** 20)
    # how far `at` may be off, in the same unit: x, the block's largest magnitude, the factor, the product and the 2^-6 added
    off = np.where(fine, np.abs(dx), 0.0) * (448.0 / most)[np.arange(x.size) // BLOCK] / spacing + 10 * U * at + 16 * U
    off = off * 2.0 ** 20 + 1.0
    sure = (np.abs(rest - 2.0 ** 20) > off) & (rest > off) & (rest < 2.0 ** 21 - off) & (at - whole > off * 2.0 ** -20) & (whole + 1 - at > off * 2.0 ** -20)
    # (a value that is a code exactly stays one, however it is approached; that is allowed for by the caller's one-off)
    if root:
        code = np.where((code == 0) & (x > 0), 1, code)
    return np.where(fine, code, 127).astype(np.int64) + np.where(np.signbit(x), 128, 0), sure
