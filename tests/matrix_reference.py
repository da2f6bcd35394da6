"""Plain 64-bit forms of the operators for matrix parameters, in numpy, from their definitions."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
USUAL = ((3.4445, -4.7750, 2.0315),) * 5


def up(v, a):
    return (v + a - 1) // a * a


def philox(c0, c1, c2, c3, seed):
    """Philox4x32-10; arrays of 32-bit values in uint64."""
    low, k0, k1 = np.uint64(0xFFFFFFFF), seed & 0xFFFFFFFF, seed >> 32
    s = np.uint64(32)
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> s) ^ c1 ^ np.uint64(k0), b & low, (a >> s) ^ c3 ^ np.uint64(k1), a & low
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def variates(count, seed, rnd, worker):
    g = np.arange(count // 8, dtype=np.uint64)
    zero = np.zeros_like(g)
    w = np.stack(philox(g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), zero + np.uint64(worker), zero + np.uint64(rnd), seed), 1)
    return np.stack((w & np.uint64(0xFFFF), w >> np.uint64(16)), 2).reshape(-1).astype(np.int64)


def quantize(x, stochastic=False, seed=0, rnd=0, worker=0):
    """x [rows, cols] in 64 bits -> codes [rows, wide] (0..15), scale bytes [rows, wide/32]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    wide = up(cols, 128)
    v = np.zeros((rows, wide))
    v[:, :cols] = x
    blocks = v.reshape(rows, -1, 32)
    fine = np.isfinite(blocks).all(2)
    blocks = np.where(fine[:, :, None], blocks, 0.0)
    top = np.abs(blocks).max(2)
    e = np.frexp(top)[1] - 1 - 2
    if stochastic:
        e = e + (top > 6.0 * np.ldexp(1.0, e))
    e = np.where(top == 0, -127, np.clip(e, -127, 125))
    a = np.ldexp(np.abs(blocks), -e[:, :, None])
    at = np.searchsorted(MAGNITUDES, a, side="right") - 1
    ends = np.append(MAGNITUDES, 8.0)
    f = (a - ends[at]) / (ends[at + 1] - ends[at]) if (at < 8).all() else None
    if stochastic:
        r = variates(rows * wide, seed, rnd, worker).reshape(a.shape)
        at = at + (r + np.floor(f * 65536) >= 65536)
    else:
        at = at + ((f > 0.5) | ((f == 0.5) & (at % 2 == 1)))
    code = np.minimum(at, 7) + 8 * np.signbit(blocks)
    code = np.where(fine[:, :, None], code, 0).reshape(rows, wide)
    return code.astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def pack(code):
    return code[:, 0::2] | (code[:, 1::2] << 4)


def values(code, scale, cols):
    """What a packed matrix stands for, [rows, cols] in 64 bits."""
    q = MAGNITUDES[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return (q.reshape(scale.shape + (32,)) * s[:, :, None]).reshape(code.shape)[:, :cols]


def newton_schulz(x, coeffs=USUAL, eps=1e-7, noise=0.0, rng=None):
    """x [rows, cols] in 64 bits.  noise: every product's result is moved by a random matrix of that size relative to the norms of
    what went into it, entry by entry."""
    x = np.asarray(x, np.float64)
    X = x / (np.linalg.norm(x) + eps) if np.linalg.norm(x) + eps > 0 else x * 0.0
    turned = X.shape[0] > X.shape[1]
    X = X.T if turned else X

    def times(a, b):
        c = a @ b
        if noise:
            c = c + noise * rng.standard_normal(c.shape) * np.outer(np.linalg.norm(a, axis=1), np.linalg.norm(b, axis=0))
        return c

    for a, b, c in coeffs:
        G = times(X, X.T)
        P = a * np.eye(len(G)) + b * G + c * times(G, G)
        X = times(P, X)
    return X.T if turned else X
