"""Plain 64-bit forms of the operators for layers of experts, in numpy, from their definitions, and what their results may be off."""
import numpy as np
import torch

import matrix_reference as R

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a step of rounding, relative; f16's subnormals have an absolute one
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
ONE = 2.0 ** -24                                               # a rounding in fp32


def host(x):
    return x.detach().double().cpu().numpy()


def rounded(want, dtype):
    """What one rounding to dtype of a result that fp32 rounded before adds to its error."""
    return HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -10) + LEAST[dtype]


def route(l, k, all_):
    """l [T, E] in 64 bits, no NaN: experts, gates, offsets, order (up to offsets[-1]), slots."""
    T, E = l.shape
    experts = np.argsort(-l, axis=1, kind="stable")[:, :k]
    chosen = np.take_along_axis(l, experts, 1)
    closed = chosen == -np.inf
    top = l.max(1, keepdims=True)
    base = np.where(top == -np.inf, 0.0, top)
    part = np.exp(chosen - base)
    total = np.exp(l - base).sum(1, keepdims=True) if all_ else part.sum(1, keepdims=True)
    gates = np.where(closed, 0.0, part / np.where(total == 0, 1.0, total))
    experts = np.where(closed, -1, experts)
    flat = experts.reshape(-1)
    order = np.argsort(np.where(flat < 0, E, flat), kind="stable")
    order = order[:(flat >= 0).sum()]
    offsets = np.concatenate(([0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))))
    slots = np.full(T * k, -1)
    slots[order] = np.arange(len(order))
    return experts, gates, offsets, order, slots


def softmax_error(l):
    """How far a softmax of each row of l may be off in fp32, relative: each exponential by the rounding of its argument (|l - max| * 2^-24) and two
    steps of its own; their sum by that, weighted, and E roundings; the division by one."""
    top = l.max(1, keepdims=True)
    d = np.where(np.isfinite(l), np.where(np.isfinite(top), top, 0.0) - l, 0.0)
    d = np.minimum(d, 110.0)                                    # beyond that the exponential is 0
    p = np.exp(-d) * np.isfinite(l)
    mean = (p * (d + 4)).sum(1, keepdims=True) / np.maximum(p.sum(1, keepdims=True), 1e-300)
    return (d + 4 + mean + l.shape[1] + 1) * ONE


def route_backward(l, experts, gates, dgates, all_):
    """Gradient of the logits in 64 bits, and the sum of the magnitudes that went into each."""
    T, E = l.shape
    there = (experts >= 0) & (experts < E)
    g, d = np.where(there, gates, 0.0), np.where(there, dgates, 0.0)
    s, size = (g * d).sum(1, keepdims=True), np.abs(g * d).sum(1, keepdims=True)
    out, mag = np.zeros((T, E)), np.zeros((T, E))
    if all_:
        top = l.max(1, keepdims=True)
        p = np.exp(l - np.where(top == -np.inf, 0.0, top))
        p = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
        out, mag = -p * s, p * size
    for j in range(experts.shape[1]):
        at = np.arange(T)[there[:, j]], experts[there[:, j], j]
        np.add.at(out, at, (g[:, j:j + 1] * (d[:, j:j + 1] - (0 if all_ else s)))[there[:, j], 0])
        np.add.at(mag, at, (np.abs(g[:, j:j + 1]) * (np.abs(d[:, j:j + 1]) + (0 if all_ else size)))[there[:, j], 0])
    return out, mag


def combine(rows, slots, gates, T, k):
    """[T, N] in 64 bits, and the sum of the magnitudes."""
    out, mag = np.zeros((T, rows.shape[1])), np.zeros((T, rows.shape[1]))
    for j in range(k):
        s = slots.reshape(T, k)[:, j]
        there = (s >= 0) & (s < len(rows))
        g = np.ones(T) if gates is None else gates.reshape(T, k)[:, j]
        out[there] += g[there, None] * rows[s[there]]
        mag[there] += np.abs(g[there, None] * rows[s[there]])
    return out, mag


def group_sizes(rng, E, R, kind):
    """Offsets of E groups in R rows: "even", "ragged" (some empty, rows left behind the last), "one" (all rows in one group), "none"."""
    if kind == "none":
        return np.zeros(E + 1, np.int64)
    if kind == "one":
        o = np.zeros(E + 1, np.int64)
        o[E // 2 + 1:] = R
        return o
    if kind == "even":
        return np.arange(E + 1) * R // E
    cuts = np.sort(rng.integers(0, R - R // 8 + 1, E - 1)) if E > 1 else np.zeros(0, np.int64)
    if E > 3:
        cuts[1] = cuts[0]
    return np.concatenate(([0], cuts, [R - R // 8])).astype(np.int64)


def group_columns(R_, E):
    return (R_ + 127 * min(E, R_)) // 128 * 128


def padded(x, offsets, columns):
    """Rows x [R, cols] -> [cols, columns], each group from a multiple of 128 on, and where each group begins."""
    out, begin, at = np.zeros((x.shape[1], columns)), [], 0
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        begin.append(at)
        out[:, at:at + hi - lo] = x[lo:hi].T
        at += R.up(hi - lo, 128)
    return out, begin, at


def q(x, stochastic=False, seed=0, rnd=0, worker=0):
    """The values of the 4-bit form of x along its rows."""
    return R.values(*R.quantize(x, stochastic, seed, rnd, worker), x.shape[1])


def packed_bytes(code, scale, rows, cols):
    """The packed form as the library lays it out."""
    wide = R.up(cols, 128)
    at = R.up(rows * wide // 2, 256)
    out = np.zeros(at + R.up(rows * wide // 32, 256), np.uint8)
    out[:rows * wide // 2] = R.pack(code).reshape(-1)
    out[at:at + rows * wide // 32] = scale.reshape(-1)
    return out


def packed_weights(w):
    """[E, N, K] -> ([E, bytes] uint8, values [E, N, K])"""
    forms = [R.quantize(x) for x in w]
    return (torch.from_numpy(np.stack([packed_bytes(c, s, *w.shape[1:]) for c, s in forms])),
            np.stack([R.values(c, s, w.shape[2]) for c, s in forms]))
