"""Plain 64-bit references (numpy, CPU) of the 4-bit operands, the root-mean-square norm, log probabilities and clipping, written from
their definitions; the CPU suite checks them against hand-made values and finite differences, the GPU tests use them."""
import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---- 4-bit floating point ----
def f4_scale_index(rows, blocks):
    r, b = np.arange(rows)[:, None], np.arange(blocks)[None, :]
    return (b // 4 * (-(-rows // 64) * 64) + r // 64 * 64) * 4 + b % 4 * 64 + r % 16 * 4 + r % 64 // 16


def f4_scale_table(byte):
    """Scale bytes [rows, blocks] in the library's layout."""
    rows, blocks = byte.shape
    t = np.zeros(-(-rows // 64) * 256 * -(-blocks // 4), np.uint8)
    t[f4_scale_index(rows, blocks)] = byte
    return t


def f4_nearest(y):
    """Code of the nearest value, ties to the even code, for |y| <= 6."""
    a = np.abs(y)
    at = np.clip(np.searchsorted(E2M1, a), 1, 7)
    lo, hi = a - E2M1[at - 1], E2M1[at] - a
    code = np.where((lo < hi) | ((lo == hi) & (at % 2 == 1)), at - 1, at)
    return (code + 8 * np.signbit(y)).astype(np.uint8)


def f4_quantize(x, block_rows=1):
    """(codes [rows, columns up to a multiple of 32], scale bytes [rows, blocks]) of x in blocks of 32 columns."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb, R = -(-cols // 32), -(-rows // block_rows) * block_rows
    full = np.zeros((R, nb * 32))
    full[:rows, :cols] = x
    blocks = full.reshape(-1, block_rows, nb, 32)
    good = np.isfinite(blocks).all((1, 3))
    top = np.where(np.isfinite(blocks), np.abs(blocks), 0.0).max((1, 3))
    e = np.full(top.shape, -127)
    for k in range(-127, 128):                                # the smallest that holds the largest, by trying all
        e = np.where((e == k) & (top > 6 * 2.0 ** k), k + 1, e)
    byte = np.where(good, e + 127, 255).repeat(block_rows, 0)[:rows].astype(np.uint8)
    scaled = full[:rows] * 2.0 ** -np.repeat(e.repeat(block_rows, 0)[:rows], 32, 1).astype(np.float64)
    bad = np.repeat(byte == 255, 32, 1)
    return np.where(bad, 0, f4_nearest(np.where(bad, 0.0, scaled))).astype(np.uint8), byte


def f4_pack(codes):
    return (codes[:, ::2] | codes[:, 1::2] << 4).astype(np.uint8)


def f4_values(codes, byte):
    v = np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7]
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return v * np.repeat(scale, 32, 1)[:, :codes.shape[1]]


# ---- root-mean-square norm ----
def rms_fwd(x, y, g, eps):
    """-> x', r, h"""
    x = x if y is None else x + y
    r = 1 / np.sqrt((x * x).mean(1) + eps)
    return x, r, x * r[:, None] * g


def rms_bwd(x, g, eps, dh, dres=None):
    """x: x' of the forward pass.  -> dx, dg"""
    r = 1 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    xh = x * r
    dx = r * (dh * g - xh * (dh * g * xh).mean(1, keepdims=True))
    return dx if dres is None else dx + dres, (dh * xh).sum(0)


# ---- log probabilities ----
def log_softmax(z, scale):
    """Rows without a distribution: -infinity throughout (nothing but -infinity), or NaN (a NaN or +infinity)."""
    z = np.asarray(z, np.float64)
    m = z.max(1, keepdims=True)
    bad = np.isnan(z).any(1, keepdims=True) | (m == np.inf)
    none = (m == -np.inf) & ~bad
    with np.errstate(invalid="ignore"):
        d = scale * (z - np.where(np.isfinite(m), m, 0.0))
        lp = d - np.log(np.where(none | bad, 1.0, np.exp(np.where(bad, 0.0, d)).sum(1, keepdims=True)))
    return np.where(bad, np.nan, np.where(none, -np.inf, lp))


def logprob_fwd(z, targets, scale=1.0, k=0):
    """-> logp, entropy, ids [rows, k], their log probabilities"""
    lp = log_softmax(z, scale)
    rows, vocab = lp.shape
    with np.errstate(invalid="ignore"):
        p = np.exp(lp)
        entropy = -np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lp)).sum(1)
    given = (targets >= 0) & (targets < vocab)
    logp = np.where(given, lp[np.arange(rows), np.where(given, targets, 0)], 0.0)
    ids, best = np.full((rows, k), -1), np.full((rows, k), -np.inf)
    for r in range(rows):
        if np.isnan(lp[r]).any():
            best[r] = np.nan
            continue
        order = np.argsort(-np.asarray(z[r], np.float64), kind="stable")[:k]
        order = order[np.asarray(z[r])[order] > -np.inf]
        ids[r, :order.size], best[r, :order.size] = order, lp[r, order]
    return logp, entropy + 0.0, ids, best


def logprob_bwd(z, targets, dlogp, dentropy, scale=1.0):
    lp = log_softmax(z, scale)
    rows, vocab = lp.shape
    with np.errstate(invalid="ignore"):
        p = np.exp(lp)
        plp = np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lp))
    h = -plp.sum(1, keepdims=True)
    given = (targets >= 0) & (targets < vocab)
    dl = np.where(given, dlogp, 0.0)[:, None]
    hot = np.zeros((rows, vocab))
    none = (np.asarray(z) == -np.inf).all(1)
    hot[np.arange(rows)[given & ~none], targets[given & ~none]] = 1.0
    return scale * (dl * (hot - p) - np.asarray(dentropy)[:, None] * (plp + p * h))


# ---- clipping ----
def clip(grads, max_norm):
    total = math.sqrt(math.fsum(float(v) ** 2 for g in grads for v in np.asarray(g, np.float64).ravel()))
    factor = max_norm / total if total > max_norm else 1.0
    return total, factor, [np.asarray(g, np.float64) * factor for g in grads]
