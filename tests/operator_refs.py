"""Plain 64-bit references (numpy, CPU) of the 8-bit operands, the dropout mask and the gated recurrence, written from their
definitions; the CPU suite checks them against published values and finite differences, the GPU tests use them."""
import math

import numpy as np


# ---- 8-bit floating point ----
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
HALF_STEP = {"e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def decode_table(fmt):
    mant, bias = (3, 7) if fmt == "e4m3" else (2, 15)
    out = np.empty(256)
    for i in range(256):
        e, f = (i & 127) >> mant, i & ((1 << mant) - 1)
        v = math.ldexp(f, 1 - bias - mant) if e == 0 else math.ldexp((1 << mant) + f, e - bias - mant)
        if fmt == "e4m3" and i & 127 == 127:
            v = math.nan
        if fmt == "e5m2" and e == 31:
            v = math.nan if f else math.inf
        out[i] = -v if i & 128 else v
    return out


def scale_index(rows, blocks):
    r, b = np.arange(rows)[:, None], np.arange(blocks)[None, :]
    return b * (-(-rows // 64) * 64) + r // 64 * 64 + r % 16 * 4 + r % 64 // 16


def scale_table(e):
    """Exponents [rows, blocks] -> bytes in the library's layout."""
    t = np.zeros(-(-e.shape[0] // 64) * 64 * e.shape[1], np.uint8)
    t[scale_index(*e.shape)] = e + 127
    return t


def nearest_code(y, fmt):
    """Byte of the nearest value, ties to the even code, for |y| within the format's range (or not finite)."""
    v = decode_table(fmt)[:128]
    n = int(np.isfinite(v).sum())
    grid = v[:n]
    a = np.abs(y)
    at = np.clip(np.searchsorted(grid, a), 1, n - 1)
    lo, hi = a - grid[at - 1], grid[at] - a
    code = np.where((lo < hi) | ((lo == hi) & (at % 2 == 1)), at - 1, at)
    if fmt == "e5m2":
        code = np.where(np.isinf(y), 124, code)
        code = np.where(np.isnan(y), 126, code)
    else:
        code = np.where(np.isfinite(y), code, 127)
    return (code + 128 * np.signbit(y)).astype(np.uint8)


def quantize(x, fmt, block_rows=1):
    """(bytes [rows, columns up to a multiple of 16], exponents [rows, blocks]) of x in blocks of 128 columns."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb, R = -(-cols // 128), -(-rows // block_rows) * block_rows
    full = np.zeros((R, nb * 128))
    full[:rows, :cols] = x
    mag = np.where(np.isfinite(full), np.abs(full), 0.0).reshape(-1, block_rows, nb, 128)
    top = mag.max((1, 3))
    e = np.maximum(np.frexp(np.where(top == 0, 0.0, top / TOP[fmt]))[1].astype(np.int64) - 1, -127)     # at most one too small or large
    e = np.where(top > TOP[fmt] * 2.0 ** e, e + 1, e)
    e = np.where((e > -127) & (top <= TOP[fmt] * 2.0 ** (e - 1.0)), e - 1, e)
    e = np.where(top == 0, -127, e).repeat(block_rows, 0)[:rows]
    scaled = full[:rows] * 2.0 ** -np.repeat(e, 128, 1).astype(np.float64)
    return nearest_code(scaled[:, :-(-cols // 16) * 16], fmt), e


def values(q, e, fmt):
    return decode_table(fmt)[q] * (2.0 ** np.repeat(e, 128, 1))[:, :q.shape[1]]


def gelu(u):
    return 0.5 * u * (1 + np.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))


def gelu_grad(u):
    c = math.sqrt(2 / math.pi)
    t = np.tanh(c * (u + 0.044715 * u ** 3))
    return 0.5 * (1 + t) + 0.5 * u * (1 - t * t) * c * (1 + 3 * 0.044715 * u * u)


# ---- dropout ----
def philox(counter, key):
    """Philox4x32-10 of four arrays of 32-bit words under a key of two."""
    c = [np.asarray(v, np.uint32) for v in counter]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        p0, p1 = c[0].astype(np.uint64) * np.uint64(0xD2511F53), c[2].astype(np.uint64) * np.uint64(0xCD9E8D57)
        h0, l0, h1, l1 = (p0 >> np.uint64(32)), p0 & np.uint64(0xFFFFFFFF), (p1 >> np.uint64(32)), p1 & np.uint64(0xFFFFFFFF)
        c = [h1.astype(np.uint32) ^ c[1] ^ np.uint32(k[0]), l1.astype(np.uint32), h0.astype(np.uint32) ^ c[3] ^ np.uint32(k[1]),
             l0.astype(np.uint32)]
        k = [(k[0] + 0x9E3779B9) % (1 << 32), (k[1] + 0xBB67AE85) % (1 << 32)]
    return c


def dropout_threshold(p):
    return int(np.rint(np.float32(p) * np.float32(65536.0)))


def dropout_keep(rows, cols, p, seed, site, step):
    g = -(-cols // 8)
    shape = (rows, g)
    w = philox([np.broadcast_to(np.arange(g), shape), np.broadcast_to(np.arange(rows)[:, None], shape), np.full(shape, site),
                np.full(shape, step % (1 << 32))], (seed % (1 << 32), seed >> 32))
    halves = np.stack([h for v in w for h in (v & np.uint32(0xFFFF), v >> np.uint32(16))], -1).reshape(rows, -1)[:, :cols]
    t = dropout_threshold(p)
    return halves >= t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


# ---- gated recurrence ----
def _sigmoid(f):
    return np.where(f >= 0, 1 / (1 + np.exp(-np.abs(f))), np.exp(-np.abs(f)) / (1 + np.exp(-np.abs(f))))


def scan_fwd(f, x, h0, lens=None):
    """f, x [B, T, D]; -> y [B, T, D], h_end [B, D]."""
    B, T, D = f.shape
    lens = np.full(B, T) if lens is None else np.clip(lens, 0, T)
    y, h = np.zeros((B, T, D)), np.array(h0, np.float64)
    for t in range(T):
        on = t < lens
        h[on] = _sigmoid(f[on, t]) * h[on] + _sigmoid(-f[on, t]) * x[on, t]
        y[on, t] = h[on]
    return y, h


def scan_bwd(f, x, h0, dy, dh_end, lens=None):
    """-> df, dx [B, T, D], dh0 [B, D]."""
    B, T, D = f.shape
    lens = np.full(B, T) if lens is None else np.clip(lens, 0, T)
    y, _ = scan_fwd(f, x, h0, lens)
    df, dx, r = np.zeros((B, T, D)), np.zeros((B, T, D)), np.array(dh_end, np.float64)
    for t in reversed(range(T)):
        on = t < lens
        a, z = _sigmoid(f[on, t]), _sigmoid(-f[on, t])
        before = y[on, t - 1] if t else np.asarray(h0)[on]
        g = dy[on, t] + r[on]
        dx[on, t] = g * z
        df[on, t] = g * (before - x[on, t]) * a * z
        r[on] = a * g
    return df, dx, r


def scan_bounds(f, x, h0, dy, dh_end, lens=None):
    """How far fp32 results may be off, element by element: allowances for y, h_end, df, dx, dh0 before y, df and dx are rounded.

    With u = 2^-24.  The argument of exp2 is a rounded product with a rounded constant, so e^-f is off by 2 |f| u, and by 2 u of the
    instruction (one unit in the last place); 1 + e^-f rounds, its reciprocal is good to 2 u: a is off by (1 - a) (2 |f| + 2) u + 3 u
    and 1 - a, a product or a difference from the larger one, by (2 |f| + 2) u + 4 u.  A term of a state passes a product and an addition
    in the thread's own chain, and two more wherever stretches of 16 steps and more meet: 4 u of the sum of magnitudes a step, and 16 u
    once.  Errors fade as the state does, by a_t a step.  A gate under 2^-126 may come out as any number under it (exp2 gives 0 there), so
    what it multiplies is off by 2^-126 of itself: 2^-120 in all, of 1 and of each magnitude, in every output."""
    B, T, D = f.shape
    u, tiny = 2.0 ** -24, 2.0 ** -120
    lens = np.full(B, T) if lens is None else np.clip(lens, 0, T)
    h0 = np.broadcast_to(np.asarray(h0, np.float64), (B, D))
    a, z = _sigmoid(f), _sigmoid(-f)
    da, dz = (z * (2 * np.abs(f) + 2) + 3) * u, (2 * np.abs(f) + 6) * u
    with np.errstate(invalid="ignore", over="ignore"):
        y, _ = scan_fwd(f, x, h0, lens)
        m, e = np.abs(h0), np.zeros((B, D))
        ey, eb = np.zeros((B, T, D)), np.zeros((B, T, D))        # of y; of the state in front of each step
        for t in range(T):
            on = t < lens
            eb[:, t] = e + 16 * u * m + tiny * (1 + m)
            v = z[on, t] * np.abs(x[on, t])
            m2 = a[on, t] * m[on] + v
            e[on] = a[on, t] * (e[on] + da[on, t] * m[on]) + dz[on, t] * v + 4 * u * m2
            m[on] = m2
            ey[on, t] = (e + 16 * u * m + tiny * (1 + m))[on]
        eh = e + 16 * u * m + tiny * (1 + m)
        n, e = np.abs(np.asarray(dh_end, np.float64)) * np.ones((B, D)), np.zeros((B, D))
        edf, edx = np.zeros((B, T, D)), np.zeros((B, T, D))
        for t in reversed(range(T)):
            on = t < lens
            before = y[on, t - 1] if t else h0[on]
            gap = np.abs(before - x[on, t])
            g = np.abs(dy[on, t]) + n[on]                        # bounds |g_t|
            eg = e[on] + 16 * u * g + tiny * (1 + g)
            edx[on, t] = z[on, t] * (eg + (dz[on, t] + 2 * u) * g) + tiny * (1 + g)
            edf[on, t] = a[on, t] * z[on, t] * (eg * gap + g * (eb[on, t] + u * gap) + g * gap * (da[on, t] + dz[on, t] + 4 * u)
                                                + eg * eb[on, t]) + tiny * (1 + g) * (1 + gap)
            n[on] = a[on, t] * g
            e[on] = a[on, t] * (e[on] + da[on, t] * g) + 4 * u * a[on, t] * g
        return ey, eh, edf, edx, e + 16 * u * n + tiny * (1 + n)


def exceeds(got, ref, allow, half_step=0.0):
    """Where `got` is off by more than `allow` and a rounding of half_step on top: NaN and infinities have to be the same ones.  Steps
    stop shrinking at 2^-126 (bf16: 2^-133 apart below it, half of which is 2^-8 * 2^-126; fp32: 2^-149, half is 2^-24 * 2^-126)."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    fin = np.isfinite(ref)
    with np.errstate(invalid="ignore", over="ignore"):
        bad = ~(np.abs(got - ref) <= allow + half_step * np.maximum(np.abs(ref) + allow, 2.0 ** -126))
    return np.where(fin, bad, ~((got == ref) | (np.isnan(got) & np.isnan(ref))))
