"""The operators' definitions (include/hpsgd_ops.h) in binary64 numpy, element by element where that is clearest.
Nothing here is shared with the library."""
import numpy as np

U64 = (1 << 64) - 1
N1, N2, N3 = 0x6A09E667, 0xBB67AE85, 0x3C6EF373


# ---- E4M3 and the 8-bit block format ---------------------------------------------------------
def e4m3_table():
    """Value of each of the 256 codes."""
    out = np.empty(256)
    for c in range(256):
        s, e, f = c >> 7, c >> 3 & 15, c & 7
        x = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out[c] = np.nan if c & 127 == 127 else (-x if s else x)
    return out


E4M3 = e4m3_table()
GRID = E4M3[:127]                    # the non-negative values, ascending


def scale_bytes(top):
    """Exponent byte e + 127 for largest finite magnitudes `top`."""
    top = np.asarray(top, dtype=np.float64)
    out = np.zeros(top.shape, dtype=np.int64)
    for idx, t in np.ndenumerate(top):
        if t > 0:
            m, k = np.frexp(t)       # t = m 2^k, m in [0.5, 1); 448 = 0.875 * 2^9
            out[idx] = max(-127, k - 9 + (m > 0.875)) + 127
    return out


def factor(byte):
    return np.ldexp(1.0, np.asarray(byte, dtype=np.int64) - 127)


def nearest_code(x):
    """Codes of values in [-448, 448], to nearest even."""
    a = np.abs(x)
    i = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 126)
    j = np.minimum(i + 1, 126)
    lo, hi = GRID[i], GRID[j]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 1))
    c = np.where(up, j, i)
    return np.where(np.signbit(x), c | 128, c).astype(np.uint8)


def blocks(x):
    """[rows, cols] -> [rows, nb, 128] with zeros behind."""
    rows, cols = x.shape
    nb = -(-cols // 128)
    out = np.zeros((rows, nb * 128))
    out[:, :cols] = x
    return out.reshape(rows, nb, 128)


def quantize(x):
    """[rows, cols] -> (codes [rows, cols], scale bytes [rows, nb])."""
    rows, cols = x.shape
    b = blocks(np.asarray(x, dtype=np.float64))
    ok = np.isfinite(b)
    e = scale_bytes(np.where(ok, np.abs(b), 0.0).max(axis=2))
    q = np.full(b.shape, 0x7F, dtype=np.uint8)
    with np.errstate(invalid="ignore"):
        v = np.where(ok, b, 0.0) / factor(e)[:, :, None]
    q[ok] = nearest_code(v)[ok]
    return q.reshape(rows, -1)[:, :cols], e


def values(q, e):
    """Codes [rows, cols], scale bytes [rows, nb] -> values."""
    return E4M3[q] * np.repeat(factor(e), 128, axis=1)[:, : q.shape[1]]


# ---- random bits -----------------------------------------------------------------------------
def mix(x):
    x ^= x >> 32
    x = x * 0x6A09E667F3BCC909 & U64
    x ^= x >> 29
    x = x * 0xBB67AE8584CAA73B & U64
    return x ^ x >> 32


def random_bits(seed, step, pos):
    key = mix((mix(seed + 0x3C6EF372FE94F82B & U64) ^ step) + 0xA54FF53A5F1D36F1 & U64)
    k0, k1 = key & 0xFFFFFFFF, key >> 32
    out = np.empty(len(pos), dtype=np.int64)
    for i, p in enumerate(pos):
        p = int(p)
        x = ((p & 0xFFFFFFFF) ^ k0) * N1 & 0xFFFFFFFF
        x ^= x >> 15
        x = (x + k1 + (p >> 32) * N3) * N2 & 0xFFFFFFFF
        x ^= x >> 14
        x = x * N3 & 0xFFFFFFFF
        out[i] = x ^ x >> 16
    return out


# ---- AdamW -----------------------------------------------------------------------------------
def adamw(p, g, m, v, lr, b1, b2, eps, step, decay, c=1.0):
    """(p, m, v) after one step, all binary64."""
    g = g * c
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    hat = (m / (1 - b1 ** step)) / (np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps)
    return p * (1 - lr * decay) - lr * hat, m, v


def round_first(x, r16):
    """x in [-448, 448]: (value rounded so that its mean is x, distance of the draw from the point where it turns)."""
    a = np.abs(x)
    i = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 126)
    step = np.where(i < 126, GRID[np.minimum(i + 1, 126)] - GRID[i], 32.0)
    t = (a - GRID[i]) / step + (r16 * 16 + 8) / 2.0 ** 20
    out = GRID[i] + step * (t >= 1)
    return np.where(x < 0, -out, out), np.abs(t - 1)


def round_second(x, r16):
    """x in [0, 448]: rounded so that the mean of the square is x^2, never to 0 from above 0."""
    i = np.clip(np.searchsorted(GRID, x, side="right") - 1, 0, 126)
    a = GRID[i]
    b = np.where(i < 126, GRID[np.minimum(i + 1, 126)], 480.0)
    share = (x * x - a * a) / (b * b - a * a)
    u = (r16 + 0.5) / 65536.0
    out = np.where(u < share, b, a)
    return np.where(x > 0, np.maximum(out, GRID[1]), out), np.abs(u - share)
