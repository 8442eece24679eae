"""Float64 numpy definitions of training in 8 bits: quantised matrices, their product, AdamW with states in 32 or 8 bits.
Written from the formulas; shares no code with the GPU path."""
from __future__ import annotations

import numpy as np

FORMATS = {"e4m3": (4, 3, 448.0), "e5m2": (5, 2, 57344.0)}  # exponent bits, fraction bits, largest finite value


def code_values(fmt):
    """The 256 values of a format's codes, from the meaning of sign, exponent and fraction."""
    eb, mb, _ = FORMATS[fmt]
    bias = 2 ** (eb - 1) - 1
    out = np.empty(256)
    for code in range(256):
        sign, exp, frac = code >> 7, (code >> mb) & (2 ** eb - 1), code & (2 ** mb - 1)
        v = frac * 2.0 ** (1 - bias - mb) if exp == 0 else (1 + frac / 2 ** mb) * 2.0 ** (exp - bias)
        if fmt == "e4m3" and (exp, frac) == (15, 7):
            v = np.nan
        if fmt == "e5m2" and exp == 31:
            v = np.inf if frac == 0 else np.nan
        out[code] = -v if sign else v
    return out


def encode(x, fmt):
    """Nearest codes, ties to the even one; |x| at most the largest finite value, or not finite."""
    v = code_values(fmt)[:128]
    top = int(np.sum(v <= FORMATS[fmt][2]))
    v, a = v[:top], np.abs(x)
    fin = np.where(np.isfinite(a), a, 0.0)
    hi = np.clip(np.searchsorted(v, fin), 1, top - 1)
    lo = hi - 1
    up = (fin - v[lo] > v[hi] - fin) | ((fin - v[lo] == v[hi] - fin) & (hi % 2 == 0))
    code = np.where(up, hi, lo)
    nan_code = 0x7F
    code = np.where(np.isnan(a) | (np.isinf(a) & (fmt == "e4m3")), nan_code, np.where(np.isinf(a), 0x7C, code))
    return (code | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def _block_max(x, block_rows):
    r, c = x.shape
    sr, sc = -(-r // block_rows), -(-c // 128)
    out = np.zeros((sr, sc))
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    for j in range(sc):
        m = a[:, j * 128:(j + 1) * 128].max(1)
        out[:, j] = [m[i * block_rows:(i + 1) * block_rows].max() for i in range(sr)]
    return out


def scale_bytes(biggest, fmt):
    """Exponents of the smallest powers of two s with biggest / s <= the largest finite value, 2^-127 at least."""
    out = np.full(biggest.shape, 127, dtype=np.int64)
    for at, b in np.ndenumerate(biggest):
        if b > 0:
            e = -200
            while b > FORMATS[fmt][2] * 2.0 ** e:
                e += 1
            out[at] = max(e, -127) + 127
    return out.astype(np.uint8)


def spread(scale, rows, cols):
    """A quantised matrix's scales as factors of its elements."""
    s = 2.0 ** (scale.astype(np.float64) - 127)
    if s.shape[0] != rows:
        s = np.repeat(s, 128, 0)[:rows]
    return np.repeat(s, 128, 1)[:, :cols]


def quantize(x, fmt, block_rows):
    s = scale_bytes(_block_max(x, block_rows), fmt)
    return encode(x / spread(s, *x.shape), fmt), s


def values(codes, scale, fmt):
    return code_values(fmt)[codes] * spread(scale, *codes.shape)


def _mix32(x):
    x = np.asarray(x, dtype=np.uint64)
    m = np.uint64(0xFFFFFFFF)
    for shift, mul in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        x = x ^ (x >> np.uint64(shift))
        x = (x * np.uint64(mul)) & m
    return x ^ (x >> np.uint64(16))


def random_parts(n, index, step, seed, first=0):
    """The two 16-bit fractions of n elements from `first` on, of m and of sqrt(v)."""
    lo, hi = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    key = _mix32(int(_mix32(lo ^ step)) ^ ((index * 0x9E3779B9) & 0xFFFFFFFF))
    i = np.arange(first, first + n, dtype=np.uint64)
    h = _mix32(_mix32(key ^ ((i >> np.uint64(7)) & np.uint64(0xFFFFFFFF)) ^ np.uint64(hi)) ^ (i & np.uint64(127)))
    return (h & np.uint64(0xFFFF)) / 65536.0, (h >> np.uint64(16)) / 65536.0


def steps_of(x):
    """(scale bytes, |x| / (the type's step there), the step as a value) of states in blocks of 128."""
    pad = -len(x) % 128
    b = np.pad(np.where(np.isfinite(x), np.abs(x), 0.0), (0, pad)).reshape(-1, 128).max(1)
    s = scale_bytes(b, "e4m3")
    scale = np.repeat(2.0 ** (s.astype(np.float64) - 127), 128)[:len(x)]
    y = np.abs(x) / scale
    step = 2.0 ** (np.floor(np.log2(np.clip(y, 2.0 ** -6, None))) - 3)
    return s, y / step, step * scale


def adamw(p, g, m, v, *, step, lr, beta1, beta2, eps, weight_decay):
    """(p, m, v) after one step; v is the second moment itself."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * weight_decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v
