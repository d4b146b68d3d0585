"""The states in 8 bits, written from their definition in include/flround.h with numpy in
64 bits: values of codes by formula, codes by search among all of them."""
import numpy as np

UNIT, BLOCK = 512, 64
TOP_M, TOP_V = 15, 31


def table(top):
    """What the magnitudes 0 .. 8 top + 6 stand for, times 2^(127 - b)."""
    out = []
    for code in range(8 * top + 7):
        e, m = code >> 3, code & 7
        out.append(2.0 ** (e - top) * (1 + m / 8) if e else 2.0 ** (1 - top) * m / 8)
    return np.array(out)


def decode(codes, exps, top):
    codes = codes.astype(np.int64).reshape(-1, BLOCK)
    sign = np.where(codes >= 128, -1.0, 1.0) if top == TOP_M else 1.0
    k = codes & 127 if top == TOP_M else codes
    t = np.append(table(top), np.nan)
    with np.errstate(over="ignore"):
        return (sign * t[k] * 2.0 ** (exps.astype(np.float64) - 127)[:, None]).astype(np.float32).ravel()


def exponent(x):
    """The exponent byte of each block of x (float32)."""
    a = np.abs(x.reshape(-1, BLOCK).astype(np.float64))
    most = np.where(np.isfinite(a), a, 0.0).max(1)
    b = np.zeros(len(most), dtype=np.int64)
    some = most >= 2.0 ** -126
    f, e = np.frexp(most[some])
    b[some] = e - 1 + 127 + (f > 0.875)
    return np.maximum(b, 12)


def encode(x, top, draws=None):
    """Codes and exponent bytes of x; draws: 20 bits for each element, or to nearest."""
    b = exponent(x)
    x = x.reshape(-1, BLOCK)
    a = np.abs(x.astype(np.float64))
    fine = np.isfinite(a)
    t = table(top)
    y = np.where(fine, a, 0.0) * 2.0 ** (127 - b)[:, None]
    small = t[1]                                     # places are held to 2^-20 of a step
    y = np.rint(y / small * 2.0 ** 20) / 2.0 ** 20 * small
    lo = np.clip(np.searchsorted(t, y, side="right") - 1, 0, len(t) - 2)
    place = (y - t[lo]) / (t[lo + 1] - t[lo])
    if draws is None:
        up = (place > 0.5) | ((place == 0.5) & (lo % 2 == 1))
    else:
        up = place + draws.reshape(-1, BLOCK) * 2.0 ** -20 >= 1.0
    code = lo + up
    if top == TOP_V:
        code = np.where(a > 0, np.maximum(code, 1), code)
    code = np.where(fine, code, 8 * top + 7)
    if top == TOP_M:
        code = code | np.signbit(x).astype(np.int64) << 7
    return code.astype(np.uint8).ravel(), b.astype(np.uint8)


def draws(n, seed, step, first=0):
    """The random bits of elements first .. first + n - 1: for m and for v."""
    key = (seed * 0x9E3779B97F4A7C15 + step * 0xD1B54A32D192ED03) % 2 ** 64
    m32 = np.uint64(0xFFFFFFFF)
    i = np.arange(first, first + n, dtype=np.uint64)
    s = np.uint64
    x = (i & m32) ^ s(key & 0xFFFFFFFF)
    x = ((x ^ (x >> s(16))) * s(0x7FEB352D)) & m32
    x = x ^ (((i >> s(32)) + s(key >> 32)) & m32)
    x = ((x ^ (x >> s(15))) * s(0x846CA68B)) & m32
    x = x ^ (x >> s(16))
    return (x >> s(12)).astype(np.float64), (((x * s(0x9E3779B1)) & m32) >> s(12)).astype(np.float64)


def split(state, n):
    """m's codes, v's, m's exponent bytes, v's."""
    k = n // BLOCK
    return state[:n], state[n:2 * n], state[2 * n:2 * n + k], state[2 * n + k:]
