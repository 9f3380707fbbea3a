"""Plain definitions in 64 bits of the 8-bit floating point operators and of the drawing of tokens (numpy)."""
import math

import numpy as np

BLOCK = 128


def e4m3_values():
    """The value of every code (0x7f and 0xff: NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v = np.where(c & 128, -v, v)
    v[[127, 255]] = np.nan
    return v


VALUES = e4m3_values()


def e4m3_round(q):
    """The code nearest to q, |q| <= 448, ties to even; NaN for what is not finite."""
    q = np.asarray(q, np.float64)
    with np.errstate(invalid="ignore"):
        a = np.where(np.isfinite(q), np.abs(q), 0.0)
        _, ex = np.frexp(np.maximum(a, 2.0 ** -6))
        step = np.ldexp(1.0, ex - 4)
        n = np.rint(a / step).astype(np.int64)             # 0 .. 16 steps
    e = np.maximum(ex - 1, -6) + 7                        # exponent field of a normal value
    code = np.where(n < 8, n, ((e << 3) + (n - 8)))       # n == 16 carries into the exponent by itself
    code = np.where(np.signbit(q), code | 128, code)
    return np.where(np.isfinite(q), code, np.where(np.signbit(q), 255, 127)).astype(np.uint8)


def quantize(X, ld=None, lds=None):
    """(codes [rows, ld], scale bytes [rows, lds])."""
    X = np.asarray(X, np.float32)
    rows, cols = X.shape
    nb = -(-cols // BLOCK)
    ld = -(-cols // 16) * 16 if ld is None else ld
    lds = -(-nb // 4) * 4 if lds is None else lds
    codes, scale = np.zeros((rows, ld), np.uint8), np.full((rows, lds), 127, np.uint8)
    for b in range(nb):
        x = X[:, b * BLOCK:(b + 1) * BLOCK].astype(np.float64)
        m = np.where(np.isfinite(x), np.abs(x), 0.0).max(1)
        mant, ex = np.frexp(m)
        e = ex - 9 + (mant > 0.875)
        none = m < 2.0 ** -100
        e = np.where(none, 0, e)
        with np.errstate(invalid="ignore"):
            q = np.ldexp(x, -e[:, None])
        q = np.where(none[:, None] & np.isfinite(q), 0.0, q)
        codes[:, b * BLOCK:b * BLOCK + x.shape[1]] = e4m3_round(q)
        scale[:, b] = (e + 127).astype(np.uint8)
    return codes, scale


def values(codes, scale, cols):
    """What codes and scales stand for, [rows, cols] in double."""
    s = np.ldexp(1.0, scale.astype(np.int64) - 127)
    return VALUES[codes[:, :cols]] * np.repeat(s, BLOCK, axis=1)[:, :cols]


def draw(v, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability, margin) of one row: the margin is how far u times the kept mass lies from the nearest border
    between two tokens, and a kept border from its neighbours, in units of the row's whole mass."""
    v = np.asarray(v, np.float32)
    live = np.flatnonzero(~np.isnan(v) & (v > -np.inf))
    if not len(live):
        return -1, -np.inf, np.inf
    x = v[live].astype(np.float64) + 0.0
    order = np.lexsort((live, -x))
    x, live = x[order], live[order]
    gap = np.zeros(len(x))
    np.subtract(x[0], x, out=gap, where=x != x[0])
    lse = math.log(math.fsum(np.exp(-gap)))
    T, u, top_p, min_p = (float(np.float32(t)) for t in (T, u, top_p, min_p))
    if not T > 0:
        return int(live[0]), -lse, np.inf
    g = np.zeros(len(gap)) if math.isinf(T) else gap / T
    w = np.exp(-np.where(np.isinf(gap), np.inf, g))
    total, margin = w.sum(), np.inf
    if top_k > 0:
        w = w[:top_k]
    cum = np.cumsum(w)
    m = len(w)
    if top_p < 1:
        need = top_p * cum[-1]
        m = max(1, min(m, int(np.searchsorted(cum, need, side="left")) + 1))
        margin = min(margin, np.abs(cum - need).min() / total) if top_p > 0 else margin
    if min_p > 0:
        m = max(1, min(m, int((w >= min_p).sum())))
        margin = min(margin, np.abs(w - min_p)[gap[:len(w)] > 0].min(initial=np.inf))     # (the best word's weight is 1 exactly)
    u = min(max(u, 0.0) if u == u else 0.0, 1 - 2.0 ** -24)
    need = u * cum[m - 1]
    at = min(int(np.searchsorted(cum[:m], need, side="right")), m - 1)
    margin = min(margin, np.abs(cum[:m] - need).min() / total) if u > 0 else margin
    return int(live[at]), -gap[at] - lse, margin
