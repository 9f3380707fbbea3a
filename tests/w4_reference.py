"""Plain definitions of 4-bit weights with group scales, in numpy: quantization, the order of the codes in memory, products."""
import numpy as np


def quantize(W, group):
    """(codes [rows, cols], scales [rows, groups], zero points [rows, groups]): whole numbers and fp32."""
    W = np.asarray(W, np.float32)
    rows, cols = W.shape
    ng = -(-cols // group)
    codes, s, z = np.zeros((rows, cols), np.uint8), np.ones((rows, ng), np.float32), np.zeros((rows, ng), np.uint8)
    for r in range(rows):
        for g in range(ng):
            x = W[r, g * group:(g + 1) * group].astype(np.float64)
            f = x[np.isfinite(x)]
            lo, hi = min(0.0, f.min(initial=0.0)), max(0.0, f.max(initial=0.0))
            if max(hi, -lo) < 2.0 ** -100:
                continue
            # the rounded range as fp32 has it, without passing its largest value
            d = np.float32(np.float64(hi) / 16 - np.float64(lo) / 16)
            t = np.float32(np.float64(d) / 15.0)
            bits = (int(t.view(np.uint32)) + 0xFFFF) & 0xFFFF0000
            sc = np.float64(np.uint32(bits).view(np.float32)) * 16
            zz = np.rint(np.float32(-lo / sc))
            x = np.where(np.isnan(x), 0.0, x)
            with np.errstate(over="ignore"):
                q = np.rint((x / sc).astype(np.float32)) + zz
            codes[r, g * group:(g + 1) * group] = np.clip(q, 0, 15)
            s[r, g], z[r, g] = sc, zz
    return codes, s, z


def values(codes, s, z, group):
    cols = codes.shape[1]
    at = np.arange(cols) // group
    return (codes.astype(np.float64) - z[:, at]) * s.astype(np.float64)[:, at]


def pack(codes, z, group, ld):
    """Codes in the order that memory has them: [rows, ld] bytes; past the columns the zero point, past the last group 0."""
    rows, cols = codes.shape
    full = np.zeros((rows, 2 * ld), np.uint32)
    full[:, :cols] = codes
    end = min(2 * ld, z.shape[1] * group)
    full[:, cols:end] = z[:, np.arange(cols, end) // group]
    words = np.zeros((rows, ld // 4), np.uint32)
    for k in range(2 * ld):
        b, t, g, e = k // 128, k % 128 // 32, k % 32 // 8, k % 8
        words[:, 16 * b + 4 * g + t] |= full[:, k] << np.uint32(4 * (e // 2) + 16 * (e % 2))
    return words.view(np.uint8).reshape(rows, ld)


def words(s, z, lds):
    out = np.full((s.shape[0], lds), np.float32(1.0).view(np.uint32))
    out[:, :s.shape[1]] = s.view(np.uint32) | z
    return out


def unpack(data, cols):
    """Codes [rows, cols] from memory."""
    w = np.ascontiguousarray(data).view(np.uint32)
    out = np.zeros((w.shape[0], cols), np.uint8)
    for k in range(cols):
        b, t, g, e = k // 128, k % 128 // 32, k % 32 // 8, k % 8
        out[:, k] = (w[:, 16 * b + 4 * g + t] >> np.uint32(4 * (e // 2) + 16 * (e % 2))) & 15
    return out


def tolerance(wv, xv, y, group):
    """What a product may be off.  A value of X is held within 2^-22 of itself or 2^-38 of its vector's largest; the K products of each of
    its two parts are exact and summed in fp32 in an order that the matrix cores choose, each addition off by at most 2^-23 of a
    partial sum, which the magnitudes bound; the groups' sums take three more operations each, scale and bias two."""
    K, ng = wv.shape[1], -(-wv.shape[1] // group)
    m = np.abs(xv) @ np.abs(wv).T
    far = 2.0 ** -38 * np.abs(xv).max(1, keepdims=True) * np.abs(wv).sum(1)[None, :]
    return ((K + 3 * ng + 2) * 2.0 ** -23 + 2.0 ** -22) * m + far + 2.0 ** -23 * np.abs(y)
