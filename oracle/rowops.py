"""Oracle for the row operators of a transformer's training step: layer normalisation's gradients, activation
checkpoints in 8 bits, embedding lookup and its gradient.  Plain numpy in float64 (checkpoints: exact), from the
operators' definitions in include/delta.h; shares no code with the GPU tree.

Pins: tests/test_oracle_rowops.py (differences, closed forms, hand-made blocks).
"""
import numpy as np

BLOCK = 32
MOST = {"int8": 127.0, "e4m3": 448.0}


def layernorm(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    c = x - x.mean(axis=1, keepdims=True)
    return c / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps) * gamma + beta


def layernorm_bwd(x, gy, gamma, eps, add=None):
    """(gx, dgamma, dbeta) of rows x [M, C]."""
    x, gy, gamma = (np.asarray(a, np.float64) for a in (x, gy, gamma))
    C = x.shape[1]
    c = x - x.sum(axis=1, keepdims=True) / C
    r = 1.0 / np.sqrt((c * c).sum(axis=1, keepdims=True) / C + eps)
    xh = c * r
    g = gy * gamma
    gx = r * (g - g.sum(axis=1, keepdims=True) / C - xh * (g * xh).sum(axis=1, keepdims=True) / C)
    if add is not None:
        gx = gx + np.asarray(add, np.float64)
    return gx, (gy * xh).sum(axis=0), gy.sum(axis=0)


def _e4m3_values():
    """The 127 non-negative numbers of OCP E4M3, by code: 0 .. 126 (127 is NaN)."""
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7))
    return np.array(v)


E4M3 = _e4m3_values()


def _nearest_e4m3(a):
    """Codes of the E4M3 numbers nearest to a >= 0, ties to the even code."""
    hi = np.clip(np.searchsorted(E4M3, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0))
    return np.where(take_hi, hi, lo)


def pack(x, fmt):
    """(payload uint8 [M, C], scale bytes uint8 [M, ceil(C / 32)]) of float x [M, C].  The payload of a block with the
    scale byte 255 is unspecified (zeros here)."""
    x = np.asarray(x, np.float64)
    M, C = x.shape
    nb = -(-C // BLOCK)
    pay, sc = np.zeros((M, C), np.uint8), np.zeros((M, nb), np.uint8)
    for b in range(nb):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        bad = ~np.isfinite(v).all(axis=1)
        v = np.where(bad[:, None], 0.0, v)
        amax = np.abs(v).max(axis=1)
        e = np.full(M, -120)
        while (amax > MOST[fmt] * np.exp2(e)).any():            # the smallest exponent that leaves no value too large
            e = np.where(amax > MOST[fmt] * np.exp2(e), e + 1, e)
        q = v / np.exp2(e)[:, None]
        if fmt == "int8":
            pay[:, b * BLOCK:(b + 1) * BLOCK] = np.rint(q).astype(np.int8).view(np.uint8)
        else:
            pay[:, b * BLOCK:(b + 1) * BLOCK] = _nearest_e4m3(np.abs(q)).astype(np.uint8) | (np.signbit(v).astype(np.uint8) << 7)
        sc[:, b] = np.where(bad, 255, e + 127)
    return pay, sc


def unpack(pay, sc, fmt):
    """float64 values of a checkpoint."""
    C = pay.shape[1]
    s = np.where(sc == 255, np.nan, np.exp2(sc.astype(np.float64) - 127))
    s = np.repeat(s, BLOCK, axis=1)[:, :C]
    if fmt == "int8":
        return np.ascontiguousarray(pay).view(np.int8).astype(np.float64) * s
    return np.where(pay & 0x80, -1.0, 1.0) * np.append(E4M3, np.nan)[pay & 0x7F] * s


def packed_bytes(rows, C):
    up16 = lambda n: (n + 15) // 16 * 16                        # noqa: E731
    return up16(rows * C) + up16(rows * -(-C // BLOCK))


def split_packed(buf, rows, C):
    """A checkpoint's bytes as (payload, scale bytes)."""
    nb, at = -(-C // BLOCK), (rows * C + 15) // 16 * 16
    return buf[:rows * C].reshape(rows, C), buf[at:at + rows * nb].reshape(rows, nb)


def embedding(ids, w, scale):
    """Rows of w [V, C] by ids, times scale [C], float64; zeros for ids outside [0, V)."""
    ids = np.asarray(ids).reshape(-1)
    there = (ids >= 0) & (ids < w.shape[0])
    return np.where(there[:, None], np.asarray(w, np.float64)[np.where(there, ids, 0)] * scale, 0.0)


def embedding_bwd(ids, gy, scale, V):
    ids = np.asarray(ids).reshape(-1)
    gw = np.zeros((V, gy.shape[1]))
    there = (ids >= 0) & (ids < V)
    np.add.at(gw, ids[there], np.asarray(gy, np.float64)[there])
    return gw * scale
