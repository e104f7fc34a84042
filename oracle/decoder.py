"""Oracle for a decoder layer's operators: root-mean-square normalisation, rotary positions, attention over packed sequences with grouped
heads, log probabilities of given tokens, and their gradients.  Plain numpy in float64, from the operators' definitions in include/delta.h; shares no code
with the GPU tree.

Pins: tests/test_oracle_decoder.py (differences, closed forms, hand-made cases).
"""
import numpy as np


def rmsnorm(s, gamma, eps):
    s = np.asarray(s, np.float64)
    return s / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps) * gamma


def rmsnorm_bwd(s, gy, gamma, eps, add=None):
    """(gx, dgamma) of rows s [M, C]."""
    s, gy = np.asarray(s, np.float64), np.asarray(gy, np.float64)
    r = 1.0 / np.sqrt((s * s).sum(axis=1, keepdims=True) / s.shape[1] + eps)
    sh, g = s * r, gy * np.asarray(gamma, np.float64)
    gx = r * (g - sh * (g * sh).sum(axis=1, keepdims=True) / s.shape[1])
    return (gx if add is None else gx + np.asarray(add, np.float64)), (gy * sh).sum(axis=0)


def angles(pos, freq):
    """theta [M, D / 2] of positions [M, A] and frequencies [A, D / 2], reduced to a turn by whole numbers where that matters: positions are whole, a
    frequency is a whole number of 2^-k."""
    pos, freq = np.asarray(pos, np.int64).reshape(len(pos), -1), np.asarray(freq, np.float32)
    return (pos.astype(np.longdouble)[:, :, None] * freq.astype(np.longdouble)[None]).sum(axis=1)


def rotary(x, theta, heads, D, pairs):
    """x [M, W]: the first `heads` heads of D channels turned by theta, the rest as it is."""
    x = np.array(x, np.float64)
    M, half = len(x), D // 2
    c, s = np.cos(theta).astype(np.float64), np.sin(theta).astype(np.float64)
    for h in range(heads):
        b = x[:, h * D:(h + 1) * D]
        lo, hi = (slice(0, D, 2), slice(1, D, 2)) if pairs else (slice(0, half), slice(half, D))
        u, v = b[:, lo].copy(), b[:, hi].copy()
        b[:, lo], b[:, hi] = u * c - v * s, u * s + v * c
    return x


def attention(x, off, heads, kv, D, causal, gy=None):
    """x [M, (heads + 2 kv) D], sequences off[i] .. off[i + 1].  Returns a dict: y [M, heads D], lse [heads, M], with gy also gx (as x) and what bounds of errors
    need: pv = sum p |v|, A = the largest sum of |q k| / sqrt(D) of a row's scores, and per element of gx `slack`(rel_p, rel_ds, dp_err, delta_err)."""
    x = np.asarray(x, np.float64)
    M = len(x)
    o = dict(y=np.zeros((M, heads * D)), lse=np.zeros((heads, M)), pv=np.zeros((M, heads * D)), A=np.zeros((heads, M)), gx=np.zeros(x.shape), parts=[])
    for a, b in zip(off, off[1:]):
        if a >= b:
            continue
        for h in range(heads):
            j = h // (heads // kv)
            cq, ck, cv = (slice(i * D, (i + 1) * D) for i in (h, heads + j, heads + kv + j))
            q, k, v = x[a:b, cq], x[a:b, ck], x[a:b, cv]
            s = (q @ k.T) / np.sqrt(float(D))
            keep = np.tril(np.ones((b - a, b - a), bool)) if causal else np.ones((b - a, b - a), bool)
            s = np.where(keep, s, -np.inf)
            m = s.max(axis=1, keepdims=True)
            e = np.exp(s - m)
            p = e / e.sum(axis=1, keepdims=True)
            o["y"][a:b, cq] = p @ v
            o["lse"][h, a:b] = (m + np.log(e.sum(axis=1, keepdims=True)))[:, 0]
            o["pv"][a:b, cq] = p @ np.abs(v)
            o["A"][h, a:b] = (np.abs(q) @ np.abs(k).T / np.sqrt(float(D))).max(axis=1)
            if gy is None:
                continue
            g = np.asarray(gy, np.float64)[a:b, cq]
            dp = g @ v.T
            delta = (g * o["y"][a:b, cq]).sum(axis=1, keepdims=True)
            ds = np.where(keep, p * (dp - delta), 0.0) / np.sqrt(float(D))
            o["gx"][a:b, cq] += ds @ k
            o["gx"][a:b, ck] += ds.T @ q
            o["gx"][a:b, cv] += p.T @ g
            o["parts"].append(dict(rows=slice(a, b), h=h, cq=cq, ck=ck, cv=cv, p=p, dp=dp, delta=delta, ds=ds, g=g, q=q, k=k, v=v))
    return o


def _order(z):
    """Sort key of logits, descending: NaN above all, -0 as 0."""
    z = np.asarray(z, np.float64) + 0.0
    return np.where(np.isnan(z), np.inf, z), np.isnan(z)


def logprob(z, ids, K=0):
    """(y [3, M], best [M, K], which [M, K]) of logits z [M, V]."""
    z = np.asarray(z, np.float64)
    M, V = z.shape
    y, best, which = np.zeros((3, M)), np.zeros((M, K)), np.full((M, K), -1, np.int64)
    with np.errstate(invalid="ignore", divide="ignore"):
        for r in range(M):
            if not 0 <= ids[r] < V:
                continue
            v, nan = _order(z[r])
            which[r] = np.lexsort((np.arange(V), -v, ~nan))[:K]
            if (z[r] == -np.inf).all():
                y[:, r] = -np.inf, 0.0, -np.inf
                best[r] = -np.inf
                continue
            if np.isnan(z[r]).any() or (z[r] == np.inf).any():
                y[:, r] = np.nan
                best[r] = np.nan
                continue
            m = z[r].max()
            e = np.exp(z[r] - m)
            logs = np.log(e.sum())
            y[0, r] = (z[r, ids[r]] - m) - logs
            y[1, r] = logs + (e * np.where(e > 0, m - z[r], 0.0)).sum() / e.sum()
            y[2, r] = m + logs
            best[r] = (z[r, which[r]] - m) - logs
    return y, best, which


def logprob_bwd(z, ids, gy):
    """gz of logits z [M, V] and gy [3, M]."""
    z = np.asarray(z, np.float64)
    gz = np.zeros(z.shape)
    y, _, _ = logprob(z, ids)
    with np.errstate(invalid="ignore"):
        for r in range(len(z)):
            if not 0 <= ids[r] < z.shape[1] or y[2, r] == -np.inf:
                continue
            lp = z[r] - y[2, r]
            p = np.exp(lp)
            t = np.where(p > 0, p * (gy[2, r] - gy[0, r] - gy[1, r] * (np.where(p > 0, lp, 0.0) + y[1, r])), 0.0 * p)
            t[ids[r]] += gy[0, r]
            gz[r] = t
    return gz
