"""What the GPU tests of the decoder operators share: an operator run through a context on given arrays, and bounds on what its arithmetic may add."""
import numpy as np

from rowops_util import EPS24, Bench, half_step, storage, values

HALF_BF16 = 2.0 ** -8
TINY = 2.0 ** -126


def rmsnorm_noise(s, gy, gamma, eps):
    """Bounds on what fp32 adds: to y relative to |y|, to gx per row, to dgamma per channel.  A sum of n values of a sign in a tree of depth <= 40 is off by
    40 e relative, r by half of that and three roundings, sh by 24 e relative; mean(g sh) by 40 e G plus G times that of sh (mean |sh| <= 1), gx / r by
    the sum of its two terms' errors, the second's size being at most H G."""
    s, gy = np.asarray(s, np.float64), np.asarray(gy, np.float64)
    r = 1.0 / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    sh = s * r
    H, G = np.abs(sh).max(axis=1, keepdims=True), np.abs(gy * gamma).max(axis=1, keepdims=True)
    e = 40 * EPS24
    depth = (s.shape[0] / 8 + 80) * EPS24
    return 26 * EPS24, r * e * G * (1 + 3 * H), ((depth + 24 * EPS24) * np.abs(gy * sh)).sum(axis=0)


def run_rmsnorm(torch, x, res, gamma, eps, dtype, pack=0, gy=None, add=None, gx=True, gw=True, stream=None):
    """Returns (bench, dict of outputs): y, sum, held (bytes), gx, gw as stored arrays."""
    import paper_2203_15980_amd as dl
    M, C = x.shape
    es = 4 if dtype == "f32" else 2
    d = dl.Delta()
    held = d.packed_bytes(M, C)
    d.close()
    b = Bench(torch, [M * C * es] * 7 + [held], stream=stream)          # x, res, y, sum, gy, add, gx, checkpoint
    b.put(0, storage(x, dtype))
    if res is not None:
        b.put(1, storage(res, dtype))
    dg = b.dev(np.asarray(gamma, np.float32))
    L = b.layer(dl.OP_RMSNORM, M, C, C, 0, 2, dtype, res=1 if res is not None else dl.NO_TENSOR, y2=3 if res is not None else dl.NO_TENSOR,
                y3=7 if pack else dl.NO_TENSOR, pack=pack, scale=dg.data_ptr(), eps=eps)
    b.d.recompute_segment([L])
    t = np.float32 if dtype == "f32" else np.uint16
    o = dict(y=b.get(2, t, (M, C)).copy(), L=L)
    o["sum"] = b.get(3, t, (M, C)).copy() if res is not None else storage(x, dtype)
    o["held"] = b.get(7, np.uint8, (held,)).copy() if pack else None
    if gy is not None:
        b.put(4, storage(gy, dtype))
        if add is not None:
            b.put(5, storage(add, dtype))
        ws, whole = b.workspace(b.d.backward_workspace(L))
        out, guard = b.guarded(C)
        b.d.backward_segment([b.bwd(L, 4, gx=6 if gx else None, add=5 if add is not None else None, gw=out if gw else None, ws=ws)])
        o["gx"] = b.get(6, t, (M, C)).copy()
        o["gw"] = out.cpu().numpy().astype(np.float64)
        g = guard.cpu().numpy()
        assert (g[:64] == 12345.0).all() and (g[64 + C:] == 12345.0).all()
        assert (whole[ws.numel():].cpu().numpy() == 0x7F).all()
    return b, o


def run_attention(torch, x, off, heads, kv, D, causal, gy=None, stream=None, keep=False):
    """x: bf16 bits [M, W].  Returns (bench, dict): y, lse, gx in float64."""
    import paper_2203_15980_amd as dl
    M, W = x.shape
    b = Bench(torch, [M * W * 2, len(off) * 8, M * heads * D * 2, M * heads * 4, M * heads * D * 2, M * W * 2], stream=stream)   # x, off, y, lse, gy, gx
    b.put(0, x)
    b.put(1, np.asarray(off, np.int64))
    L = b.layer(dl.OP_ATTENTION_PACKED, M, W, heads * D, 0, 2, res=1, y2=3, y3=dl.NO_TENSOR, R=heads, S=kv, flags=dl.ATTENTION_CAUSAL if causal else 0)
    b.d.recompute_segment([L])
    o = dict(L=L, y=values(b.get(2, np.uint16, (M, heads * D)), "bf16"), lse=b.get(3, np.float32, (heads, M)).astype(np.float64))
    if gy is not None:
        b.put(4, gy)
        ws, whole = b.workspace(b.d.backward_workspace(L))
        o["bwd"] = b.bwd(L, 4, gx=5, ws=ws)
        b.d.backward_segment([o["bwd"]])
        o["gx"] = values(b.get(5, np.uint16, (M, W)), "bf16")
        assert (whole[ws.numel():].cpu().numpy() == 0x7F).all()
    return b, o


def check_attention(o, ref, heads, D, longest, backward=True):
    """o from run_attention against ref from oracle.decoder.attention (float64 on the same bf16 inputs).

    Forward: a score is a sum of D products in fp32, off by (D + 2) e A with A = the largest sum |q k| / sqrt(D) of the row, and by two roundings on
    its way into 2^x; p then is off by that (doubled: its own score's and the maximum's) relative, and by 2^-8 where bf16 holds it; the sum of n
    weights by n e.  y is off by that share of sum p |v| and by its own rounding, the log-sum-exp by the scores' error and n e.
    Backward: p also by the stored log-sum-exp's error; delta by the error of the stored y; ds by all of these and 2^-8.
    Numbers below 2^-126, the smallest normal one, may be held as zero: a p by the exponential (2^-126 |dp - delta| of a ds, 2^-126 |g| of a term of gv), a ds where
    it becomes bf16 (2^-126, before 1 / sqrt(D)), a gradient where it does."""
    e_s = 2 * (D + 8) * EPS24 * (ref["A"] + 1)                                      # [heads, M]
    n = (longest + 16) * EPS24
    per = lambda a: np.repeat(a.T, D, axis=1)                                       # noqa: E731
    tol_y = HALF_BF16 * np.abs(ref["y"]) + (HALF_BF16 + per(e_s) + n) * ref["pv"] * 1.02
    assert (np.abs(o["y"] - ref["y"]) <= tol_y).all(), float((np.abs(o["y"] - ref["y"]) / np.maximum(tol_y, 1e-300)).max())
    tol_l = e_s + n + 4 * EPS24 * np.abs(ref["lse"])
    assert (np.abs(o["lse"] - ref["lse"]) <= tol_l).all(), float((np.abs(o["lse"] - ref["lse"]) / np.maximum(tol_l, 1e-300)).max())
    if not backward:
        return
    tol = HALF_BF16 * np.abs(ref["gx"]) + TINY
    sums = n + 2 * EPS24                                                           # sums of n products in fp32 (a group's: at most 16 times as many)
    for t in ref["parts"]:
        rows, h = t["rows"], t["h"]
        e_p = (2 * e_s[h, rows] + tol_l[h, rows] + 4 * EPS24)[:, None]
        d_dp = (D + 2) * EPS24 * (np.abs(t["g"]) @ np.abs(t["v"]).T)
        d_delta = (np.abs(t["g"]) * tol_y[rows, t["cq"]]).sum(axis=1, keepdims=True) + (D + 2) * EPS24 * (np.abs(t["g"]) * np.abs(ref["y"][rows, t["cq"]])).sum(axis=1, keepdims=True)
        sc = 1 / np.sqrt(float(D))
        err = np.abs(t["ds"]) * (HALF_BF16 + e_p + 16 * sums) + t["p"] * sc * 1.02 * (d_dp + d_delta) + TINY * sc * (1 + np.abs(t["dp"] - t["delta"]))
        tol[rows, t["cq"]] += err @ np.abs(t["k"])
        tol[rows, t["ck"]] += err.T @ np.abs(t["q"])
        tol[rows, t["cv"]] += (t["p"] * (HALF_BF16 + e_p + 16 * sums) + TINY).T @ np.abs(t["g"])
    bad = np.abs(o["gx"] - ref["gx"]) > 1.01 * tol
    assert not bad.any(), (int(bad.sum()), float((np.abs(o["gx"] - ref["gx"]) / np.maximum(tol, 1e-300))[bad].max()), float(np.abs(o["gx"][bad]).max()), float(np.abs(ref["gx"][bad]).max()))


def logprob_noise(z, ref_y):
    """Bounds on the absolute errors of the three rows of y and of an alternative's log probability at distance d from the maximum.  With d_j = max - z_j,
    W = sum p d: a weight is off by (2 d + 4) e relative (two roundings of its argument, the exponential), the sum s of n weights by
    those and by its depth in e; log s by that, w / s (w = sum d exp(-d)) by twice that of W + 1."""
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore"):
        m = np.max(z, axis=1)
        d = m[:, None] - z
        p = np.where(d < 700, np.exp(-d), 0.0)
        s = p.sum(axis=1)
        W = (p * np.where(p > 0, d, 0.0)).sum(axis=1) / s
        W2 = (p * np.where(p > 0, d * d, 0.0)).sum(axis=1) / s
    rel = (max(64, z.shape[1] / 1024) + 80 + 2 * W + 4) * EPS24
    logs = np.log(s)
    lp = lambda dist: (rel + EPS24 * (4 * logs + 1) + EPS24 * 2 * np.abs(np.asarray(dist).T)).T      # noqa: E731  dist: [M] or [M, K]
    H = rel * (1 + 2 * W) + EPS24 * (4 * logs + 4 * W + 2 * W2 + 2)
    lse = rel + EPS24 * (4 * logs + 2 * np.abs(m) + 1)
    return lp, H, lse


def run_logprob(torch, z, ids, dtype, K=0, gy=None, stream=None):
    """z: stored array [M, V].  Returns (bench, dict): y, best, which, gz."""
    import paper_2203_15980_amd as dl
    M, V = z.shape
    es = 4 if dtype == "f32" else 2
    b = Bench(torch, [M * V * es, M * 8, M * 12, max(M * K * 4, 1), max(M * K * 8, 1), M * 12, M * V * es], stream=stream)   # z, ids, y, best, which, gy, gz
    b.put(0, z)
    b.put(1, np.asarray(ids, np.int64))
    L = b.layer(dl.OP_LOGPROB, M, V, K, 0, 2, dtype, res=1, y2=3 if K else dl.NO_TENSOR, y3=4 if K else dl.NO_TENSOR)
    b.d.recompute_segment([L])
    o = dict(L=L, y=b.get(2, np.float32, (3, M)).astype(np.float64))
    if K:
        o["best"], o["which"] = b.get(3, np.float32, (M, K)).astype(np.float64), b.get(4, np.int64, (M, K)).copy()
    if gy is not None:
        b.put(5, np.asarray(gy, np.float32))
        b.d.backward_segment([b.bwd(L, 5, gx=6)])
        o["gz"] = values(b.get(6, np.float32 if dtype == "f32" else np.uint16, (M, V)), dtype)
    return b, o


__all__ = ["EPS24", "HALF_BF16", "half_step", "storage", "values"]
